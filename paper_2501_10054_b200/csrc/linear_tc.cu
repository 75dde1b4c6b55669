// The products of linear.cuh for bf16 operands on the 5th-generation tensor cores.
//
// The weights are the M side of the MMAs, the rows of x (tokens) the N side: an accumulator has an output channel per TMEM lane and a
// token per column.  N is chosen for every tile (16 .. 256 in steps of 16, in pairs 32), so a group of any size wastes few columns, and the
// tokens of a group are cut into tiles of equal width; with the tokens on the M side every group would be padded to 128 rows.  The epilogue
// comes to 32 neighbouring channels of a token in the 32 lanes of a warp: bias is one value per thread, y and the residual are touched in pieces of 64
// or 128 bytes.
//
// A CTA is persistent: warp 0 stages 128 x 64 (weights) and up to NT x 64 (tokens) boxes with TMA (128-byte swizzle, no multicast), the tokens as boxes
// of 32 rows or, where the rows of a group are picked by an index array, four rows at a time by their indices (tile::gather4, four more warps); warp 1 issues the MMAs into
// one of two accumulators; warps 2 .. 9 run the epilogue of the other.  CTAS = 2: two CTAs share a tile of 256 channels, each with 128 of them and half of
// the tokens in shared memory (cta_group::2).  SPLIT: the CTAs of a cluster share the channels k of a tile; each hands the others the columns that
// they finish through their shared memory, and the owner of a column adds the parts in the order of their ranks: no atomics, no scratch, the same bits
// every time.
//
// PRECISE (fp32 outputs): the tensor cores cut every sum off to 24 bits, towards zero, so that a long row of products loses 1.5e-8 of the sum per instruction, 1.1e-5 with
// 11752 channels; the epilogue warps then take the accumulator over after every 512 channels and add it up in registers, rounded to nearest.  Of outputs of 16 bits that is less than 1/32 of
// their own rounding up to kMostCutOff channels; above, they are computed like this too (in tiles of 64 tokens: in the larger ones both epilogues spill).  That also keeps every wait
// for an accumulator short, whatever the number of channels is.
//
// Every wait on an mbarrier is bounded: when it runs out the CTA stops issuing, fills what it would have written with NaN and ends after its copies have landed.
#include <cuda.h>
#include <math.h>
#include <math_constants.h>

#include "linear.cuh"
#include "tc.cuh"

namespace tardis {
namespace linear {
using namespace tc;

constexpr int BM = 128, BK = 64, BOX = 32;       // channels of a CTA's tile; k per stage; rows per copy of tokens
constexpr int NTHREADS = 320, GATHER_WARPS = 4;
constexpr int PRECISE_BLOCKS = 8;                // k blocks of an accumulator, PRECISE

constexpr int STAGING_LD = 36, STAGING_WARP = 16 * STAGING_LD * 4;    // 16 columns x 32 channels of a warp

template <int CTAS, int NT, int SPLITS> struct Cfg {
  static constexpr int A_BYTES = BM * BK * 2, B_ROWS = NT / CTAS, STAGE_BYTES = A_BYTES + B_ROWS * BK * 2;
  static constexpr int SHARE = (7 + SPLITS) / SPLITS;                // of the 8 quads of columns in a block of 32, how many a CTA of the cluster finishes at most
  static constexpr int PART_LD = NT / 32 * SHARE * 4 + 4;            // floats of a channel in a part (4 apart from a multiple of 8: no bank conflicts)
  static constexpr int EXCHANGE = SPLITS > 1 ? SPLITS * BM * PART_LD * 4 : 0;
  static constexpr int STAGING = SPLITS > 1 ? 0 : 8 * STAGING_WARP;                    // the epilogue's, see finish
  static constexpr int NS = (212 * 1024 - EXCHANGE - STAGING) / STAGE_BYTES;
  static constexpr int TMEM_COLS = 2 * NT;
  static constexpr int STEP = 16 * CTAS;                             // of N
  static_assert(NS >= 4, "");
  static constexpr int FIXED = NS * STAGE_BYTES + EXCHANGE + STAGING + 1024 /* alignment slack */ + 256 /* barriers */;
};

struct Params {
  LinearArgs a;
  int kblocks, band, tokens_fast;
  int wide;                        // y (and the residual) can be stored 16 bytes at a time
};

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
// four rows, one below the other in shared memory (the map's box is one row high)
__device__ __forceinline__ void tma_gather4(void* dst, const CUtensorMap* map, int x, const int (&r)[4], uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tma_gather4_pair(void* dst, const CUtensorMap* map, int x, const int (&r)[4], uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(bar), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ uint32_t in_rank(const void* p, int rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
// a bounded wait of a whole warp for what other CTAs of the cluster have written
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* b, uint32_t parity) {
  uint32_t ok = 0;
  const long long t0 = clock64();
  do {
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
  } while (!ok && clock64() - t0 <= WAIT_CYCLES);
  return __all_sync(0xffffffffu, ok != 0);
}

// One tile as a role sees it.
struct Tile { int e, o0, first, rows, nt, turn; };     // group, first output, first row, rows, columns of the MMA, k block to begin with

// The epilogue takes sixteen columns of a warp's 32 channels o0 .. o0 + 31 at a time through shared memory (`stage`, column-major), `count` of them rows of y
// from `row` on.  Where y and the residual are aligned and all channels are inside, a lane has 8 channels of a token and touches both 16 bytes at a
// time; else its own channel of all sixteen tokens.  The residual of the next sixteen columns is on its way meanwhile.  (Two bytes per lane throughout: the
// epilogue of 1024 x 64 x 16384 with a residual took 51 us, with the residual read when it is needed 35, so 30.)
template <typename O> struct alignas(16) Out8 { O v[8]; };
// Sixteen residuals as words, packed as they lie in memory (wide: eight of token c, eight of c + 8) or one each (one of every token: packing them would wait
// for each in turn)
template <typename O> struct Old {
  uint32_t w[16];
  __device__ __forceinline__ float packed(int i) const {
    return __uint_as_float(sizeof(O) == 4 ? w[i] : i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ float one(int i) const { return __uint_as_float(sizeof(O) == 4 ? w[i] : w[i] << 16); }
};
template <typename O>
__device__ __forceinline__ void read_residual(const LinearArgs& a, bool wide, long long row, int count, int o0, int lane, Old<O>& old) {
  constexpr int HALF = 2 * sizeof(O);                          // words of eight
  if (wide) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < HALF; i += 4)
        if (h * 8 + (lane >> 2) < count) {
          const uint4 v = reinterpret_cast<const uint4*>(static_cast<const O*>(a.res) + (row + h * 8 + (lane >> 2)) * a.ldr + o0 + (lane & 3) * 8)[i / 4];
          old.w[h * HALF + i] = v.x; old.w[h * HALF + i + 1] = v.y; old.w[h * HALF + i + 2] = v.z; old.w[h * HALF + i + 3] = v.w;
        }
  } else {
    const O* const r = static_cast<const O*>(a.res) + row * a.ldr + o0 + lane;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bool there = i < count && o0 + lane < a.o;
      if (sizeof(O) == 4) old.w[i] = there ? *reinterpret_cast<const uint32_t*>(r + i * a.ldr) : 0u;
      else old.w[i] = there ? *reinterpret_cast<const unsigned short*>(r + i * a.ldr) : 0u;
    }
  }
}
template <int ACT, typename O>
__device__ __forceinline__ void finish(const LinearArgs& a, bool wide, long long row, int count, int o0, const float* stage, int lane, const Old<O>& old) {
  if (wide) {
    const int c = lane >> 2, ch = (lane & 3) * 8;                // this lane's column of 8 and its channels
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = h * 8 + c;
      if (col >= count) continue;
      const float4 lo = *reinterpret_cast<const float4*>(stage + col * STAGING_LD + ch);
      const float4 hi = *reinterpret_cast<const float4*>(stage + col * STAGING_LD + ch + 4);
      const float z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      Out8<O> y;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v = apply_act(z[i], ACT);
        if (a.res) v += old.packed(h * 8 + i);
        y.v[i] = from_f32<O>(v);
      }
      *reinterpret_cast<Out8<O>*>(static_cast<O*>(a.y) + (row + col) * a.ldy + o0 + ch) = y;
    }
  } else if (o0 + lane < a.o) {
    O* const y = static_cast<O*>(a.y) + row * a.ldy + o0 + lane;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i >= count) break;
      float v = apply_act(stage[i * STAGING_LD + lane], ACT);
      if (a.res) v += old.one(i);
      y[i * a.ldy] = from_f32<O>(v);
    }
  }
}
template <typename O>
__device__ __forceinline__ void finish_as(const LinearArgs& a, bool wide, long long row, int count, int o0, const float* stage, int lane, const Old<O>& old) {
  switch (a.act) {
    case TARDIS_ACT_GELU_TANH: finish<TARDIS_ACT_GELU_TANH, O>(a, wide, row, count, o0, stage, lane, old); break;
    case TARDIS_ACT_GELU_ERF: finish<TARDIS_ACT_GELU_ERF, O>(a, wide, row, count, o0, stage, lane, old); break;
    case TARDIS_ACT_RELU: finish<TARDIS_ACT_RELU, O>(a, wide, row, count, o0, stage, lane, old); break;
    default: finish<TARDIS_ACT_NONE, O>(a, wide, row, count, o0, stage, lane, old);
  }
}
// A warp's share of a tile: columns first, first + step, ... in blocks of 16 of the accumulator at `tacc`.  wait() returns whether it has been computed.
template <typename O, typename Wait>
__device__ __forceinline__ void finish_tile(const LinearArgs& a, bool wide, long long row, int rows, int first, int step, int o0, float bias, uint32_t tacc, float* stage,
                                            int lane, Wait wait) {
  Old<O> old, next;
  if (a.res) read_residual<O>(a, wide, row + first, rows - first, o0, lane, next);
  const bool ok = wait();
#pragma unroll 1
  for (int c = first; c < rows; c += step) {
    old = next;
    if (a.res) read_residual<O>(a, wide, row + c + step, rows - c - step, o0, lane, next);
    float v[16];
    tmem_ld16(tacc + uint32_t(c), v);
#pragma unroll
    for (int i = 0; i < 16; ++i) stage[i * STAGING_LD + lane] = ok ? v[i] + bias : CUDART_NAN_F;
    __syncwarp();
    finish_as<O>(a, wide, row + c, rows - c, o0, stage, lane, old);
    __syncwarp();
  }
}

// The same of a warp's sums in registers, columns half * 32 + 64 i + j
template <typename O, int BLOCKS>
__device__ __forceinline__ void finish_sums(const LinearArgs& a, bool wide, const Tile& t, int half, int o0, bool ok, float bias, const float (&sum)[BLOCKS][32], float* stage,
                                            int lane) {
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const int c = half * 32 + 64 * i + h;
      if (c >= t.rows) continue;
      Old<O> old;
      if (a.res) read_residual<O>(a, wide, t.first + c, t.rows - c, o0, lane, old);
#pragma unroll
      for (int j = 0; j < 16; ++j) stage[j * STAGING_LD + lane] = ok ? sum[i][h + j] + bias : CUDART_NAN_F;
      __syncwarp();
      finish_as<O>(a, wide, t.first + c, t.rows - c, o0, stage, lane, old);
      __syncwarp();
    }
}

template <int CTAS, int NT, int SPLITS, bool GATHER, bool PRECISE>
__global__ void __launch_bounds__(NTHREADS + (GATHER ? 32 * GATHER_WARPS : 0), 1)
k_linear_tc(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ Params p) {
  using C = Cfg<CTAS, NT, SPLITS>;
  constexpr bool SPLIT = SPLITS > 1;
  static_assert(!(SPLIT && CTAS == 2) && !(PRECISE && CTAS == 2 && GATHER) && C::B_ROWS <= 128, "");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* const exchange = reinterpret_cast<float*>(smem + C::NS * C::STAGE_BYTES);      // [SPLITS][128][PART_LD]
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::NS * C::STAGE_BYTES + C::EXCHANGE + C::STAGING);
  uint64_t* empty = full + C::NS;
  uint64_t* accum_full = empty + C::NS;        // [2]
  uint64_t* accum_empty = accum_full + 2;      // [2]
  uint64_t* parts_full = accum_empty + 2;      // SPLIT: the other CTAs' parts are here; ... have been taken everywhere
  uint64_t* parts_empty = parts_full + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(parts_empty + 1);
  volatile uint32_t* failed = tmem_slot + 1;
  const Groups groups = groups_at(smem + C::NS * C::STAGE_BYTES + C::EXCHANGE + C::STAGING + 256, p.a.groups);     // (grouped only)
  static_assert((2 * C::NS + 6) * 8 + 8 <= 256, "");

  const LinearArgs& a = p.a;
  const int warp = __shfl_sync(0xffffffffu, int(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  constexpr int in_cluster = SPLITS * CTAS;
  const int rank = in_cluster > 1 ? int(cluster_rank()) : 0, first_tile = blockIdx.x / in_cluster, step = gridDim.x / in_cluster;
  const int mt = (a.o + BM * CTAS - 1) / (BM * CTAS);
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::NS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&accum_full[b], 1); mbar_init(&accum_empty[b], 8 * CTAS); }
    if (SPLIT) { mbar_init(parts_full, 8 * SPLITS); mbar_init(parts_empty, 8 * SPLITS); }
    *failed = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmW) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmX) : "memory");
  }
  if (warp == 1) {
    if (CTAS == 2) tmem_alloc_pair(tmem_slot, C::TMEM_COLS);
    else tmem_alloc(tmem_slot, C::TMEM_COLS);
  }
  // this CTA's part of the k blocks
  const int per_split = SPLIT ? (p.kblocks + SPLITS - 1) / SPLITS : p.kblocks;
  const int kb_lo = SPLIT ? min(rank * per_split, p.kblocks) : 0, nkb = SPLIT ? min(p.kblocks, kb_lo + per_split) - kb_lo : p.kblocks;

  auto decode = [&](int tile) {
    Tile t;
    t.e = 0;
    int group_first = 0, group_rows = a.n, rem = tile;
    if (a.offsets) {
      const int place = place_of(groups, a.groups, tile);
      t.e = groups.order[place];
      rem = tile - groups.firsts[place];
      group_first = groups.starts[t.e];
      group_rows = groups.starts[t.e + 1] - group_first;
    }
    const int tiles = (group_rows + NT - 1) / NT;
    const int per = ((group_rows + tiles - 1) / tiles + C::STEP - 1) & ~(C::STEP - 1);         // tokens per tile: as even as the steps allow
    // raster: bands along one dimension, walked across the other, so that CTAs running at the same time share operands in L2
    const int F = p.tokens_fast ? tiles : mt, S = p.tokens_fast ? mt : tiles;
    const int bi = rem / (p.band * S), r2 = rem - bi * (p.band * S);
    const int w = min(p.band, F - bi * p.band);
    const int slow = r2 / w, fast = bi * p.band + (r2 - slow * w);
    const int ni = p.tokens_fast ? fast : slow, mi = p.tokens_fast ? slow : fast;
    t.o0 = mi * (BM * CTAS) + (CTAS == 2 ? rank * BM : 0);
    t.first = group_first + ni * per;
    t.rows = max(0, min(per, group_rows - ni * per));
    // A few tokens are read by all channel tiles at once: every other one begins in the middle of its channels, so that they do not all ask for the same lines (us in
    // step / apart: 64 tokens of 4096 -> 16384 27.0 / 25.0, 128 29.9 / 27.7, 64 of 16384 -> 4096 29.3 / 28.3).
    t.turn = tiles == 1 && (mi & 1) ? nkb >> 1 : 0;
    t.nt = max(C::STEP, (t.rows + C::STEP - 1) & ~(C::STEP - 1));
    return t;
  };
  if (CTAS == 1 && !SPLIT && !a.offsets && warp == 0 && first_tile < (a.n + NT - 1) / NT * mt) {
    // while the launch before ends: the first weights on their way into L2 (64 tokens of 4096 -> 16384 25.5 -> 24.9 us; clusters gained nothing)
    const Tile t = decode(first_tile);
    if (elect_one())
      for (int kb = 0; kb < min(nkb, C::NS); ++kb)
        asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(&tmW), "r"((kb_lo + (kb + t.turn) % nkb) * BK), "r"(t.o0), "r"(0) : "memory");
    __syncwarp();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");             // (x, offsets, ... may come from the launch before)
  if (a.offsets) build_groups(a.offsets, a.groups, a.n, NT, mt, groups);
  tc_fence_before();
  __syncthreads();
  if (in_cluster > 1) cluster_sync();                            // (the other CTAs' barriers are reported to)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (this CTA has its tensor memory)
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int ntiles = a.offsets ? groups.firsts[a.groups] : (a.n + NT - 1) / NT * mt;

  int issued = 0;
  if (warp == 0) {
    // ---------------- copies ----------------
    int s = 0, parity = 1;
    for (int tile = first_tile; tile < ntiles; tile += step) {
      const Tile t = decode(tile);
      const int half = t.nt / CTAS, row0 = t.first + (CTAS == 2 ? rank * half : 0);      // this CTA's tokens
      const int boxes = (half + BOX - 1) / BOX;
      const uint32_t bytes = C::A_BYTES + (GATHER ? half * 128 : boxes * (BOX * 128));       // (of the gathered rows too)
      for (int kb = kb_lo; kb < kb_lo + nkb; ++kb) {
        if (!mbar_wait_issue(&empty[s], parity, failed)) break;
        ++issued;
        uint8_t* const sa = smem + s * C::STAGE_BYTES;
        uint8_t* const sb = sa + C::A_BYTES;
        int kx = kb + t.turn;                                    // (the turned order ends with the blocks in front of its beginning)
        if (kx >= kb_lo + nkb) kx -= nkb;
        kx *= BK;
        if (elect_one()) {
          if (rank == 0 || CTAS == 1) mbar_expect_tx(&full[s], CTAS * bytes);
          if (CTAS == 2) tma_load_3d_pair(sa, &tmW, kx, t.o0, t.e, in_rank_0(&full[s]));
          else tma_load_3d(sa, &tmW, kx, t.o0, t.e, &full[s]);
          if (!GATHER)
            for (int i = 0; i < boxes; ++i) {
              if (CTAS == 2) tma_load_2d_pair(sb + i * (BOX * 128), &tmX, kx, row0 + i * BOX, in_rank_0(&full[s]));
              else tma_load_2d(sb + i * (BOX * 128), &tmX, kx, row0 + i * BOX, &full[s]);
            }
        }
        if (++s == C::NS) { s = 0; parity ^= 1; }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMAs (of a pair: rank 0) ----------------
    const uint64_t adesc = smem_desc_k_major_sw128(smem_u32(smem)), bdesc = smem_desc_k_major_sw128(smem_u32(smem) + C::A_BYTES);
    int s = 0, parity = 0;
    uint32_t use = 0;
    for (int tile = (CTAS == 1 || rank == 0) && nkb > 0 ? first_tile : ntiles; tile < ntiles; tile += step) {
      const Tile t = decode(tile);
      const uint32_t idesc = instr_desc_bf16(BM * CTAS, t.nt);
      const int most = PRECISE ? PRECISE_BLOCKS : nkb;           // k blocks of an accumulator
      for (int kb0 = 0; kb0 < nkb; kb0 += most) {
        const uint32_t ab = use & 1u;
        bool ok = mbar_wait_issue(&accum_empty[ab], ((use >> 1) & 1) ^ 1, failed);
        tc_fence_after();
        const uint32_t tacc = tmem_base + ab * NT;
        for (int kb = kb0; kb < min(nkb, kb0 + most); ++kb) {
          ok = mbar_wait_issue(&full[s], parity, failed);
          tc_fence_after();
          const uint64_t da = adesc + uint32_t(s * (C::STAGE_BYTES >> 4)), db = bdesc + uint32_t(s * (C::STAGE_BYTES >> 4));
          if (elect_one() && ok) {
#pragma unroll
            for (int k = 0; k < BK / 16; ++k) {
              if (CTAS == 2) umma_f16_pair(tacc, da + k * 2, db + k * 2, idesc, (kb != kb0 || k != 0) ? 1u : 0u);
              else umma_f16(tacc, da + k * 2, db + k * 2, idesc, (kb != kb0 || k != 0) ? 1u : 0u);
            }
            if (CTAS == 2) umma_commit_pair(&empty[s]);
            else umma_commit(&empty[s]);
          }
          if (++s == C::NS) { s = 0; parity ^= 1; }
        }
        if (elect_one() && ok) {
          if (CTAS == 2) umma_commit_pair(&accum_full[ab]);
          else umma_commit(&accum_full[ab]);
        }
        ++use;
      }
    }
  } else if (GATHER && warp >= NTHREADS / 32) {
    // ---------------- rows of x by their indices ----------------
    // Each of four warps has a quarter of this CTA's rows, their indices in registers that all lanes hold alike, and copies them four at a time.
    // (Issued by the 32 lanes of one warp, 80 cycles each, 8192 rows of 8 experts, 4096 -> 16384, took 2.8 times as long; copied by threads, whose writes need a fence towards
    // the tensor cores, 2.3 times.)
    constexpr int QUADS = C::B_ROWS / (4 * GATHER_WARPS);
    const int w = warp - NTHREADS / 32;
    int s = 0, parity = 1;
    for (int tile = first_tile; tile < ntiles; tile += step) {
      const Tile t = decode(tile);
      const int half = t.nt / CTAS, row0 = t.first + (CTAS == 2 ? rank * half : 0);
      int idx[QUADS][4];
#pragma unroll
      for (int j = 0; j < QUADS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = row0 + (w + j * GATHER_WARPS) * 4 + i;
          const int at = r < t.first + t.rows ? a.rows[r] : -1;
          idx[j][i] = at >= 0 && at < a.nx ? at : a.nx;          // (behind the last row: zeros)
        }
      for (int kb = kb_lo; kb < kb_lo + nkb; ++kb) {
        if (!mbar_wait_issue(&empty[s], parity, failed)) break;
        int kx = kb + t.turn;
        if (kx >= kb_lo + nkb) kx -= nkb;
        if (elect_one()) {
          uint8_t* const sb = smem + s * C::STAGE_BYTES + C::A_BYTES + w * 512;
#pragma unroll
          for (int j = 0; j < QUADS; ++j)
            if ((w + j * GATHER_WARPS) * 4 < half) {
              if (CTAS == 2) tma_gather4_pair(sb + j * (GATHER_WARPS * 512), &tmX, kx * BK, idx[j], in_rank_0(&full[s]));
              else tma_gather4(sb + j * (GATHER_WARPS * 512), &tmX, kx * BK, idx[j], &full[s]);
            }
        }
        if (++s == C::NS) { s = 0; parity ^= 1; }
      }
    }
  } else {
    // ---------------- epilogue: a warp has TMEM lanes 32 (warp % 4) .. + 31 and every other block of columns ----------------
    const int q = warp & 3, half = (warp - 2) >> 2;
    float* const staging = reinterpret_cast<float*>(smem + C::NS * C::STAGE_BYTES + C::EXCHANGE + (warp - 2) * STAGING_WARP);
    uint32_t use = 0, tiles_done = 0;                            // accumulators taken; tiles
    bool ok = true;
    for (int tile = first_tile; tile < ntiles; tile += step) {
      const Tile t = decode(tile);
      const int o = t.o0 + q * 32 + lane;
      const uint32_t ab = use & 1u;                              // (not PRECISE: the tile's accumulator)
      const float bias = a.bias && o < a.o ? a.bias[(long long)(t.e) * a.o + o] : 0.f;
      auto computed = [&]() {
        if (nkb > 0) ok = ok && mbar_wait_warp(&accum_full[ab], (use >> 1) & 1);
        if (!ok) *failed = 1u;
        tc_fence_after();
        return ok;
      };
      float sum[PRECISE ? NT / 64 : 1][32];                      // PRECISE: columns half * 32 + 64 i + j
      if (PRECISE) {
#pragma unroll
        for (int i = 0; i < NT / 64; ++i)
#pragma unroll
          for (int j = 0; j < 32; ++j) sum[i][j] = 0.f;
        for (int kb0 = 0; kb0 < nkb; kb0 += PRECISE_BLOCKS) {
          const uint32_t a_now = use & 1u;
          ok = ok && mbar_wait_warp(&accum_full[a_now], (use >> 1) & 1);
          if (!ok) *failed = 1u;
          tc_fence_after();
#pragma unroll
          for (int i = 0; i < NT / 64; ++i) {
            if (half * 32 + 64 * i >= t.rows) continue;
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
              float v[16];
              tmem_ld16(tmem_base + a_now * NT + (uint32_t(q * 32) << 16) + uint32_t(half * 32 + 64 * i + h), v);
#pragma unroll
              for (int j = 0; j < 16; ++j) sum[i][h + j] += v[j];
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (CTAS == 2) mbar_arrive_cluster(in_rank_0(&accum_empty[a_now]));
            else mbar_arrive(&accum_empty[a_now]);
          }
          ++use;
        }
      }
      if (PRECISE && !SPLIT) {
        const int o0 = o - lane;
        const bool wide = p.wide && o0 + 32 <= a.o;
        if (NT == 64 && a.out_dtype == TARDIS_BF16) finish_sums<__nv_bfloat16>(a, wide, t, half, o0, ok, bias, sum, staging, lane);
        else finish_sums<float>(a, wide, t, half, o0, ok, bias, sum, staging, lane);
      } else if (!SPLIT) {
        const int o0 = o - lane;
        const bool wide = p.wide && o0 + 32 <= a.o;
        const uint32_t tacc = tmem_base + ab * NT + (uint32_t(q * 32) << 16);
        if (a.out_dtype == TARDIS_BF16) finish_tile<__nv_bfloat16>(a, wide, t.first, t.rows, half * 16, 32, o0, bias, tacc, staging, lane, computed);
        else finish_tile<float>(a, wide, t.first, t.rows, half * 16, 32, o0, bias, tacc, staging, lane, computed);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CTAS == 2) mbar_arrive_cluster(in_rank_0(&accum_empty[ab]));
          else mbar_arrive(&accum_empty[ab]);
        }
      } else {
        constexpr int SHARE = C::SHARE, QUADS = NT / 32 * SHARE, LD = C::PART_LD;
        // this CTA finishes two quads of columns at a time, their residuals loaded ahead
        float old[8], next[8];
        auto read_old = [&](int w0) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int w = w0 + j / 4, i = w % SHARE * SPLITS + rank, c = w / SHARE * 32 + i * 4 + j % 4;
            next[j] = a.res && o < a.o && w < QUADS && i < 8 && c < t.rows ? load_out(a.res, (t.first + c) * a.ldr + o, a.out_dtype) : 0.f;
          }
        };
        read_old(half * 2);
        if (!PRECISE) computed();
        // of every block of 32 columns, quad i (four columns) belongs to CTA i % SPLITS; the parts of the tile before have been taken by then
        if (tiles_done > 0 && ok) ok = mbar_wait_cluster(parts_empty, (tiles_done - 1) & 1);
        uint32_t to[SPLITS];
#pragma unroll
        for (int r = 0; r < SPLITS; ++r) to[r] = in_rank(exchange + (rank * BM + q * 32 + lane) * LD, r);
#pragma unroll
        for (int block = 0; block < NT / 64; ++block) {
          const int c = half * 32 + 64 * block;
          if (c >= t.rows) continue;
          float v[32];
          if (PRECISE) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = sum[PRECISE ? block : 0][i];
          } else tmem_ld32(tmem_base + ab * NT + (uint32_t(q * 32) << 16) + uint32_t(c), v);
          if (!ok || nkb == 0) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = ok ? 0.f : CUDART_NAN_F;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + 4 * i < t.rows)
              asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to[i % SPLITS] + uint32_t(c / 32 * SHARE + i / SPLITS) * 16),
                           "f"(v[4 * i]), "f"(v[4 * i + 1]), "f"(v[4 * i + 2]), "f"(v[4 * i + 3]) : "memory");
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (!PRECISE && nkb > 0) mbar_arrive(&accum_empty[ab]);
#pragma unroll
          for (int r = 0; r < SPLITS; ++r) mbar_arrive_cluster(in_rank(parts_full, r));
        }
        ok = mbar_wait_cluster(parts_full, tiles_done & 1) && ok;
        if (!ok) *failed = 1u;
        for (int w0 = half * 2; w0 < QUADS; w0 += 4) {
#pragma unroll
          for (int j = 0; j < 8; ++j) old[j] = next[j];
          read_old(w0 + 4);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int w = w0 + h, i = w % SHARE * SPLITS + rank, c = w / SHARE * 32 + i * 4;
            if (w >= QUADS || i >= 8 || c >= t.rows || o >= a.o) continue;
            float z[4] = {};
#pragma unroll
            for (int r = 0; r < SPLITS; ++r) {
              const float4 part = *reinterpret_cast<const float4*>(exchange + (r * BM + q * 32 + lane) * LD + w * 4);
              z[0] += part.x; z[1] += part.y; z[2] += part.z; z[3] += part.w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (c + j >= t.rows) break;
              float y = apply_act(z[j] + bias, a.act);
              if (a.res) y += old[h * 4 + j];
              store_out(a.y, (t.first + c + j) * a.ldy + o, a.out_dtype, ok ? y : CUDART_NAN_F);
            }
          }
        }
        __syncwarp();
        if (lane == 0)
          for (int r = 0; r < SPLITS; ++r) mbar_arrive_cluster(in_rank(parts_empty, r));
      }
      if (!PRECISE) ++use;
      ++tiles_done;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) {
    // neither ends while the other may still report to it or its MMAs read it; copies of both report to rank 0
    if (threadIdx.x == 0 && rank == 1 && *failed) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_rank_0(const_cast<uint32_t*>(failed))), "r"(1u) : "memory");
    cluster_sync();
    if (rank == 0 && warp == 0 && *failed) land_copies<C::NS>(full, issued);
    if (warp == 1) tmem_dealloc_pair(tmem_base, C::TMEM_COLS);
    cluster_sync();
  } else {
    if (warp == 0 && *failed) land_copies<C::NS>(full, issued);
    if (warp == 1) tmem_dealloc(tmem_base, C::TMEM_COLS);
    if (SPLIT) cluster_sync();
  }
}

// ---- host side ------------------------------------------------------------------------------------------
// Clusters of one CTA per SM that run at once: of three and four the SMs of a GPC leave a rest (45 and 33 of 148 SMs, as the occupancy query says).
static long long clusters_at_once(int sms, int ctas) { return ctas <= 2 ? sms / ctas : (long long)(sms * (ctas == 3 ? 0.305 : 0.223)); }

static bool make_weight_map(CUtensorMap* map, const LinearArgs& a) {
  return make_map_3d(map, a.W, a.o, a.groups, a.k, a.ldw, a.groups > 1 ? a.stride_w : a.ldw, BM);
}

template <int CTAS, int NT, int SPLITS, bool GATHER, bool PRECISE>
static tardis_status_t launch(const LinearArgs& a, int dev, int sms, cudaStream_t s) {
  using C = Cfg<CTAS, NT, SPLITS>;
  static_assert(C::FIXED + groups_bytes(kMaxExperts) <= 227 * 1024, "");
  CUtensorMap w, x;
  if (!make_weight_map(&w, a) || !make_map(&x, a.x, a.nx, a.k, a.ldx, GATHER ? 1 : BOX)) return TARDIS_ERR_INVALID_ARG;
  Params p;
  p.a = a; p.kblocks = (a.k + BK - 1) / BK;
  const long long mt = (a.o + BM * CTAS - 1) / (BM * CTAS), nt = (a.n + NT - 1) / NT;
  p.tokens_fast = nt <= mt ? 1 : 0;
  p.band = 8;
  const size_t unit = a.out_dtype == TARDIS_BF16 ? 2 : 4;
  auto fits = [&](const void* q, long long ld) { return !q || ((reinterpret_cast<uintptr_t>(q) | size_t(ld) * unit) & 15) == 0; };
  p.wide = fits(a.y, a.ldy) && fits(a.res, a.ldr);
  const int smem = C::FIXED + (a.offsets ? groups_bytes(a.groups) : 0);
  static thread_local int room_on = -1;               // the device on which this thread last gave the kernel its shared memory
  if (dev != room_on) {
    TARDIS_CUDA_TRY(cudaFuncSetAttribute(k_linear_tc<CTAS, NT, SPLITS, GATHER, PRECISE>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::FIXED + groups_bytes(kMaxExperts)));
    room_on = dev;
  }
  long long tiles = (nt + (a.offsets ? (a.groups < a.n ? a.groups : a.n) : 0)) * mt;     // at most
  constexpr int in_cluster = SPLITS * CTAS;
  const long long at_once = clusters_at_once(sms, in_cluster);
  if (tiles > at_once) tiles = at_once;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tiles * in_cluster)); cfg.blockDim = dim3(NTHREADS + (GATHER ? 32 * GATHER_WARPS : 0)); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = in_cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = in_cluster > 1 ? 2 : 1;
  TARDIS_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_linear_tc<CTAS, NT, SPLITS, GATHER, PRECISE>, w, x, p));
  return TARDIS_OK;
}

template <int CTAS, int NT, int SPLITS, bool PRECISE>
static tardis_status_t launch_rows(const LinearArgs& a, int dev, int sms, cudaStream_t s) {
  return a.rows ? launch<CTAS, NT, SPLITS, true, PRECISE>(a, dev, sms, s) : launch<CTAS, NT, SPLITS, false, PRECISE>(a, dev, sms, s);
}
template <int NT, bool PRECISE>
static tardis_status_t launch_splits(const LinearArgs& a, int splits, int dev, int sms, cudaStream_t s) {
  switch (splits) {
    case 2: return launch_rows<1, NT, 2, PRECISE>(a, dev, sms, s);
    case 3: return launch_rows<1, NT, 3, PRECISE>(a, dev, sms, s);
    case 4: return launch_rows<1, NT, 4, PRECISE>(a, dev, sms, s);
  }
  return launch_rows<1, NT, 1, PRECISE>(a, dev, sms, s);
}

struct Choice { int kind, splits; double us; };      // kind: 0, 1: 64 or 128 tokens by one CTA; 2: 256 by a pair
// The variant with the shortest estimate.  A CTA takes some 0.235 us per block of 64 k (less than its MMAs only with 256 tokens), all of them
// together the time of the weights that they read at once at 6.3 TB/s; clusters of 2, 3 and 4 leave SMs of a GPC unused.  What a launch takes beside
// that, and a further wave of clusters that exchange parts, is measured too.  (Estimate / measured, us: 128 tokens of 4096 -> 4096, splits of 2 of 64 tokens 16.8 / 15.5, of 4
// of 128 18.5 / 17.1, whole 64 19.8 / 18.6, 128 20.6 / 20.6; 160 of 4096 -> 16384, 128 35.0 / 37.4, pairs 27.0 / 30.5; 512 of 4096 -> 1024, 4 of 128 16.9 / 15.8.)
static Choice choose(const LinearArgs& a, int sms) {
  const int kblocks = (a.k + BK - 1) / BK;
  const long long groups = a.offsets ? (a.groups < a.n ? a.groups : a.n) : 1, rows = (a.n + groups - 1) / groups;
  Choice best = {0, 1, 1e30};
  const int kinds = a.precise && a.out_dtype != TARDIS_F32 ? 1 : a.precise && a.rows ? 2 : 3;
  for (int kind = 0; kind < kinds; ++kind)
    for (int splits = 1; splits <= (kind == 2 || (a.precise && kind == 1) ? 1 : 4); ++splits) {
      if (splits > 1 && kblocks < 4 * splits) continue;
      const int ctas = kind == 2 ? 2 : 1, most = 64 << kind;
      const long long cuts = (rows + most - 1) / most, tiles = (a.o + BM * ctas - 1) / (BM * ctas) * cuts * groups;
      const double width = double((rows + cuts - 1) / cuts), at_once = double(clusters_at_once(sms, splits * ctas));
      const double waves = ceil(tiles / at_once), running = tiles < at_once ? double(tiles) : at_once;
      double step = fmax(0.235, running / cuts * (splits * ctas) * (BM * BK * 2) / 6.3e6);
      if (kind == 2) step = fmax(step, fmax(0.245, 0.275 * width / 256));
      if (a.rows) step = fmax(step, 0.0035 * width / ctas);                                // (rows picked one by one)
      double us = waves * ((kblocks + splits - 1) / splits) * step;
      us += splits == 1 ? 4.0 + 0.012 * width : waves * (3.5 + 0.06 * width) + 2.;
      if (us < best.us) best = {kind, splits, us};
    }
  return best;
}

// a.work[r] = x[a.rows[r]], a warp per row: 16 bytes per lane
__global__ void __launch_bounds__(256) k_gather_rows(const __grid_constant__ LinearArgs a) {
  const int r = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, pieces = a.k / 8;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (r >= a.n) return;
  const int src = a.rows[r];
  const bool there = src >= 0 && src < a.nx;
  const uint4* const from = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.x) + (there ? src : 0) * a.ldx);
  uint4* const to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.work) + (long long)(r) * a.k);
  for (int i0 = lane; i0 < pieces; i0 += 128) {
    uint4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = there && i0 + 32 * j < pieces ? from[i0 + 32 * j] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + 32 * j < pieces) to[i0 + 32 * j] = v[j];
  }
}
static tardis_status_t launch_gather_rows(const LinearArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned((a.n - 1) / 8 + 1)); cfg.blockDim = dim3(256); cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  TARDIS_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_gather_rows, a));
  return TARDIS_OK;
}

}  // namespace linear

double estimate_linear_tc(const LinearArgs& a, int sms) { return linear::choose(a, sms).us; }

tardis_status_t launch_linear_tc(const LinearArgs& given, cudaStream_t s) {
  using namespace linear;
  LinearArgs a = given;
  if (!tensor_maps_available()) return TARDIS_ERR_UNSUPPORTED;
  int dev = 0, sms = 0;
  TARDIS_CUDA_TRY(cudaGetDevice(&dev));
  TARDIS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const Choice best = choose(a, sms);
  if (best.kind == 2) {
    // Every tile of 256 outputs picks its rows again, at a third of the rate of whole boxes: with scratch and many outputs they are picked once (us picked tile by tile / once:
    // 8192 rows of 8 experts 4096 -> 16384 1008 / 835, -> 4096 262 / 235, -> 2048 133 / 128; 4000 rows of 16 experts 8192 -> 4224 359 / 339, -> 2048, where the weights of
    // small groups take as long, 170 / 175).
    if (a.rows && a.work && a.o >= 4096) {
      const tardis_status_t st = launch_gather_rows(a, s);
      if (st != TARDIS_OK) return st;
      a.x = a.work; a.ldx = a.k; a.nx = a.n; a.rows = nullptr;
    }
    return a.precise ? launch<2, 256, 1, false, true>(a, dev, sms, s) : launch_rows<2, 256, 1, false>(a, dev, sms, s);      // (with row indices: enough registers for pairs only without PRECISE)
  }
  if (a.precise) return best.kind == 1 ? launch_rows<1, 128, 1, true>(a, dev, sms, s) : launch_splits<64, true>(a, best.splits, dev, sms, s);
  return best.kind == 1 ? launch_splits<128, false>(a, best.splits, dev, sms, s) : launch_splits<64, false>(a, best.splits, dev, sms, s);
}

}  // namespace tardis
