// The dense products of unfolded feed-forward blocks: fp32, up to eight rows of bf16, the weighted return to the tokens, and which kernel serves a call
// (more rows of bf16: linear_tc.cu).
#include <math.h>

#include "linear.cuh"
#include "ptx.cuh"

namespace tardis {
namespace linear {

// ---- fp32: plain multiply-adds ----
// 16 bytes into shared memory, zeros where `there` is false
__device__ __forceinline__ void copy16(void* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// 256 threads compute a tile of ROWS x OUTS, a thread 8 x 8 of them (rows ty + TY i, outputs tx + TX j): what bounds this kernel is reading shared memory, 16 multiply-adds
// per 16-byte read are what it takes to keep up.  (With 4 x 8 per thread 2048 x 1024 x 2048 took 264 us, with packed multiply-adds too, now 220 = 39
// TFLOP/s; a tile of 32 x 32 with 2 x 2 took 0.6 us for 32 channels.)  Small tiles need fewer threads than that: G groups of them share the channels of a step, and all
// threads add them up in a fixed order at the end.  Steps of BK channels lie in shared memory as they do in global memory, STAGES - 1 of them on their way (16-byte asynchronous copies).
template <int ROWS_, int OUTS_, int BK_, int STAGES_> struct CfgF32 {
  static constexpr int ROWS = ROWS_, OUTS = OUTS_, STAGES = STAGES_, TY = ROWS / 8, TX = OUTS / 8, G = 256 / (TX * TY);
  static constexpr int BK = BK_, LD = BK + 4, PASS = 1024 / BK /* rows that the threads copy at a time */, STAGE = (ROWS + OUTS) * LD, RING = STAGES * STAGE * 4, SUMS = G > 1 ? G * ROWS * OUTS * 4 : 0;
  static constexpr int SMEM = RING > SUMS ? RING : SUMS;
};
template <typename C>
__global__ void __launch_bounds__(256, 2) k_linear_f32(const __grid_constant__ LinearArgs a) {
  constexpr int BK = C::BK, LD = C::LD, STAGES = C::STAGES, XR = C::ROWS / C::PASS, WR = C::OUTS / C::PASS;      // rows of x and of W that a thread copies
  extern __shared__ __align__(16) float smem_f32[];
  const GroupTile t = find_group_tile(a.offsets, a.groups, a.n, C::ROWS, blockIdx.x);
  if (t.rows == 0) return;
  const int o0 = blockIdx.y * C::OUTS, k_at = threadIdx.x % (BK / 4) * 4, r_at = threadIdx.x / (BK / 4);
  const int tx = threadIdx.x % C::TX, ty = threadIdx.x / C::TX % C::TY, g = threadIdx.x / (C::TX * C::TY);
  int from[XR];                                              // rows of x (-1: zeros)
#pragma unroll
  for (int i = 0; i < XR; ++i) {
    const int r = r_at + C::PASS * i;
    from[i] = -1;
    if (r < t.rows) from[i] = a.rows ? a.rows[t.first + r] : t.first + r;
    if (from[i] >= a.nx) from[i] = -1;
  }
  const float* const x_at = static_cast<const float*>(a.x) + k_at;
  const float* const w_at = static_cast<const float*>(a.W) + t.e * a.stride_w + k_at;
  const int steps = (a.k + BK - 1) / BK;
  auto load = [&](int step) {
    if (step < steps) {
      float* const to = smem_f32 + step % STAGES * C::STAGE + r_at * LD + k_at;
      const bool in = step * BK + k_at < a.k;
#pragma unroll
      for (int i = 0; i < XR; ++i) {
        const bool there = in && from[i] >= 0;
        copy16(to + C::PASS * i * LD, there ? x_at + from[i] * a.ldx + step * BK : static_cast<const float*>(a.x), there);
      }
#pragma unroll
      for (int i = 0; i < WR; ++i) {
        const int o = o0 + r_at + C::PASS * i;
        const bool there = in && o < a.o;
        copy16(to + (C::ROWS + C::PASS * i) * LD, there ? w_at + o * a.ldw + step * BK : static_cast<const float*>(a.W), there);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float acc[8][8] = {};
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) load(s);
  for (int step = 0; step < steps; ++step) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
    __syncthreads();                                         // (the stage is there, and nobody still reads the one that is filled next)
    load(step + STAGES - 1);
    const float* const sx = smem_f32 + step % STAGES * C::STAGE + ty * LD, *const sw = smem_f32 + step % STAGES * C::STAGE + (C::ROWS + tx) * LD;
#pragma unroll 1
    for (int kk = g * 4; kk < BK; kk += C::G * 4) {
      float4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const float4*>(sx + C::TY * i * LD + kk);
#pragma unroll
      for (int j = 0; j < 8; j += 2) {                       // (two outputs at a time: sixteen independent sums; with one 300 x 1024 x 2048 took 62 us, now 54)
        const float4 w = *reinterpret_cast<const float4*>(sw + C::TX * j * LD + kk), u = *reinterpret_cast<const float4*>(sw + C::TX * (j + 1) * LD + kk);
#pragma unroll
        for (int i = 0; i < 8; ++i) { acc[i][j] = fmaf(x[i].x, w.x, acc[i][j]); acc[i][j + 1] = fmaf(x[i].x, u.x, acc[i][j + 1]); }
#pragma unroll
        for (int i = 0; i < 8; ++i) { acc[i][j] = fmaf(x[i].y, w.y, acc[i][j]); acc[i][j + 1] = fmaf(x[i].y, u.y, acc[i][j + 1]); }
#pragma unroll
        for (int i = 0; i < 8; ++i) { acc[i][j] = fmaf(x[i].z, w.z, acc[i][j]); acc[i][j + 1] = fmaf(x[i].z, u.z, acc[i][j + 1]); }
#pragma unroll
        for (int i = 0; i < 8; ++i) { acc[i][j] = fmaf(x[i].w, w.w, acc[i][j]); acc[i][j + 1] = fmaf(x[i].w, u.w, acc[i][j + 1]); }
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  auto finish = [&](int r, int c, float z) {
    const int o = o0 + c;
    if (r >= t.rows || o >= a.o) return;
    const long long row = t.first + r;
    if (a.bias) z += a.bias[(long long)(t.e) * a.o + o];
    z = apply_act(z, a.act);
    if (a.res) z += static_cast<const float*>(a.res)[row * a.ldr + o];
    static_cast<float*>(a.y)[row * a.ldy + o] = z;
  };
  if (C::G == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) finish(ty + C::TY * i, tx + C::TX * j, acc[i][j]);
    return;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) smem_f32[(g * C::ROWS + ty + C::TY * i) * C::OUTS + tx + C::TX * j] = acc[i][j];
  __syncthreads();
#pragma unroll 4
  for (int at = threadIdx.x; at < C::ROWS * C::OUTS; at += 256) {
    float z = 0.f;
#pragma unroll
    for (int other = 0; other < C::G; ++other) z += smem_f32[other * C::ROWS * C::OUTS + at];
    finish(at / C::OUTS, at % C::OUTS, z);
  }
}

template <typename C>
static tardis_status_t launch_f32_tiles(const LinearArgs& a, int dev, cudaStream_t s) {
  const long long tiles = (a.n + C::ROWS - 1) / C::ROWS + (a.offsets ? (a.groups < a.n ? a.groups : a.n) : 0);     // at most
  const int outputs = (a.o + C::OUTS - 1) / C::OUTS;
  if (outputs > 65535) return TARDIS_ERR_UNSUPPORTED;
  static thread_local int room_on = -1;               // the device on which this thread last gave the kernel its shared memory
  if (dev != room_on) {
    TARDIS_CUDA_TRY(cudaFuncSetAttribute(k_linear_f32<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM));
    room_on = dev;
  }
  k_linear_f32<C><<<dim3(unsigned(tiles), unsigned(outputs)), 256, C::SMEM, s>>>(a);
  TARDIS_CUDA_TRY(cudaGetLastError());
  return TARDIS_OK;
}

// Up to R <= 8 rows of fp32: a CTA has four outputs, its eight warps share the channels (a lane four at a time) and add their parts in a fixed order.
template <int R>
__global__ void __launch_bounds__(256) k_linear_few_f32(const __grid_constant__ LinearArgs a) {
  constexpr int O = 4;
  __shared__ float part[8][O * R];
  const GroupTile t = find_group_tile(a.offsets, a.groups, a.n, R, blockIdx.y);
  if (t.rows == 0) return;
  const int o0 = blockIdx.x * O, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float *w[O], *x[R];
#pragma unroll
  for (int i = 0; i < O; ++i) w[i] = static_cast<const float*>(a.W) + t.e * a.stride_w + min(o0 + i, a.o - 1) * a.ldw;
  bool there[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    int src = -1;
    if (r < t.rows) src = a.rows ? a.rows[t.first + r] : t.first + r;
    there[r] = src >= 0 && src < a.nx;
    x[r] = static_cast<const float*>(a.x) + (there[r] ? src : 0) * a.ldx;
  }
  float acc[O][R] = {};
  for (int k = threadIdx.x * 4; k < a.k; k += 1024) {
    float4 wv[O];
#pragma unroll
    for (int i = 0; i < O; ++i) wv[i] = *reinterpret_cast<const float4*>(w[i] + k);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= t.rows) continue;
      const float4 xv = there[r] ? *reinterpret_cast<const float4*>(x[r] + k) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < O; ++i) acc[i][r] = fmaf(wv[i].w, xv.w, fmaf(wv[i].z, xv.z, fmaf(wv[i].y, xv.y, fmaf(wv[i].x, xv.x, acc[i][r]))));
    }
  }
#pragma unroll
  for (int i = 0; i < O; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float v = acc[i][r];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
      if (lane == 0) part[warp][r * O + i] = v;
    }
  __syncthreads();
  const int r = threadIdx.x / O, o = o0 + threadIdx.x % O;
  if (threadIdx.x >= O * R || r >= t.rows || o >= a.o) return;
  float z = 0.f;
  for (int i = 0; i < 8; ++i) z += part[i][threadIdx.x];
  const long long row = t.first + r;
  if (a.bias) z += a.bias[(long long)(t.e) * a.o + o];
  z = apply_act(z, a.act);
  if (a.res) z += static_cast<const float*>(a.res)[row * a.ldr + o];
  static_cast<float*>(a.y)[row * a.ldy + o] = z;
}

static tardis_status_t launch_f32(const LinearArgs& a, cudaStream_t s) {
  if (a.n <= 8) {
    const dim3 grid(unsigned((a.o + 3) / 4), a.offsets ? unsigned(a.n) : 1u);          // at most (a group's tile has a row)
    if (a.n == 1) k_linear_few_f32<1><<<grid, 256, 0, s>>>(a);
    else if (a.n <= 3) k_linear_few_f32<3><<<grid, 256, 0, s>>>(a);
    else k_linear_few_f32<8><<<grid, 256, 0, s>>>(a);
    TARDIS_CUDA_TRY(cudaGetLastError());
    return TARDIS_OK;
  }
  int dev = 0, sms = 0;
  TARDIS_CUDA_TRY(cudaGetDevice(&dev));
  TARDIS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  // The largest tiles that keep the SMs busy (a tile's time hardly depends on how many there are; us with tiles of 128 x 128, 64 x 64, 32 x 64, 16 x 32: 2048 x 64 x
  // 2048 26 / 34 / 46 / 178, 1024 x 256 x 1024 42 / 24 / 28 / 56, 256 x 256 x 1024 42 / 15 / 9.6 / 17, 64 x 256 x 1024 37 / 14 / 9 / 5.7).
  // No more groups than rows have any: 12 rows of 64 experts, 256 -> 1024, took 34 us with the tiles for 64 groups, now 13.5.
  const long long groups = a.offsets ? (a.groups < a.n ? a.groups : a.n) : 1, rows = (a.n + groups - 1) / groups;
  auto tiles = [&](int high, int wide) { return (a.o + wide - 1) / wide * (groups * ((rows + high - 1) / high)); };
  if (tiles(128, 128) * 10 >= sms * 13) return launch_f32_tiles<CfgF32<128, 128, 32, 3>>(a, dev, s);
  if (tiles(64, 64) * 10 >= sms * 15) return launch_f32_tiles<CfgF32<64, 64, 32, 4>>(a, dev, s);
  return tiles(32, 64) * 10 >= sms * 6 ? launch_f32_tiles<CfgF32<32, 64, 32, 6>>(a, dev, s) : launch_f32_tiles<CfgF32<16, 32, 128, 3>>(a, dev, s);
}

// ---- up to eight rows of bf16 (a few times eight of small weights): bound by reading the weights once ----
// An item is 16 outputs of up to 8 rows of a group.  Weights go straight from global memory into the A fragments of mma.m16n8k16 and the rows of x into its B
// fragments: a sum over channels may be taken in any order, so lane (g, t) reads 16 bytes, channels 8 t .. 8 t + 7 of a block of 32, of weight rows
// g and g + 8 and of row g of x, and each pair of words is the fragment of one instruction.  The eight warps of a CTA share the channels in blocks
// of 64, taken in turn, so that together they read whole lines of every weight row; their parts are added in a fixed order.  Two CTAs per SM
// walk the items (a contiguous run each, outputs first), and the loads of the next step, of the next item too, are under way while one is
// multiplied, summed up and stored.
constexpr int FEW_ROWS = 8, FEW_WARPS = 8, FEW_U = 2;      // U: blocks of 64 channels of a warp and step

// Weights pass L1 by.  Not the read-only path: this kernel begins while the launch before, which may write what is read here, is still running.
__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

__global__ void __launch_bounds__(FEW_WARPS * 32, 2) k_linear_few(const __grid_constant__ LinearArgs a) {
  constexpr int ROWS = FEW_ROWS, WARPS = FEW_WARPS, U = FEW_U;
  extern __shared__ int table[];                           // (grouped only)
  __shared__ float part[2][WARPS][ROWS][17];
  const Groups groups = groups_at(table, a.groups);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int nkb = (a.k + 63) / 64, ot = (a.o + 15) / 16, cuts = (a.n + ROWS - 1) / ROWS;     // (cuts: without groups)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (!a.offsets) {                                        // while the launch before ends: the first steps' weights on their way into L2
    const int o0 = int((long long)(blockIdx.x) * ot * cuts / gridDim.x) / cuts * 16;
    const __nv_bfloat16* const w = static_cast<const __nv_bfloat16*>(a.W) + min(o0 + (lane & 15), a.o - 1) * a.ldw;
    for (int kb = warp + (lane >> 4) * WARPS; kb < min(nkb, 2 * U * WARPS); kb += 2 * WARPS) asm volatile("prefetch.global.L2 [%0];" ::"l"(w + kb * 64));
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (a.offsets) {
    build_groups(a.offsets, a.groups, a.n, ROWS, ot, groups);
    __syncthreads();
  }
  const int items = a.offsets ? groups.firsts[a.groups] : ot * cuts;
  const int from = int((long long)(blockIdx.x) * items / gridDim.x), to = int((long long)(blockIdx.x + 1) * items / gridDim.x);
  if (from == to) return;

  struct Where { int e, o0, first, rows; };
  auto locate = [&](int item) {
    Where w = {0, item / cuts * 16, item % cuts * ROWS, min(ROWS, a.n - item % cuts * ROWS)};
    if (a.offsets) {
      const int place = place_of(groups, a.groups, item);
      w.e = groups.order[place];
      const int i = item - groups.firsts[place], tile = i / ot;
      w.o0 = (i - tile * ot) * 16;
      w.first = groups.starts[w.e] + tile * ROWS;
      w.rows = min(ROWS, groups.starts[w.e + 1] - w.first);
    }
    return w;
  };
  // the loading side: its item and step
  int item = from, kb = warp;
  const __nv_bfloat16 *w0, *w1, *x;
  bool there;
  auto aim = [&]() {
    const Where w = locate(item);
    const __nv_bfloat16* const W = static_cast<const __nv_bfloat16*>(a.W) + w.e * a.stride_w + t * 8;
    w0 = W + min(w.o0 + g, a.o - 1) * a.ldw;               // (outputs behind the last are computed and dropped)
    w1 = W + min(w.o0 + g + 8, a.o - 1) * a.ldw;
    int at = -1;
    if (g < w.rows) at = a.rows ? a.rows[w.first + g] : w.first + g;
    there = at >= 0 && at < a.nx;
    x = static_cast<const __nv_bfloat16*>(a.x) + (there ? at : 0) * a.ldx + t * 8;
  };
  uint4 A[2][U][4], B[2][U][2];
  auto load = [&](uint4 (&A)[U][4], uint4 (&B)[U][2]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (kb + u * WARPS) * 64 + h * 32;
        const bool in = k + t * 8 < a.k;
        A[u][h] = in ? load_once(w0 + k) : make_uint4(0u, 0u, 0u, 0u);
        A[u][2 + h] = in ? load_once(w1 + k) : make_uint4(0u, 0u, 0u, 0u);
        B[u][h] = in && there ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0u, 0u, 0u, 0u);
      }
    kb += U * WARPS;
    if (kb - warp >= nkb) {
      kb = warp;
      if (++item < to) aim();
    }
  };
  const int steps = (nkb + U * WARPS - 1) / (U * WARPS);
  int done = from, step = 0, buf = 0;                      // the computing side
  float sum[4] = {};                                       // (a step's accumulator starts at zero: the tensor cores cut sums off, and what they lose grows with their number)
  auto compute = [&](const uint4 (&A)[U][4], const uint4 (&B)[U][2]) {
    float acc[4] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 v = A[u][h], w = A[u][2 + h], b = B[u][h];
        ptx::mma_bf16(acc, v.x, w.x, v.y, w.y, b.x, b.y);
        ptx::mma_bf16(acc, v.z, w.z, v.w, w.w, b.z, b.w);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += acc[i];
    if (++step < steps) return;
    step = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      part[buf][warp][2 * t + (i & 1)][g + 8 * (i >> 1)] = sum[i];
      sum[i] = 0.f;
    }
    __syncthreads();                                       // (the buffer before is read by threads that have not passed here again)
    if (threadIdx.x < ROWS * 16) {
      const Where w = locate(done);
      const int r = threadIdx.x >> 4, c = threadIdx.x & 15, o = w.o0 + c;
      if (r < w.rows && o < a.o) {
        const long long row = w.first + r;
        float z = 0.f;
        const float bias = a.bias ? a.bias[(long long)(w.e) * a.o + o] : 0.f, old = a.res ? load_out(a.res, row * a.ldr + o, a.out_dtype) : 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) z += part[buf][i][r][c];
        z = apply_act(z + bias, a.act);
        store_out(a.y, row * a.ldy + o, a.out_dtype, a.res ? z + old : z);
      }
    }
    buf ^= 1;
    ++done;
  };
  aim();
  load(A[0], B[0]);
  while (done < to) {
    if (item < to) load(A[1], B[1]);
    compute(A[0], B[0]);
    if (done == to) break;
    if (item < to) load(A[0], B[0]);
    compute(A[1], B[1]);
  }
}

static tardis_status_t launch_few(const LinearArgs& a, cudaStream_t s) {
  int dev = 0, sms = 0;
  TARDIS_CUDA_TRY(cudaGetDevice(&dev));
  TARDIS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const long long items = (long long)((a.o + 15) / 16) * (a.offsets ? a.n : (a.n + FEW_ROWS - 1) / FEW_ROWS);      // at most (a group's tile has a row)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(items < 2 * sms ? items : 2 * sms)); cfg.blockDim = dim3(FEW_WARPS * 32); cfg.stream = s;
  cfg.dynamicSmemBytes = a.offsets ? groups_bytes(a.groups) : 0;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  TARDIS_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_linear_few, a));
  return TARDIS_OK;
}

// ---- the return to the tokens: bound by reading f ----
// A thread adds up four outputs of a token, its choices in their order (four loads of f under way at a time).  wide: y and the residual are touched four at a time too.
// (Eight CTAs per SM: with six, what more registers than 32 leave, 4096 tokens of 4096 outputs took 194 us with their product, now 177.)
template <typename O>
__global__ void __launch_bounds__(256, 8) k_combine(const __grid_constant__ LinearArgs a, int top_k, const float* f, int ldf, const int* slots,
                                                                  const float* weights, int wide) {
  struct alignas(4 * sizeof(O)) Out { O v[4]; };
  const long long t = blockIdx.x;
  const int c = (blockIdx.y * 256 + threadIdx.x) * 4;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The groups end at the largest offset (none ends before the one before it does): that is the last one, unless offsets fall.
  int hi = 0;
#pragma unroll 4
  for (int e = threadIdx.x & 31; e <= a.groups; e += 32) hi = max(hi, a.offsets[e]);
  hi = min(__reduce_max_sync(0xffffffffu, hi), a.n);
  if (c >= a.o) return;
  const int lo = max(a.offsets[0], 0), count = min(4, a.o - c);
  const O* const res = static_cast<const O*>(a.res) + t * a.ldr + c;
  O* const to = static_cast<O*>(a.y) + t * a.ldy + c;
  float sum[4] = {};
  Out old;
  if (a.res) {
    if (wide) old = *reinterpret_cast<const Out*>(res);
    else {
#pragma unroll
      for (int i = 0; i < 4; ++i) old.v[i] = i < count ? res[i] : from_f32<O>(0.f);
    }
  }
  for (int j0 = 0; j0 < top_k; j0 += 4) {
    float4 part[4];
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = j0 + j < top_k ? slots[t * top_k + j0 + j] : -1;
      const bool there = slot >= lo && slot < hi;
      w[j] = there ? weights[t * top_k + j0 + j] : 0.f;
      part[j] = there ? *reinterpret_cast<const float4*>(f + (long long)(slot) * ldf + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum[0] = fmaf(w[j], part[j].x, sum[0]);
      sum[1] = fmaf(w[j], part[j].y, sum[1]);
      sum[2] = fmaf(w[j], part[j].z, sum[2]);
      sum[3] = fmaf(w[j], part[j].w, sum[3]);
    }
  }
  Out y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y.v[i] = from_f32<O>(a.res ? sum[i] + to_f32(old.v[i]) : sum[i]);
  if (wide) *reinterpret_cast<Out*>(to) = y;
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < count) to[i] = y.v[i];
  }
}

}  // namespace linear

tardis_status_t launch_combine(int tokens, int top_k, const LinearArgs& a, const float* f, int ldf, const int* slots, const float* weights,
                               cudaStream_t s) {
  using namespace linear;
  const size_t unit = a.out_dtype == TARDIS_BF16 ? 2 : 4;
  auto fits = [&](const void* p, long long ld) { return !p || ((reinterpret_cast<uintptr_t>(p) | size_t(ld) * unit) & (4 * unit - 1)) == 0; };
  const int wide = a.o % 4 == 0 && fits(a.y, a.ldy) && fits(a.res, a.ldr);
  if ((a.o + 1023) / 1024 > 65535) return TARDIS_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tokens), unsigned((a.o + 1023) / 1024)); cfg.blockDim = dim3(256); cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  TARDIS_CUDA_TRY(a.out_dtype == TARDIS_BF16 ? cudaLaunchKernelEx(&cfg, k_combine<__nv_bfloat16>, a, top_k, f, ldf, slots, weights, wide)
                                             : cudaLaunchKernelEx(&cfg, k_combine<float>, a, top_k, f, ldf, slots, weights, wide));
  return TARDIS_OK;
}

tardis_status_t launch_linear(const LinearArgs& given, cudaStream_t s) {
  using namespace linear;
  LinearArgs a = given;
  if (a.k > kMostCutOff) a.precise = 1;
  if (a.dtype == TARDIS_F32) return launch_f32(a, s);
  if (a.n <= FEW_ROWS) return launch_few(a, s);
  if (a.n <= 64) {
    // Rows in several cuts of eight where the weights are small: a launch of the tensor-core kernel takes longer to begin and to end.  A step of two blocks of 64 channels
    // for each warp takes 0.9 us or the time of the CTAs' 32 KB each, from memory the first time and from L2 for the other cuts.  (Estimate / measured, us: 16 rows of 4096 ->
    // 4096 13.9 / 12.6, with tcgen05 11.8; 16 of 2048 -> 2048 5.0 / 4.9, 8.1; 24 of 1024 -> 1024 3.6 / 3.7, 7.7; 32 of 1024 -> 4096 8.3 / 9.0, 7.6.)
    int dev = 0, sms = 0;
    TARDIS_CUDA_TRY(cudaGetDevice(&dev));
    TARDIS_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const int groups = a.offsets ? (a.groups < a.n ? a.groups : a.n) : 1, cuts = ((a.n + groups - 1) / groups + FEW_ROWS - 1) / FEW_ROWS;
    const double items = double((a.o + 15) / 16) * cuts * groups, at_once = 2. * sms, running = items < at_once ? items : at_once;
    const double step = fmax(0.9, running * 32768 * (1. / cuts / 6.3e6 + (1. - 1. / cuts) / 8e6));
    const int steps = ((a.k + 63) / 64 + FEW_WARPS * FEW_U - 1) / (FEW_WARPS * FEW_U);
    if (2.4 + ceil(items / at_once) * (0.2 + steps * step) < estimate_linear_tc(a, sms)) return launch_few(a, s);
  }
  return launch_linear_tc(a, s);
}

}  // namespace tardis
