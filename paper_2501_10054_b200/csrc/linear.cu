// The dense products of unfolded feed-forward blocks: dispatch, the kernel for every type and size, the weighted return to the tokens.
#include "linear.cuh"
#include "ptx.cuh"

namespace tardis {
namespace linear {

// ---- fp32: plain multiply-adds ----
// 256 threads compute a tile of 16 T outputs x 16 T rows, T x T of them each, over steps of 16 channels in shared memory (channel-major, so that a thread
// reads its T outputs and its T rows as vectors); the next step's operands are on their way into registers meanwhile.
template <int T> struct alignas(T > 4 ? 16 : 4 * T) Vec { float v[T]; };

template <int T>
__global__ void __launch_bounds__(256) k_linear_f32(const __grid_constant__ LinearArgs a) {
  constexpr int TILE = 16 * T, BK = 16, LD = TILE + 4, PER = TILE * BK / 4 / 256 + (TILE * BK / 4 % 256 != 0);     // PER: 16-byte loads per thread and operand
  __shared__ __align__(16) float sw[BK][LD], sx[BK][LD];
  const GroupTile t = find_group_tile(a.offsets, a.groups, a.n, TILE, blockIdx.x);
  if (t.rows == 0) return;
  const int o0 = blockIdx.y * TILE, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;      // tx: outputs, ty: rows
  const float *w[PER], *x[PER];                              // this thread's rows of W and x (null: zeros), four channels at a time
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = threadIdx.x + 256 * i, r = at / (BK / 4);
    w[i] = x[i] = nullptr;
    if (at >= TILE * BK / 4) continue;
    if (o0 + r < a.o) w[i] = static_cast<const float*>(a.W) + t.e * a.stride_w + (o0 + r) * a.ldw + at % (BK / 4) * 4;
    if (r < t.rows) {
      const int src = a.rows ? a.rows[t.first + r] : t.first + r;
      if (src >= 0 && src < a.nx) x[i] = static_cast<const float*>(a.x) + src * a.ldx + at % (BK / 4) * 4;
    }
  }
  float4 nw[PER], nx[PER];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool in = k0 + int(threadIdx.x + 256 * i) % (BK / 4) * 4 < a.k;
      nw[i] = in && w[i] ? *reinterpret_cast<const float4*>(w[i] + k0) : make_float4(0.f, 0.f, 0.f, 0.f);
      nx[i] = in && x[i] ? *reinterpret_cast<const float4*>(x[i] + k0) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  float acc[T][T] = {};
  load(0);
  for (int k0 = 0; k0 < a.k; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x + 256 * i, r = at / (BK / 4), c = at % (BK / 4) * 4;
      if (at >= TILE * BK / 4) continue;
      sw[c][r] = nw[i].x; sw[c + 1][r] = nw[i].y; sw[c + 2][r] = nw[i].z; sw[c + 3][r] = nw[i].w;
      sx[c][r] = nx[i].x; sx[c + 1][r] = nx[i].y; sx[c + 2][r] = nx[i].z; sx[c + 3][r] = nx[i].w;
    }
    __syncthreads();
    if (k0 + BK < a.k) load(k0 + BK);
#pragma unroll
    for (int kk = 0; kk < BK; ++kk) {
      const Vec<T> v = *reinterpret_cast<const Vec<T>*>(&sx[kk][ty * T]), u = *reinterpret_cast<const Vec<T>*>(&sw[kk][tx * T]);
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j) acc[i][j] = fmaf(v.v[i], u.v[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < T; ++i) {
    const int r = ty * T + i;
    if (r >= t.rows) continue;
    const long long row = t.first + r;
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int o = o0 + tx * T + j;
      if (o >= a.o) continue;
      float z = acc[i][j];
      if (a.bias) z += a.bias[(long long)(t.e) * a.o + o];
      z = apply_act(z, a.act);
      if (a.res) z += static_cast<const float*>(a.res)[row * a.ldr + o];
      static_cast<float*>(a.y)[row * a.ldy + o] = z;
    }
  }
}

template <int T>
static tardis_status_t launch_f32_tiles(const LinearArgs& a, cudaStream_t s) {
  const int tile = 16 * T;
  const long long tiles = (a.n + tile - 1) / tile + (a.offsets ? (a.groups < a.n ? a.groups : a.n) : 0);     // at most
  const int outputs = (a.o + tile - 1) / tile;
  if (outputs > 65535) return TARDIS_ERR_UNSUPPORTED;
  k_linear_f32<T><<<dim3(unsigned(tiles), unsigned(outputs)), 256, 0, s>>>(a);
  TARDIS_CUDA_TRY(cudaGetLastError());
  return TARDIS_OK;
}

// Up to eight rows of fp32: a CTA has four outputs, its eight warps share the channels (a lane four at a time) and add their parts in a fixed order.
__global__ void __launch_bounds__(256) k_linear_few_f32(const __grid_constant__ LinearArgs a) {
  constexpr int O = 4, ROWS = 8;
  __shared__ float part[8][O * ROWS];
  const GroupTile t = find_group_tile(a.offsets, a.groups, a.n, ROWS, blockIdx.y);
  if (t.rows == 0) return;
  const int o0 = blockIdx.x * O, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float *w[O], *x[ROWS];
#pragma unroll
  for (int i = 0; i < O; ++i) w[i] = static_cast<const float*>(a.W) + t.e * a.stride_w + min(o0 + i, a.o - 1) * a.ldw;
  bool there[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    int src = -1;
    if (r < t.rows) src = a.rows ? a.rows[t.first + r] : t.first + r;
    there[r] = src >= 0 && src < a.nx;
    x[r] = static_cast<const float*>(a.x) + (there[r] ? src : 0) * a.ldx;
  }
  float acc[O][ROWS] = {};
  for (int k = threadIdx.x * 4; k < a.k; k += 1024) {
    float4 wv[O];
#pragma unroll
    for (int i = 0; i < O; ++i) wv[i] = *reinterpret_cast<const float4*>(w[i] + k);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (!there[r]) continue;
      const float4 xv = *reinterpret_cast<const float4*>(x[r] + k);
#pragma unroll
      for (int i = 0; i < O; ++i) acc[i][r] = fmaf(wv[i].w, xv.w, fmaf(wv[i].z, xv.z, fmaf(wv[i].y, xv.y, fmaf(wv[i].x, xv.x, acc[i][r]))));
    }
  }
#pragma unroll
  for (int i = 0; i < O; ++i)
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float v = acc[i][r];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
      if (lane == 0) part[warp][r * O + i] = v;
    }
  __syncthreads();
  const int r = threadIdx.x / O, o = o0 + threadIdx.x % O;
  if (threadIdx.x >= O * ROWS || r >= t.rows || o >= a.o) return;
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
    const unsigned tiles = a.offsets ? unsigned(a.n) : 1u;                             // at most (a group's tile has a row)
    k_linear_few_f32<<<dim3(unsigned((a.o + 3) / 4), tiles), 256, 0, s>>>(a);
    TARDIS_CUDA_TRY(cudaGetLastError());
    return TARDIS_OK;
  }
  // the largest tiles that give every SM one: few rows and outputs are all latency
  const long long groups = a.offsets ? a.groups : 1, rows = (a.n + groups - 1) / groups;
  auto tiles = [&](int tile) { return (a.o + tile - 1) / tile * (groups * ((rows + tile - 1) / tile)); };
  if (tiles(128) >= 148) return launch_f32_tiles<8>(a, s);
  return tiles(64) >= 148 ? launch_f32_tiles<4>(a, s) : launch_f32_tiles<2>(a, s);
}

// ---- up to eight rows of bf16: bound by reading the weights once ----
// An item is 16 outputs of up to 8 rows of a group.  Weights go straight from global memory into the A fragments of mma.m16n8k16 and the rows of x into its B
// fragments: a sum over channels may be taken in any order, so lane (g, t) reads 16 bytes, channels 8 t .. 8 t + 7 of a block of 32, of weight rows
// g and g + 8 and of row g of x, and each pair of words is the fragment of one instruction.  The eight warps of a CTA share the channels in blocks
// of 64, taken in turn, so that together they read whole lines of every weight row; their parts are added in a fixed order.  Two CTAs per SM
// walk the items (a contiguous run each, outputs first), and the loads of the next step, of the next item too, are under way while one is
// multiplied, summed up and stored.
constexpr int FEW_ROWS = 8, FEW_WARPS = 8, FEW_U = 2;      // U: blocks of 64 channels of a warp and step

__global__ void __launch_bounds__(FEW_WARPS * 32, 2) k_linear_few(const __grid_constant__ LinearArgs a) {
  constexpr int ROWS = FEW_ROWS, WARPS = FEW_WARPS, U = FEW_U;
  extern __shared__ int table[];                           // (grouped only)
  __shared__ float part[2][WARPS][ROWS][17];
  const Groups groups = groups_at(table, a.groups);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int nkb = (a.k + 63) / 64, ot = (a.o + 15) / 16;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (!a.offsets) {                                        // while the launch before ends: the first steps' weights on their way into L2
    const int o0 = int((long long)(blockIdx.x) * ot / gridDim.x) * 16;
    const __nv_bfloat16* const w = static_cast<const __nv_bfloat16*>(a.W) + min(o0 + (lane & 15), a.o - 1) * a.ldw;
    for (int kb = warp + (lane >> 4) * WARPS; kb < min(nkb, 2 * U * WARPS); kb += 2 * WARPS) asm volatile("prefetch.global.L2 [%0];" ::"l"(w + kb * 64));
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (a.offsets) {
    build_groups(a.offsets, a.groups, a.n, ROWS, ot, groups);
    __syncthreads();
  }
  const int items = a.offsets ? groups.firsts[a.groups] : ot;
  const int from = int((long long)(blockIdx.x) * items / gridDim.x), to = int((long long)(blockIdx.x + 1) * items / gridDim.x);
  if (from == to) return;

  struct Where { int e, o0, first, rows; };
  auto locate = [&](int item) {
    Where w = {0, item * 16, 0, a.n};
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
        A[u][h] = in ? ptx::ldg_stream(w0 + k) : make_uint4(0u, 0u, 0u, 0u);
        A[u][2 + h] = in ? ptx::ldg_stream(w1 + k) : make_uint4(0u, 0u, 0u, 0u);
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
  float acc[4] = {};
  auto compute = [&](const uint4 (&A)[U][4], const uint4 (&B)[U][2]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 v = A[u][h], w = A[u][2 + h], b = B[u][h];
        ptx::mma_bf16(acc, v.x, w.x, v.y, w.y, b.x, b.y);
        ptx::mma_bf16(acc, v.z, w.z, v.w, w.w, b.z, b.w);
      }
    if (++step < steps) return;
    step = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      part[buf][warp][2 * t + (i & 1)][g + 8 * (i >> 1)] = acc[i];
      acc[i] = 0.f;
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
  const long long items = (long long)((a.o + 15) / 16) * (a.offsets ? a.n : 1);      // at most (a group's tile has a row)
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
// A thread adds up V outputs of a token, its choices in their order (four loads of f under way at a time).
template <int V, typename O>
__global__ void __launch_bounds__(256) k_combine(const __grid_constant__ LinearArgs a, int top_k, const float* __restrict__ f,
                                                 const int* __restrict__ slots, const float* __restrict__ weights) {
  const long long t = blockIdx.x;
  const int c = (blockIdx.y * 256 + threadIdx.x) * V;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (c >= a.o) return;
  const int lo = max(a.offsets[0], 0), hi = min(a.offsets[a.groups], a.n);
  Vec<V> sum = {};
  struct alignas(sizeof(O) * V) Out { O v[V]; };
  Out old;
  if (a.res) old = *reinterpret_cast<const Out*>(static_cast<const O*>(a.res) + t * a.ldr + c);
  for (int j0 = 0; j0 < top_k; j0 += 4) {
    Vec<V> part[4];
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = j0 + j < top_k ? slots[t * top_k + j0 + j] : -1;
      const bool there = slot >= lo && slot < hi;
      w[j] = there ? weights[t * top_k + j0 + j] : 0.f;
      part[j] = there ? *reinterpret_cast<const Vec<V>*>(f + (long long)(slot) * a.o + c) : Vec<V>{};
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) sum.v[i] = fmaf(w[j], part[j].v[i], sum.v[i]);
  }
  Out y;
#pragma unroll
  for (int i = 0; i < V; ++i) y.v[i] = from_f32<O>(a.res ? sum.v[i] + to_f32(old.v[i]) : sum.v[i]);
  *reinterpret_cast<Out*>(static_cast<O*>(a.y) + t * a.ldy + c) = y;
}

template <int V, typename O>
static tardis_status_t launch_combine_as(int tokens, int top_k, const LinearArgs& a, const float* f, const int* slots, const float* weights,
                                         cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tokens), unsigned((a.o + 256 * V - 1) / (256 * V))); cfg.blockDim = dim3(256); cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  TARDIS_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_combine<V, O>, a, top_k, f, slots, weights));
  return TARDIS_OK;
}

}  // namespace linear

tardis_status_t launch_combine(int tokens, int top_k, const LinearArgs& a, const float* f, const int* slots, const float* weights,
                               cudaStream_t s) {
  using namespace linear;
  const size_t unit = a.out_dtype == TARDIS_BF16 ? 2 : 4;
  auto fits = [&](const void* p, long long ld) { return !p || ((reinterpret_cast<uintptr_t>(p) | size_t(ld) * unit) & (4 * unit - 1)) == 0; };
  const bool wide = a.o % 4 == 0 && fits(a.y, a.ldy) && fits(a.res, a.ldr);        // four outputs at a time
  if (a.o > 65535 * 256) return TARDIS_ERR_UNSUPPORTED;
  if (a.out_dtype == TARDIS_BF16)
    return wide ? launch_combine_as<4, __nv_bfloat16>(tokens, top_k, a, f, slots, weights, s) : launch_combine_as<1, __nv_bfloat16>(tokens, top_k, a, f, slots, weights, s);
  return wide ? launch_combine_as<4, float>(tokens, top_k, a, f, slots, weights, s) : launch_combine_as<1, float>(tokens, top_k, a, f, slots, weights, s);
}

tardis_status_t launch_linear(const LinearArgs& a, cudaStream_t s) {
  using namespace linear;
  if (a.dtype == TARDIS_BF16 && a.n <= FEW_ROWS) return launch_few(a, s);
  return a.dtype == TARDIS_BF16 ? launch_linear_tc(a, s) : launch_f32(a, s);
}

}  // namespace tardis
