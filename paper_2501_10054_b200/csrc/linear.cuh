// The dense products of the feed-forward blocks that stay unfolded (internal): what the kernels of linear.cu (fp32, few rows)
// and linear_tc.cu (tensor cores) take.
//   y[r, o] = act(sum_k x[row(r), k] W_e[o, k] + bias_e[o]) + res[r, o]       e = the group of row r
#pragma once
#include "common.cuh"

namespace tardis {

constexpr int kMaxExperts = 1024;
constexpr int kMostCutOff = 1 << 17;   // channels whose sum may be cut off at every instruction, 1.5e-8 of it each: 1.2e-4, 1/32 of half a step of bf16

struct LinearArgs {
  int n, k, o;                       // rows of the output, channels, outputs
  int dtype, out_dtype, act;         // act: TARDIS_ACT_NONE or one of tardis_act_t
  int precise;                       // sums are not left to the tensor cores' cut-off: the call's result is fp32 (out_dtype is, too, where bf16 results are put together from fp32),
                                     // or there are more than kMostCutOff channels
  const void* x; long long ldx;      // [nx, k]
  int nx;
  const void* W; long long ldw, stride_w;      // [groups][o, k]
  const float* bias;                 // [groups][o] or null
  const void* res; long long ldr;    // [n, o] in out_dtype or null
  void* y; long long ldy;
  int groups;                        // 1 without offsets
  const int* offsets;                // [groups + 1] or null (one group of all rows)
  void* work;                        // with rows: [n, k] in bf16, where they may be gathered, or null
  const int* rows;                   // [n] or null: row r of the product takes row rows[r] of x (zeros where that is outside [0, nx))
};

tardis_status_t launch_linear(const LinearArgs& a, cudaStream_t s);
tardis_status_t launch_linear_tc(const LinearArgs& a, cudaStream_t s);       // bf16, n > 0
double estimate_linear_tc(const LinearArgs& a, int sms);                     // us it will take
// What a gives in fp32 as f [a.n, a.o] (rows of ldf, a multiple of 4), returned to the tokens: a.y[t, o] = a.res[t, o] + sum_j weights[t, j] f[slots[t, j], o]; slots outside
// the groups add nothing
tardis_status_t launch_combine(int tokens, int top_k, const LinearArgs& a, const float* f, int ldf, const int* slots, const float* weights,
                               cudaStream_t s);
tardis_status_t launch_route(int tokens, int experts, int top_k, int normalise, const float* logits, long long ldl, int* chosen,
                             float* weights, int* offsets, int* rows, int* slots, int* work, cudaStream_t s);

// ---- device side ----
// One thread's view of the grouped rows.  Offsets come from device memory: each is clamped to [0, n] and to its predecessors, so whatever
// they hold, groups are disjoint and inside the output.
struct GroupTile { int e, first, rows; };     // group, first row of the tile, rows of the tile (0: no such tile)

// Tile `tile` of the sequence that cuts every group into tiles of `per` rows, groups in order, by one converged warp (all lanes get it).
__device__ __forceinline__ GroupTile find_group_tile(const int* offsets, int groups, int n, int per, int tile) {
  GroupTile t = {0, 0, 0};
  if (!offsets) {
    const long long first = (long long)(tile) * per;
    if (first < n) { t.first = int(first); t.rows = min(per, n - int(first)); }
    return t;
  }
  const int lane = threadIdx.x & 31;
  int end = min(max(offsets[0], 0), n), before = 0;          // where the groups so far end, and their tiles
  for (int e0 = 0; e0 < groups; e0 += 32) {
    const int e = e0 + lane;
    int mine = e < groups ? min(max(offsets[e + 1], 0), n) : 0;
    mine = max(mine, end);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, mine, d);
      if (lane >= d) mine = max(mine, other);
    }
    int start = __shfl_up_sync(0xffffffffu, mine, 1);
    if (lane == 0) start = end;
    int tiles = (mine - start + per - 1) / per;
    const int own = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, tiles, d);
      if (lane >= d) tiles += other;
    }
    const int skip = before + tiles - own;                    // tiles in front of this lane's group
    const unsigned hit = __ballot_sync(0xffffffffu, tile >= skip && tile < skip + own);
    if (hit) {
      const int src = __ffs(hit) - 1;
      const int g_first = __shfl_sync(0xffffffffu, start, src), g_end = __shfl_sync(0xffffffffu, mine, src);
      t.e = e0 + src;
      t.first = g_first + (tile - __shfl_sync(0xffffffffu, skip, src)) * per;
      t.rows = min(per, g_end - t.first);
      return t;
    }
    end = __shfl_sync(0xffffffffu, mine, 31);
    before += __shfl_sync(0xffffffffu, tiles, 31);
  }
  return t;
}

// The same as a table in shared memory, made by all threads of a CTA (callers synchronise afterwards).  The groups come in order of falling size where
// there are at most kSorted of them (equal sizes in their own order): the tiles that take longest first, the tail of a launch is made of short ones.
constexpr int kSorted = 256;
struct Groups {
  int* starts;      // [groups + 1] where group e begins; it ends at starts[e + 1]
  int* firsts;      // [groups + 1] tiles in front of the i-th group of the order
  int* order;       // [groups] the i-th group (before the table is complete: sizes)
};
__host__ __device__ constexpr int groups_bytes(int groups) { return 4 * (3 * groups + 2); }
__device__ __forceinline__ Groups groups_at(void* p, int groups) {
  int* const at = static_cast<int*>(p);
  return {at, at + groups + 1, at + 2 * groups + 2};
}
// per: rows of a tile; each: tiles that so many rows make
__device__ __forceinline__ void build_groups(const int* offsets, int groups, int n, int per, int each, Groups t) {
  for (int e = threadIdx.x; e <= groups; e += blockDim.x) t.starts[e] = min(max(offsets[e], 0), n);
  __syncthreads();
  const int lane = threadIdx.x & 31;
  if (threadIdx.x < 32) {
    int end = t.starts[0];
    __syncwarp();
    for (int e0 = 0; e0 < groups; e0 += 32) {
      const int e = e0 + lane;
      int mine = e < groups ? max(t.starts[e + 1], end) : end;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int other = __shfl_up_sync(0xffffffffu, mine, d);
        if (lane >= d) mine = max(mine, other);
      }
      if (e < groups) t.starts[e + 1] = mine;
      end = __shfl_sync(0xffffffffu, mine, 31);
      __syncwarp();
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < groups; e += blockDim.x) {
    int place = e;
    if (groups <= kSorted) {
      const int size = t.starts[e + 1] - t.starts[e];
      place = 0;
      for (int f = 0; f < groups; ++f) {
        const int other = t.starts[f + 1] - t.starts[f];
        place += other > size || (other == size && f < e) ? 1 : 0;
      }
    }
    t.order[place] = e;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    int before = 0;
    for (int i0 = 0; i0 < groups; i0 += 32) {
      const int i = i0 + lane, e = i < groups ? t.order[i] : 0;
      const int own = i < groups ? (t.starts[e + 1] - t.starts[e] + per - 1) / per * each : 0;
      int tiles = own;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int other = __shfl_up_sync(0xffffffffu, tiles, d);
        if (lane >= d) tiles += other;
      }
      if (i < groups) t.firsts[i] = before + tiles - own;
      before += __shfl_sync(0xffffffffu, tiles, 31);
    }
    if (lane == 0) t.firsts[groups] = before;
  }
}
// the place in the order of the group that has tile `tile` (below firsts[groups])
__device__ __forceinline__ int place_of(const Groups& t, int groups, int tile) {
  int lo = 0, hi = groups;                                   // the last group whose first tile is not behind this one
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.firsts[mid] <= tile) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The activations, in one form for all kernels here, so that a token's values do not depend on how many others come with it.  Neither takes a difference of numbers near 1:
// the negative tails keep their relative accuracy, some units of 2^-24 times z^2 (0.5 z (1 + erf(..)) in fp32 is off by a third at -5).  The erf form: z Phi(z) = max(z, 0) - |z| / 2
// erfc(|z| / sqrt 2), erfc by the Chebyshev fit of Press et al., Numerical Recipes, section 6.2 (relative error below 1.2e-7 everywhere).  777 tokens of 4544 -> 18176 take 103
// us without activation, 107 with the tanh form, 112 with this, 120 with erfcf.
__device__ __forceinline__ float gelu_erf_fit(float z) {
  const float x = fabsf(z) * 0.7071067811865476f, t = __fdividef(1.f, fmaf(0.5f, x, 1.f));
  float p = fmaf(0.17087277f, t, -0.82215223f);
  p = fmaf(p, t, 1.48851587f);
  p = fmaf(p, t, -1.13520398f);
  p = fmaf(p, t, 0.27886807f);
  p = fmaf(p, t, -0.18628806f);
  p = fmaf(p, t, 0.09678418f);
  p = fmaf(p, t, 0.37409196f);
  p = fmaf(p, t, 1.00002368f);
  p = fmaf(p, t, -1.26551223f);
  const float half = 0.5f * z;
  return (half + fabsf(half)) - fminf(fabsf(half), 3.0e38f) * (t * __expf(fmaf(-x, x, p)));
}
__device__ __forceinline__ float apply_act(float z, int act) {
  if (act == TARDIS_ACT_NONE) return z;
  if (act == TARDIS_ACT_RELU) return z < 0.f ? 0.f : z;              // (of -inf 0, of NaN NaN)
  return act == TARDIS_ACT_GELU_TANH ? gelu_tanh_f32(z) : gelu_erf_fit(z);
}
__device__ __forceinline__ float load_out(const void* p, long long i, int dtype) {
  return dtype == TARDIS_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_out(void* p, long long i, int dtype, float v) {
  if (dtype == TARDIS_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<float*>(p)[i] = v;
}

}  // namespace tardis
