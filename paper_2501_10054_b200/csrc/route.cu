// The router of expert-grouped products: per token the top_k largest logits and their softmax weights, and all (token, choice) pairs sorted
// by expert, stable in the token.
//
// 8, 16 or 32 lanes take a token: its logits lie in registers (lane l of L holds experts l, l + L, ...; the next token's are loaded meanwhile), each of top_k
// rounds takes the largest value by a maximum over an order-preserving integer image and then the lowest expert that has it.  (A warp per token
// executes three times the instructions for 64 experts and four choices: 10 us for 16384 tokens.)  Sorting is counting: a part of the tokens counts its
// choices per expert, the places of a part's pairs start behind those of all smaller experts and of the same expert in earlier parts, and inside a block
// of 128 tokens the earlier tokens of an expert are the set bits below the token's in the expert's bit mask.  Up to 128 tokens are one launch; more
// are two: choices and counts of small parts, then the places.  Nothing waits for another CTA and no order of atomics shows in the result.
#include <limits.h>
#include <math_constants.h>

#include "linear.cuh"

namespace tardis {
namespace route {

constexpr int kBlock = 128;                // tokens whose pairs are placed together: four mask words per expert
constexpr int kMaxParts = 1024;            // rows of counts in the caller's scratch

struct Params {
  int tokens, experts, top_k, normalise;
  int part, parts, per_place;              // tokens of a CTA of the first launch, how many, CTAs of the first launch per CTA of the second
  const float* logits; long long ldl;
  int* chosen; float* weights; int* offsets; int* rows; int* slots;
  int* counts;                             // [parts][experts]
};

// unsigned image of a float that keeps its order (no NaN; -0 has been turned into +0)
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
constexpr uint32_t kNone = 0x007fffffu;                   // ordered(-inf)

template <int L> __device__ __forceinline__ uint32_t most_of(uint32_t v) {          // over the L lanes of a token
  if constexpr (L == 32) return __reduce_max_sync(0xffffffffu, v);
  else {
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
  }
}
template <int L> __device__ __forceinline__ float sum_of(float v) {
#pragma unroll
  for (int d = L / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
template <int L, int PER> __device__ __forceinline__ void fetch(const Params& p, long long t, bool there, int l, float (&f)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) f[i] = there && l + L * i < p.experts ? p.logits[t * p.ldl + l + L * i] : -CUDART_INF_F;
}
// Top-k of the tokens of a converged warp (32 / L of them); lane l < top_k of a token returns its l-th choice (-1: none left) and writes it with its
// weight where the token is there.
template <int L, int PER> __device__ __forceinline__ int choose(const Params& p, long long t, bool there, int l, const float (&f)[PER]) {
  uint32_t v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = f[i] == f[i] ? ordered(f[i] + 0.f) : kNone;       // NaN is no candidate; -0 is +0
  uint32_t most = kNone;
  float top = 0.f, total = 0.f, share = 0.f;
  int mine = -1;
  for (int j = 0; j < p.top_k; ++j) {
    uint32_t best = v[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) best = max(best, v[i]);
    best = most_of<L>(best);
    uint32_t at = 0xffffffffu;                            // the lowest expert that has it, as its complement
#pragma unroll
    for (int i = PER - 1; i >= 0; --i)
      if (v[i] == best) at = l + L * i;
    at = ~most_of<L>(~at);
    if (j == 0) {
      most = best;
      top = unordered(most);
      if (!p.normalise) {                                 // softmax over all: the sum before candidates leave
#pragma unroll
        for (int i = 0; i < PER; ++i) total += v[i] == kNone ? 0.f : v[i] == most ? 1.f : expf(unordered(v[i]) - top);
        total = sum_of<L>(total);
      }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (at == uint32_t(l + L * i)) v[i] = kNone;
    if (l == j && best != kNone) { mine = int(at); share = best == most ? 1.f : expf(unordered(best) - top); }
  }
  if (p.normalise) total = sum_of<L>(share);
  if (there && l < p.top_k) {
    p.chosen[t * p.top_k + l] = mine;
    p.weights[t * p.top_k + l] = mine >= 0 ? share / total : 0.f;
  }
  return there && l < p.top_k ? mine : -1;
}

// Exclusive prefix sum of cnt[0 .. experts) into out[0 .. experts], by one warp.
__device__ __forceinline__ void scan(const int* cnt, int* out, int experts, int lane) {
  int before = 0;
  for (int e0 = 0; e0 < experts; e0 += 32) {
    const int e = e0 + lane, own = e < experts ? cnt[e] : 0;
    int sum = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int other = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += other;
    }
    if (e < experts) out[e] = before + sum - own;
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  if (lane == 0) out[experts] = before;
}

// The places of the pairs of tokens t0 .. t0 + count - 1 (count <= kBlock), whose choices are in `chosen`.  next[e]: the place of expert e's next
// pair; moved on.
__device__ __forceinline__ void place(const Params& p, long long t0, int count, const int* chosen, int* next, uint32_t (*mask)[kBlock / 32]) {
  for (int i = threadIdx.x; i < p.experts * (kBlock / 32); i += blockDim.x) mask[i / (kBlock / 32)][i % (kBlock / 32)] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < count * p.top_k; i += blockDim.x) {
    const int e = chosen[i], t = i / p.top_k;
    if (e >= 0) atomicOr(&mask[e][t >> 5], 1u << (t & 31));
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count * p.top_k; i += blockDim.x) {
    const int e = chosen[i], t = i / p.top_k;
    int slot = -1;
    if (e >= 0) {
      slot = next[e] + __popc(mask[e][t >> 5] & ((1u << (t & 31)) - 1u));
      for (int w = 0; w < (t >> 5); ++w) slot += __popc(mask[e][w]);
      p.rows[slot] = int(t0 + t);
    }
    p.slots[t0 * p.top_k + i] = slot;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
    int c = 0;
    for (int w = 0; w < kBlock / 32; ++w) c += __popc(mask[e][w]);
    next[e] += c;
  }
  __syncthreads();
}

__device__ __forceinline__ void fill_rest(const Params& p, int from, int step0, int step) {
  const long long all = (long long)(p.tokens) * p.top_k;
  for (long long i = (long long)(from) + step0; i < all; i += step) p.rows[i] = -1;
}

// ONLY: the whole call in this launch (32 warps); otherwise choices and counts
template <int L, int PER, bool ONLY> __global__ void __launch_bounds__(ONLY ? 1024 : 512) k_choose(const __grid_constant__ Params p) {
  extern __shared__ int sm[];
  int* const count = sm;                                  // [experts]
  int* const chosen = sm + 6 * p.experts + 1;             // ONLY: [kBlock][top_k]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % L, each = blockDim.x / L;      // each: tokens at a time
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) count[e] = 0;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long t0 = (long long)(blockIdx.x) * p.part;
  const int n = int(min((long long)(p.part), p.tokens - t0));
  float f[PER], g[PER];
  int i = threadIdx.x / L;
  fetch<L, PER>(p, t0 + i, i < n, l, f);
  for (int w = warp * (32 / L); w < n; w += each, i += each) {                  // (w: the warp's first token)
    if (w + each < n) fetch<L, PER>(p, t0 + i + each, i + each < n, l, g);
    const int e = choose<L, PER>(p, t0 + i, i < n, l, f);
    if (e >= 0) atomicAdd(&count[e], 1);
    if (ONLY && i < n && l < p.top_k) chosen[i * p.top_k + l] = e;
#pragma unroll
    for (int j = 0; j < PER; ++j) f[j] = g[j];
  }
  __syncthreads();
  if (ONLY) {
    int* const next = sm + p.experts;                     // [experts + 1]
    if (warp == 0) scan(count, next, p.experts, lane);
    __syncthreads();
    for (int e = threadIdx.x; e <= p.experts; e += blockDim.x) p.offsets[e] = next[e];
    fill_rest(p, next[p.experts], threadIdx.x, blockDim.x);
    __syncthreads();
    place(p, 0, n, chosen, next, reinterpret_cast<uint32_t(*)[kBlock / 32]>(sm + 2 * p.experts + 1));
  } else {
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) p.counts[(long long)(blockIdx.x) * p.experts + e] = count[e];
  }
}

__global__ void __launch_bounds__(512) k_place(const __grid_constant__ Params p) {
  extern __shared__ int sm[];
  int* const all = sm;                                    // [experts] counts of all parts
  int* const next = sm + p.experts;                       // [experts + 1]
  int* const mine = next + p.experts + 1;                 // [experts] counts of the parts before this CTA's
  int* const chosen = mine + 5 * p.experts;               // [kBlock][top_k]; the masks in between
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int e = threadIdx.x; e < p.experts; e += 512) all[e] = mine[e] = 0;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int first = blockIdx.x * p.per_place;
  // threads side by side take experts, sets of them a share of the parts, eight loads under way at a time
  const int wide = min(512, (p.experts + 31) & ~31), sets = 512 / wide, set = threadIdx.x / wide;
  if (set < sets)
    for (int e = threadIdx.x % wide; e < p.experts; e += wide) {
      int sum = 0, before = 0;
      for (int b0 = set; b0 < p.parts; b0 += 8 * sets) {
        int c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = b0 + j * sets < p.parts ? p.counts[(long long)(b0 + j * sets) * p.experts + e] : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum += c[j];
          before += b0 + j * sets < first ? c[j] : 0;
        }
      }
      atomicAdd(&all[e], sum);
      atomicAdd(&mine[e], before);
    }
  __syncthreads();
  if (warp == 0) scan(all, next, p.experts, lane);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= p.experts; e += 512) p.offsets[e] = next[e];
  fill_rest(p, next[p.experts], blockIdx.x * 512 + threadIdx.x, gridDim.x * 512);
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += 512) next[e] += mine[e];
  const long long t0 = (long long)(first) * p.part;
  const int n = int(min((long long)(p.part) * p.per_place, p.tokens - t0));
  for (int i = 0; i < n; i += kBlock) {
    const int count = min(kBlock, n - i);
    for (int j = threadIdx.x; j < count * p.top_k; j += 512) chosen[j] = p.chosen[(t0 + i) * p.top_k + j];
    __syncthreads();
    place(p, t0 + i, count, chosen, next, reinterpret_cast<uint32_t(*)[kBlock / 32]>(mine + p.experts));
  }
}

static tardis_status_t launch(void (*kernel)(Params), const Params& p, int blocks, int threads, int words, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(blocks)); cfg.blockDim = dim3(unsigned(threads)); cfg.dynamicSmemBytes = words * 4; cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  TARDIS_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p));
  return TARDIS_OK;
}
template <int L, int PER> static tardis_status_t launch_choose(const Params& p, cudaStream_t s) {
  if (p.parts == 1) return launch(k_choose<L, PER, true>, p, 1, 1024, 6 * p.experts + 1 + kBlock * p.top_k, s);
  return launch(k_choose<L, PER, false>, p, p.parts, 512, p.experts, s);
}

}  // namespace route

tardis_status_t launch_route(int tokens, int experts, int top_k, int normalise, const float* logits, long long ldl, int* chosen,
                             float* weights, int* offsets, int* rows, int* slots, int* work, cudaStream_t s) {
  using namespace route;
  Params p = {tokens, experts, top_k, normalise, kBlock, 1, 1, logits, ldl, chosen, weights, offsets, rows, slots, work};
  const bool narrow = top_k <= 8 && experts <= 64, half = top_k <= 16 && experts <= 128;
  if (tokens > kBlock) {
    p.part = narrow ? 64 : 32;                             // one or two passes of a CTA's 16 warps
    while ((tokens - 1) / p.part >= kMaxParts) p.part *= 2;
    p.parts = (tokens - 1) / p.part + 1;
    p.per_place = p.part < kBlock ? kBlock / p.part : 1;
  }
  tardis_status_t st = narrow ? (experts <= 8 ? launch_choose<8, 1>(p, s) : experts <= 32 ? launch_choose<8, 4>(p, s) : launch_choose<8, 8>(p, s))
                     : half ? launch_choose<16, 8>(p, s) : experts <= 128 ? launch_choose<32, 4>(p, s)
                     : experts <= 256 ? launch_choose<32, 8>(p, s) : launch_choose<32, 32>(p, s);
  if (st == TARDIS_OK && p.parts > 1)
    st = launch(k_place, p, (p.parts - 1) / p.per_place + 1, 512, 7 * experts + 1 + kBlock * top_k, s);
  return st;
}

}  // namespace tardis
