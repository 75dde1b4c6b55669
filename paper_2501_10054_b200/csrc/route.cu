// The router of expert-grouped products: per token the top_k largest logits and their softmax weights, and all (token, choice) pairs sorted
// by expert, stable in the token.
//
// A warp takes a token: its logits lie in registers (lane l holds experts l, l + 32, ...; the next token's are loaded meanwhile), each of top_k rounds takes
// the largest value by a warp-wide maximum over an order-preserving integer image and then the lowest expert that has it.  Sorting is counting: a
// part of the tokens counts its choices per expert, the places of a part's pairs start behind those of all smaller experts and of the same expert in
// earlier parts, and inside a block of 128 tokens the earlier tokens of an expert are the set bits below the token's in the expert's bit mask.  Up to
// 128 tokens are one launch; more are two: choices and counts of small parts (two tokens per warp of 16: the rounds are a chain of latencies), then the
// places.  Nothing waits for another CTA and no order of atomics shows in the result.
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

template <int PER> __device__ __forceinline__ void fetch(const Params& p, long long t, int lane, float (&f)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) f[i] = lane + 32 * i < p.experts ? p.logits[t * p.ldl + lane + 32 * i] : -CUDART_INF_F;
}
// Top-k of one token by a converged warp; lane j < top_k returns its j-th choice (-1: none left) and writes it with its weight.
template <int PER> __device__ __forceinline__ int choose(const Params& p, long long t, int lane, const float (&f)[PER]) {
  uint32_t v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = f[i] == f[i] ? ordered(f[i] + 0.f) : kNone;       // NaN is no candidate; -0 is +0
  // softmax over all: the sum before candidates leave
  uint32_t most = v[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) most = max(most, v[i]);
  most = __reduce_max_sync(0xffffffffu, most);
  const float top = unordered(most);
  float total = 0.f;
  if (!p.normalise && most > kNone) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (v[i] > kNone) total += v[i] == most ? 1.f : expf(unordered(v[i]) - top);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  }
  int mine = -1;
  float share = 0.f;
  for (int j = 0; j < p.top_k; ++j) {
    uint32_t best = v[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) best = max(best, v[i]);
    best = __reduce_max_sync(0xffffffffu, best);
    if (best <= kNone) break;                             // (uniform)
    int at = INT_MAX;
#pragma unroll
    for (int i = PER - 1; i >= 0; --i)
      if (v[i] == best) at = lane + 32 * i;
    at = int(__reduce_min_sync(0xffffffffu, unsigned(at)));
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (at == lane + 32 * i) v[i] = kNone;
    if (lane == j) { mine = at; share = best == most ? 1.f : expf(unordered(best) - top); }
  }
  if (p.normalise) {
    total = share;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  }
  if (lane < p.top_k) {
    p.chosen[t * p.top_k + lane] = mine;
    p.weights[t * p.top_k + lane] = mine >= 0 ? share / total : 0.f;
  }
  return mine;
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
template <int PER, bool ONLY> __global__ void __launch_bounds__(ONLY ? 1024 : 512) k_choose(const __grid_constant__ Params p) {
  extern __shared__ int sm[];
  int* const count = sm;                                  // [experts]
  int* const chosen = sm + 6 * p.experts + 1;             // ONLY: [kBlock][top_k]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) count[e] = 0;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long t0 = (long long)(blockIdx.x) * p.part;
  const int n = int(min((long long)(p.part), p.tokens - t0));
  float f[PER], g[PER];
  if (warp < n) fetch<PER>(p, t0 + warp, lane, f);
  for (int i = warp; i < n; i += warps) {
    if (i + warps < n) fetch<PER>(p, t0 + i + warps, lane, g);
    const int e = choose<PER>(p, t0 + i, lane, f);
    if (e >= 0) atomicAdd(&count[e], 1);
    if (ONLY && lane < p.top_k) chosen[i * p.top_k + lane] = e;
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
template <int PER> static tardis_status_t launch_choose(const Params& p, cudaStream_t s) {
  if (p.parts == 1) return launch(k_choose<PER, true>, p, 1, 1024, 6 * p.experts + 1 + kBlock * p.top_k, s);
  return launch(k_choose<PER, false>, p, p.parts, 512, p.experts, s);
}

}  // namespace route

tardis_status_t launch_route(int tokens, int experts, int top_k, int normalise, const float* logits, long long ldl, int* chosen,
                             float* weights, int* offsets, int* rows, int* slots, int* work, cudaStream_t s) {
  using namespace route;
  Params p = {tokens, experts, top_k, normalise, kBlock, 1, 1, logits, ldl, chosen, weights, offsets, rows, slots, work};
  if (tokens > kBlock) {
    p.part = 32;
    while ((tokens - 1) / p.part >= kMaxParts) p.part *= 2;
    p.parts = (tokens - 1) / p.part + 1;
    p.per_place = p.part < kBlock ? kBlock / p.part : 1;
  }
  tardis_status_t st = experts <= 32 ? launch_choose<1>(p, s) : experts <= 64 ? launch_choose<2>(p, s) : experts <= 128 ? launch_choose<4>(p, s)
                     : experts <= 256 ? launch_choose<8>(p, s) : launch_choose<32>(p, s);
  if (st == TARDIS_OK && p.parts > 1)
    st = launch(k_place, p, (p.parts - 1) / p.per_place + 1, 512, 7 * experts + 1 + kBlock * top_k, s);
  return st;
}

}  // namespace tardis
