// The router of expert-grouped products: per token the top_k largest logits and their softmax weights, and all (token, choice) pairs sorted
// by expert, stable in the token.
//
// A warp takes a token: its logits lie in registers (lane l holds experts l, l + 32, ...), each of top_k rounds takes the largest value by a
// warp-wide maximum over an order-preserving integer image and then the lowest expert that has it.  Sorting is counting: a block of tokens
// counts its choices per expert, the places of a block's pairs start behind those of all smaller experts and of the same expert in earlier
// blocks, and inside a block the earlier tokens of an expert are the set bits below the token's in the expert's bit mask.  Up to kBlock tokens
// are one launch; more are two, with the counts of at most kMaxBlocks blocks in the caller's scratch.  Nothing waits for another CTA and no
// order of atomics shows in the result.
#include <limits.h>
#include <math_constants.h>

#include "linear.cuh"

namespace tardis {
namespace route {

constexpr int kBlock = 128;                // tokens per pass of a CTA: four mask words per expert
constexpr int kMaxBlocks = 256;
constexpr int kThreads = 512, kWarps = kThreads / 32;

struct Params {
  int tokens, experts, top_k, normalise, per_block;       // per_block: tokens of a CTA
  const float* logits; long long ldl;
  int* chosen; float* weights; int* offsets; int* rows; int* slots;
  int* counts;                                            // [blocks][experts]
};

// unsigned image of a float that keeps its order (no NaN; -0 has been turned into +0)
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
constexpr uint32_t kNone = 0x007fffffu;                   // ordered(-inf)

// Top-k of one token by a converged warp; lane j < top_k returns its j-th choice (-1: none left) and writes it with its weight.
template <int PER> __device__ __forceinline__ int choose(const Params& p, long long t, int lane) {
  uint32_t v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 32 * i;
    float f = e < p.experts ? p.logits[t * p.ldl + e] + 0.f : -CUDART_INF_F;
    v[i] = f == f ? ordered(f) : kNone;                   // NaN is no candidate
  }
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

// The places of the pairs of tokens t0 .. t0 + count - 1 (count <= kBlock).  next[e]: the place of expert e's next pair; moved on.
__device__ __forceinline__ void place(const Params& p, long long t0, int count, int* next, uint32_t (*mask)[kBlock / 32]) {
  for (int i = threadIdx.x; i < p.experts * (kBlock / 32); i += kThreads) mask[i / (kBlock / 32)][i % (kBlock / 32)] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < count * p.top_k; i += kThreads) {
    const int e = p.chosen[t0 * p.top_k + i], t = i / p.top_k;
    if (e >= 0) atomicOr(&mask[e][t >> 5], 1u << (t & 31));
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count * p.top_k; i += kThreads) {
    const int e = p.chosen[t0 * p.top_k + i], t = i / p.top_k;
    int slot = -1;
    if (e >= 0) {
      slot = next[e] + __popc(mask[e][t >> 5] & ((1u << (t & 31)) - 1u));
      for (int w = 0; w < (t >> 5); ++w) slot += __popc(mask[e][w]);
      p.rows[slot] = int(t0 + t);
    }
    p.slots[t0 * p.top_k + i] = slot;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += kThreads) {
    int c = 0;
    for (int w = 0; w < kBlock / 32; ++w) c += __popc(mask[e][w]);
    next[e] += c;
  }
  __syncthreads();
}

__device__ __forceinline__ void fill_rest(const Params& p, int from, int step0, int step) {
  const long long all = (long long)(p.tokens) * p.top_k;
  for (long long i = from + step0; i < all; i += step) p.rows[i] = -1;
}

// ONLY: the whole call in this launch; otherwise choices and counts
template <int PER, bool ONLY> __global__ void __launch_bounds__(kThreads) k_choose(const Params p) {
  extern __shared__ int sm[];
  int* const count = sm;                                  // [experts]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int e = threadIdx.x; e < p.experts; e += kThreads) count[e] = 0;
  __syncthreads();
  const long long t0 = (long long)(blockIdx.x) * p.per_block;
  const int n = int(min((long long)(p.per_block), p.tokens - t0));
  for (int i = warp; i < n; i += kWarps) {
    const int e = choose<PER>(p, t0 + i, lane);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  if (ONLY) {
    int* const next = sm + p.experts;                     // [experts + 1]
    if (warp == 0) scan(count, next, p.experts, lane);
    __syncthreads();
    for (int e = threadIdx.x; e <= p.experts; e += kThreads) p.offsets[e] = next[e];
    const int end = next[p.experts];
    __syncthreads();
    fill_rest(p, end, threadIdx.x, kThreads);
    place(p, 0, n, next, reinterpret_cast<uint32_t(*)[kBlock / 32]>(sm + 2 * p.experts + 1));
  } else {
    for (int e = threadIdx.x; e < p.experts; e += kThreads) p.counts[(long long)(blockIdx.x) * p.experts + e] = count[e];
  }
}

__global__ void __launch_bounds__(kThreads) k_place(const Params p) {
  extern __shared__ int sm[];
  int* const all = sm;                                    // [experts] counts of all blocks
  int* const next = sm + p.experts;                       // [experts + 1]
  int* const mine = next + p.experts + 1;                 // [experts] counts of the blocks before this one
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int e = threadIdx.x; e < p.experts; e += kThreads) all[e] = mine[e] = 0;
  __syncthreads();
  const int blocks = gridDim.x;
  for (long long i = threadIdx.x; i < (long long)(blocks) * p.experts; i += kThreads) {
    const int b = int(i / p.experts), e = int(i - (long long)(b) * p.experts), c = p.counts[i];
    if (c) {
      atomicAdd(&all[e], c);
      if (b < int(blockIdx.x)) atomicAdd(&mine[e], c);
    }
  }
  __syncthreads();
  if (warp == 0) scan(all, next, p.experts, lane);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= p.experts; e += kThreads) p.offsets[e] = next[e];
  const int end = next[p.experts];
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += kThreads) next[e] += mine[e];
  fill_rest(p, end, blockIdx.x * kThreads + threadIdx.x, gridDim.x * kThreads);
  __syncthreads();
  const long long t0 = (long long)(blockIdx.x) * p.per_block;
  const int n = int(min((long long)(p.per_block), p.tokens - t0));
  for (int i = 0; i < n; i += kBlock)
    place(p, t0 + i, min(kBlock, n - i), next, reinterpret_cast<uint32_t(*)[kBlock / 32]>(mine + p.experts));
}

template <int PER> static void launch_choose(const Params& p, int blocks, cudaStream_t s) {
  if (blocks == 1) k_choose<PER, true><<<1, kThreads, (6 * p.experts + 1) * 4, s>>>(p);
  else k_choose<PER, false><<<blocks, kThreads, p.experts * 4, s>>>(p);
}

}  // namespace route

tardis_status_t launch_route(int tokens, int experts, int top_k, int normalise, const float* logits, long long ldl, int* chosen,
                             float* weights, int* offsets, int* rows, int* slots, int* work, cudaStream_t s) {
  using namespace route;
  int blocks = tokens > kBlock ? (tokens - 1) / kBlock + 1 : 1, per = kBlock;
  if (blocks > kMaxBlocks) {
    per = (tokens - 1) / kMaxBlocks + 1;
    blocks = (tokens - 1) / per + 1;
  }
  const Params p = {tokens, experts, top_k, normalise, per, logits, ldl, chosen, weights, offsets, rows, slots, work};
  if (experts <= 32) launch_choose<1>(p, blocks, s);
  else if (experts <= 64) launch_choose<2>(p, blocks, s);
  else if (experts <= 128) launch_choose<4>(p, blocks, s);
  else if (experts <= 256) launch_choose<8>(p, blocks, s);
  else launch_choose<32>(p, blocks, s);
  TARDIS_CUDA_TRY(cudaGetLastError());
  if (blocks > 1) {
    k_place<<<blocks, kThreads, (7 * experts + 1) * 4, s>>>(p);
    TARDIS_CUDA_TRY(cudaGetLastError());
  }
  return TARDIS_OK;
}

}  // namespace tardis
