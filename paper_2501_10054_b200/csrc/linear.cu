// The dense products of unfolded feed-forward blocks: dispatch, the kernel for every type and size, the weighted return to the tokens.
#include "linear.cuh"

namespace tardis {
namespace linear {

// 256 threads compute a tile of TO outputs x TN rows, T x T of them each (TO = TN = 16 T), over steps of 32 channels staged in shared memory.
template <typename E, int T>
__global__ void __launch_bounds__(256) k_linear_any(const LinearArgs a) {
  constexpr int TILE = 16 * T, BK = 32, LD = TILE + 4;
  __shared__ float sw[BK][LD], sx[BK][LD];
  const GroupTile t = find_group_tile(a.offsets, a.groups, a.n, TILE, blockIdx.y);
  if (t.rows == 0) return;
  const int o0 = blockIdx.x * TILE, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;      // tx: outputs, ty: rows
  const E* const W = static_cast<const E*>(a.W) + t.e * a.stride_w;
  const E* const x = static_cast<const E*>(a.x);
  float acc[T][T] = {};
  for (int k0 = 0; k0 < a.k; k0 += BK) {
    for (int i = threadIdx.x; i < TILE * BK; i += 256) {
      const int kk = i % BK, r = i / BK, k = k0 + kk;
      float w = 0.f, v = 0.f;
      if (k < a.k) {
        if (o0 + r < a.o) w = to_f32(W[(o0 + r) * a.ldw + k]);
        if (r < t.rows) {
          const int src = a.rows ? a.rows[t.first + r] : t.first + r;
          if (src >= 0 && src < a.nx) v = to_f32(x[src * a.ldx + k]);
        }
      }
      sw[kk][r] = w;
      sx[kk][r] = v;
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < BK; ++kk) {
      float w[T], v[T];
#pragma unroll
      for (int i = 0; i < T; ++i) { w[i] = sw[kk][tx + 16 * i]; v[i] = sx[kk][ty + 16 * i]; }
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j) acc[i][j] = fmaf(v[i], w[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < T; ++i) {
    const int r = ty + 16 * i;
    if (r >= t.rows) continue;
    const long long row = t.first + r;
#pragma unroll
    for (int j = 0; j < T; ++j) {
      const int o = o0 + tx + 16 * j;
      if (o >= a.o) continue;
      float z = acc[i][j];
      if (a.bias) z += a.bias[(long long)(t.e) * a.o + o];
      z = apply_act(z, a.act);
      if (a.res) z += load_out(a.res, row * a.ldr + o, a.out_dtype);
      store_out(a.y, row * a.ldy + o, a.out_dtype, z);
    }
  }
}

template <typename E, int T>
static tardis_status_t launch_any(const LinearArgs& a, cudaStream_t s) {
  const int tile = 16 * T;
  const long long tiles = (a.n + tile - 1) / tile + (a.offsets ? (a.groups < a.n ? a.groups : a.n) : 0);     // at most
  if (tiles > 65535) return TARDIS_ERR_UNSUPPORTED;
  k_linear_any<E, T><<<dim3(unsigned((a.o + tile - 1) / tile), unsigned(tiles)), 256, 0, s>>>(a);
  TARDIS_CUDA_TRY(cudaGetLastError());
  return TARDIS_OK;
}

// A thread adds up one output of a token after the other, in the order of the token's choices.
__global__ void __launch_bounds__(256) k_combine(const LinearArgs a, int top_k, const float* __restrict__ f, const int* __restrict__ slots,
                                                 const float* __restrict__ weights) {
  const long long t = blockIdx.x;
  const int lo = max(a.offsets[0], 0), hi = min(a.offsets[a.groups], a.n);
  for (int c = blockIdx.y * 256 + threadIdx.x; c < a.o; c += gridDim.y * 256) {
    float sum = 0.f;
    for (int j = 0; j < top_k; ++j) {
      const int slot = slots[t * top_k + j];
      if (slot >= lo && slot < hi) sum = fmaf(weights[t * top_k + j], f[(long long)(slot) * a.o + c], sum);
    }
    if (a.res) sum += load_out(a.res, t * a.ldr + c, a.out_dtype);
    store_out(a.y, t * a.ldy + c, a.out_dtype, sum);
  }
}

}  // namespace linear

tardis_status_t launch_combine(int tokens, int top_k, const LinearArgs& a, const float* f, const int* slots, const float* weights,
                               cudaStream_t s) {
  linear::k_combine<<<dim3(unsigned(tokens), unsigned(a.o > 8192 ? 8 : (a.o + 1023) / 1024)), 256, 0, s>>>(a, top_k, f, slots, weights);
  TARDIS_CUDA_TRY(cudaGetLastError());
  return TARDIS_OK;
}

tardis_status_t launch_linear(const LinearArgs& a, cudaStream_t s) {
  using namespace linear;
  return a.dtype == TARDIS_BF16 ? launch_linear_tc(a, s) : launch_any<float, 4>(a, s);
}

}  // namespace tardis
