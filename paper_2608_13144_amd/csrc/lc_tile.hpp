// A plain tiled product in float32 for operands behind functors.
#pragma once

#include "lc_common.hpp"

namespace lc {

// One element of a float32, bfloat16 or float16 array as float32, and back
// (rounded to nearest even).
template <typename T>
__device__ __forceinline__ float load_f32(const T* p) { return static_cast<float>(*p); }
template <typename T>
__device__ __forceinline__ T round_to(float v) { return static_cast<T>(v); }

// C(i, j) = sum_k a(z, i, k) b(z, j, k) for i < M, j < N, one 64 x 64 tile a
// workgroup (blockIdx.z = z), 4 x 4 outputs a thread, float32 throughout.
// The functors answer 0 outside their ranges; `ep(z, i, j, sum)` stores.
template <class LA, class LB, class EP>
__global__ __launch_bounds__(256) void tile_product_kernel(int64_t M, int64_t N, int64_t K, LA a, LB b, EP ep) {
  __shared__ float sa[16][65], sb[16][65];
  const int tid = static_cast<int>(threadIdx.x);
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * 64, j0 = static_cast<int64_t>(blockIdx.y) * 64;
  const int z = static_cast<int>(blockIdx.z);
  const int ti = tid / 16, tj = tid % 16;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < K; k0 += 16) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = (tid >> 4) + 16 * e, k = tid & 15;
      const bool in = k0 + k < K;
      sa[k][row] = in && i0 + row < M ? a(z, i0 + row, k0 + k) : 0.0f;
      sb[k][row] = in && j0 + row < N ? b(z, j0 + row, k0 + k) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float av[4], bv[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        av[e] = sa[k][ti + 16 * e];
        bv[e] = sb[k][tj + 16 * e];
      }
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(av[p], bv[q], acc[p][q]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int p = 0; p < 4; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t i = i0 + ti + 16 * p, j = j0 + tj + 16 * q;
      if (i < M && j < N) ep(z, i, j, acc[p][q]);
    }
}

template <class LA, class LB, class EP>
inline hipError_t tile_product(int64_t M, int64_t N, int64_t K, int batch, LA a, LB b, EP ep, hipStream_t s) {
  if (M <= 0 || N <= 0 || batch <= 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>((M + 63) / 64), static_cast<unsigned>((N + 63) / 64),
                  static_cast<unsigned>(batch));
  tile_product_kernel<<<grid, 256, 0, s>>>(M, N, K, a, b, ep);
  return hipGetLastError();
}

}  // namespace lc
