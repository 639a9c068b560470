// Low-rank adapters of many requests beside a shared projection, forward and
// backward (see lipcache.h for the formulas).
#include "lc_common.hpp"
#include "lc_tile.hpp"

namespace lc {

constexpr int kAdMaxRank = 128;
constexpr int64_t kAdMaxWidth = 1 << 20;

// The pair of row t (-1: none): the last request whose first row is at or
// before t, if t is one of its rows.  Any offsets end the search in range.
__device__ __forceinline__ int pair_of_row(int64_t t, const int32_t* __restrict__ offsets,
                                           const int32_t* __restrict__ adapter, int R, int S) {
  int lo = 0, hi = R + 1;  // first index whose offset is past t
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= t) lo = mid + 1; else hi = mid;
  }
  if (lo < 1 || lo > R) return -1;
  const int a = adapter[lo - 1];
  return a >= 0 && a < S ? a : -1;
}

__global__ __launch_bounds__(256) void ad_pairs_kernel(int64_t T, const int32_t* __restrict__ offsets,
                                                       const int32_t* __restrict__ adapter, int R, int S,
                                                       int32_t* __restrict__ pair) {
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (t < T) pair[t] = R > 0 ? pair_of_row(t, offsets, adapter, R, S) : -1;
}

// v_t = A_a x_t (or u_t = B_a^T dy_t): one wave a row and rank.
template <typename T, bool kTransposed>
__global__ __launch_bounds__(256) void ad_shrink_kernel(int64_t rows, const T* __restrict__ x, int64_t ldx, int width,
                                                        const T* __restrict__ F, int r,
                                                        const int32_t* __restrict__ pair, float* __restrict__ out) {
  const int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / kWave;
  if (w >= rows * r) return;
  const int64_t t = w / r;
  const int rho = static_cast<int>(w % r);
  const int a = pair[t];
  float sum = 0.0f;
  if (a >= 0) {
    const T* f = F + static_cast<int64_t>(a) * r * width;
    for (int k = lane_id(); k < width; k += kWave)
      sum = fmaf(load_f32(x + t * ldx + k),
                 load_f32(f + (kTransposed ? static_cast<int64_t>(k) * r + rho : static_cast<int64_t>(rho) * width + k)),
                 sum);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  if (lane_id() == 0) out[w] = sum;
}

struct AdArgs {
  const void *x, *W, *dy;
  int64_t ldx, ldw, lddy, T;
  int K, N;
  lipcache_adapters ad;
};

template <typename T>
lipcache_status ad_forward(const AdArgs& g, const float* bias, void* y_, int64_t ldy, float* v, int32_t* pair,
                           hipStream_t s) {
  const T *x = static_cast<const T*>(g.x), *W = static_cast<const T*>(g.W), *A = static_cast<const T*>(g.ad.A),
          *B = static_cast<const T*>(g.ad.B);
  const float* scale = g.ad.scale;
  T* y = static_cast<T*>(y_);
  const int64_t ldx = g.ldx, ldw = g.ldw, N = g.N;
  const int r = g.ad.r;
  ad_pairs_kernel<<<static_cast<unsigned>((g.T + 255) / 256), 256, 0, s>>>(g.T, g.ad.offsets, g.ad.adapter, g.ad.R,
                                                                          g.ad.S, pair);
  LC_LAUNCHED();
  ad_shrink_kernel<T, false><<<static_cast<unsigned>((g.T * r + 3) / 4), 256, 0, s>>>(g.T, x, ldx, g.K, A, r, pair, v);
  LC_LAUNCHED();
  LC_HIP(tile_product(
      g.T, N, g.K, 1, [=] __device__(int, int64_t i, int64_t k) { return load_f32(x + i * ldx + k); },
      [=] __device__(int, int64_t j, int64_t k) { return load_f32(W + j * ldw + k); },
      [=] __device__(int, int64_t i, int64_t j, float sum) {
        const int a = pair[i];
        if (bias) sum += bias[j];
        if (a >= 0) {
          const T* b = B + (static_cast<int64_t>(a) * N + j) * r;
          float low = 0.0f;
          for (int rho = 0; rho < r; ++rho) low = fmaf(v[i * r + rho], load_f32(b + rho), low);
          sum = fmaf(scale[a], low, sum);
        }
        y[i * ldy + j] = round_to<T>(sum);
      },
      s));
  return LIPCACHE_OK;
}

template <typename T>
lipcache_status ad_backward(const AdArgs& g, const float* v_in, void* dx_, int64_t lddx, void* dA_, void* dB_,
                            int32_t* pair, float* u, float* v_ws, hipStream_t s) {
  const T *x = static_cast<const T*>(g.x), *W = static_cast<const T*>(g.W), *A = static_cast<const T*>(g.ad.A),
          *B = static_cast<const T*>(g.ad.B), *dy = static_cast<const T*>(g.dy);
  const float* scale = g.ad.scale;
  T *dx = static_cast<T*>(dx_), *dA = static_cast<T*>(dA_), *dB = static_cast<T*>(dB_);
  const int64_t ldx = g.ldx, ldw = g.ldw, lddy = g.lddy, N = g.N, K = g.K;
  const int r = g.ad.r, S = g.ad.S;
  if (g.T > 0) {
    ad_pairs_kernel<<<static_cast<unsigned>((g.T + 255) / 256), 256, 0, s>>>(g.T, g.ad.offsets, g.ad.adapter, g.ad.R, S,
                                                                            pair);
    LC_LAUNCHED();
    const unsigned waves = static_cast<unsigned>((g.T * r + 3) / 4);
    ad_shrink_kernel<T, true><<<waves, 256, 0, s>>>(g.T, dy, lddy, g.N, B, r, pair, u);
    LC_LAUNCHED();
    if (!v_in) {
      ad_shrink_kernel<T, false><<<waves, 256, 0, s>>>(g.T, x, ldx, g.K, A, r, pair, v_ws);
      LC_LAUNCHED();
      v_in = v_ws;
    }
  }
  if (dx)
    LC_HIP(tile_product(
        g.T, K, N, 1, [=] __device__(int, int64_t i, int64_t k) { return load_f32(dy + i * lddy + k); },
        [=] __device__(int, int64_t j, int64_t k) { return load_f32(W + k * ldw + j); },
        [=] __device__(int, int64_t i, int64_t j, float sum) {
          const int a = pair[i];
          if (a >= 0) {
            const T* f = A + static_cast<int64_t>(a) * r * K + j;
            float low = 0.0f;
            for (int rho = 0; rho < r; ++rho) low = fmaf(u[i * r + rho], load_f32(f + rho * K), low);
            sum = fmaf(scale[a], low, sum);
          }
          dx[i * lddx + j] = round_to<T>(sum);
        },
        s));
  if (dA && S > 0) {
    LC_HIP(tile_product(
        r, K, g.T, S, [=] __device__(int z, int64_t i, int64_t t) { return pair[t] == z ? u[t * r + i] : 0.0f; },
        [=] __device__(int z, int64_t j, int64_t t) { return pair[t] == z ? load_f32(x + t * ldx + j) : 0.0f; },
        [=] __device__(int z, int64_t i, int64_t j, float sum) {
          dA[(static_cast<int64_t>(z) * r + i) * K + j] = round_to<T>(scale[z] * sum);
        },
        s));
    LC_HIP(tile_product(
        N, r, g.T, S,
        [=] __device__(int z, int64_t i, int64_t t) { return pair[t] == z ? load_f32(dy + t * lddy + i) : 0.0f; },
        [=] __device__(int z, int64_t j, int64_t t) { return pair[t] == z ? v_in[t * r + j] : 0.0f; },
        [=] __device__(int z, int64_t i, int64_t j, float sum) {
          dB[(static_cast<int64_t>(z) * N + i) * r + j] = round_to<T>(scale[z] * sum);
        },
        s));
  }
  return LIPCACHE_OK;
}

// ------------------------------------------------------------- validation
bool ad_sizes_bad(int64_t T, int32_t K, int32_t N, int32_t dtype) {
  return T < 0 || K < 1 || N < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16;
}

bool ad_unaligned(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == LIPCACHE_F32 ? 3u : 1u)) != 0;
}

lipcache_status ad_check(const lipcache_adapters* ad, int64_t T, int32_t K, int32_t N, int32_t dtype) {
  if (!ad || ad_sizes_bad(T, K, N, dtype)) return LIPCACHE_EINVAL;
  if (ad->S < 0 || ad->R < 0 || ad->r < 1) return LIPCACHE_EINVAL;
  if (ad->S > 0 && (!ad->A || !ad->B || !ad->scale || ad_unaligned(ad->A, dtype) || ad_unaligned(ad->B, dtype) ||
                    ad_unaligned(ad->scale, LIPCACHE_F32)))
    return LIPCACHE_EINVAL;
  if (ad->R > 0 && (!ad->offsets || !ad->adapter || ad_unaligned(ad->offsets, LIPCACHE_F32) ||
                    ad_unaligned(ad->adapter, LIPCACHE_F32)))
    return LIPCACHE_EINVAL;
  if (ad->r > kAdMaxRank || K > kAdMaxWidth || N > kAdMaxWidth || T > 0x7fffffff || ad->S > 65535)
    return LIPCACHE_EUNSUPPORTED;
  return LIPCACHE_OK;
}

}  // namespace lc

using namespace lc;

extern "C" size_t lipcache_adapter_forward_workspace_bytes(int64_t T, int32_t K, int32_t N, int32_t r, int32_t S,
                                                           int32_t dtype) {
  if (ad_sizes_bad(T, K, N, dtype) || r < 1 || S < 0) return 0;
  return align_up(static_cast<size_t>(T) * 4, 256) + align_up(static_cast<size_t>(T) * r * 4, 256);
}

extern "C" lipcache_status lipcache_adapter_forward(const void* x, int64_t ldx, int64_t T, const void* W, int64_t ldw,
                                                    const float* bias, int32_t K, int32_t N,
                                                    const lipcache_adapters* ad, int32_t dtype, void* y, int64_t ldy,
                                                    float* v, void* ws, size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = ad_check(ad, T, K, N, dtype); st != LIPCACHE_OK) return st;
  if (ldx < K || ldw < K || ldy < N) return LIPCACHE_EINVAL;
  if (T > 0 && (!x || !W || !y)) return LIPCACHE_EINVAL;
  if (ad_unaligned(x, dtype) || ad_unaligned(W, dtype) || ad_unaligned(y, dtype) || ad_unaligned(bias, LIPCACHE_F32) ||
      ad_unaligned(v, LIPCACHE_F32))
    return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < lipcache_adapter_forward_workspace_bytes(T, K, N, ad->r, ad->S, dtype))
    return LIPCACHE_EWORKSPACE;
  if (T == 0) return LIPCACHE_OK;
  char* p = static_cast<char*>(ws);
  int32_t* pair = reinterpret_cast<int32_t*>(p);
  p += align_up(static_cast<size_t>(T) * 4, 256);
  if (!v) v = reinterpret_cast<float*>(p);
  AdArgs g{x, W, nullptr, ldx, ldw, 0, T, K, N, *ad};
  switch (dtype) {
    case LIPCACHE_F32: return ad_forward<float>(g, bias, y, ldy, v, pair, stream);
    case LIPCACHE_BF16: return ad_forward<__bf16>(g, bias, y, ldy, v, pair, stream);
    default: return ad_forward<_Float16>(g, bias, y, ldy, v, pair, stream);
  }
}

extern "C" size_t lipcache_adapter_backward_workspace_bytes(int64_t T, int32_t K, int32_t N, int32_t r, int32_t S,
                                                            int32_t dtype) {
  if (ad_sizes_bad(T, K, N, dtype) || r < 1 || S < 0) return 0;
  return align_up(static_cast<size_t>(T) * 4, 256) + 2 * align_up(static_cast<size_t>(T) * r * 4, 256);
}

extern "C" lipcache_status lipcache_adapter_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t T,
                                                     const void* W, int64_t ldw, int32_t K, int32_t N,
                                                     const lipcache_adapters* ad, int32_t dtype, const float* v,
                                                     void* dx, int64_t lddx, void* dA, void* dB, void* ws,
                                                     size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = ad_check(ad, T, K, N, dtype); st != LIPCACHE_OK) return st;
  if (lddy < N || ldx < K || ldw < K || (dx && lddx < K) || !dA != !dB) return LIPCACHE_EINVAL;
  if (T > 0 && (!dy || !x || !W)) return LIPCACHE_EINVAL;
  if (ad_unaligned(dy, dtype) || ad_unaligned(x, dtype) || ad_unaligned(W, dtype) || ad_unaligned(dx, dtype) ||
      ad_unaligned(dA, dtype) || ad_unaligned(dB, dtype) || ad_unaligned(v, LIPCACHE_F32))
    return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < lipcache_adapter_backward_workspace_bytes(T, K, N, ad->r, ad->S, dtype))
    return LIPCACHE_EWORKSPACE;
  char* p = static_cast<char*>(ws);
  int32_t* pair = reinterpret_cast<int32_t*>(p);
  p += align_up(static_cast<size_t>(T) * 4, 256);
  float* u = reinterpret_cast<float*>(p);
  float* v_ws = reinterpret_cast<float*>(p + align_up(static_cast<size_t>(T) * ad->r * 4, 256));
  AdArgs g{x, W, dy, ldx, ldw, lddy, T, K, N, *ad};
  switch (dtype) {
    case LIPCACHE_F32: return ad_backward<float>(g, v, dx, lddx, dA, dB, pair, u, v_ws, stream);
    case LIPCACHE_BF16: return ad_backward<__bf16>(g, v, dx, lddx, dA, dB, pair, u, v_ws, stream);
    default: return ad_backward<_Float16>(g, v, dx, lddx, dA, dB, pair, u, v_ws, stream);
  }
}
