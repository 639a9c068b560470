// Orthogonalisation by Newton-Schulz products and the momentum step around it
// (see lipcache.h for the formulas).
#include <math.h>

#include "lc_common.hpp"
#include "lc_tile.hpp"

namespace lc {

// ||U||_F of matrix z: float64 sums in a fixed order, one workgroup a matrix.
// With a momentum (kStep) U is formed first: M <- mu M + G, U = mu M + G or M.
template <typename T, bool kStep>
__global__ __launch_bounds__(256) void ns_norm_kernel(const T* __restrict__ G, float* __restrict__ M, int64_t size,
                                                      float mu, int nesterov, float* __restrict__ X,
                                                      double* __restrict__ norm2) {
  __shared__ double part[256 / kWave];
  const int64_t z = blockIdx.x;
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < size; i += 256) {
    float u = load_f32(G + z * size + i);
    if constexpr (kStep) {
      const float m = fmaf(mu, M[z * size + i], u);
      M[z * size + i] = m;
      u = nesterov ? fmaf(mu, m, u) : m;
    }
    X[z * size + i] = u;
    sum += static_cast<double>(u) * static_cast<double>(u);
  }
  sum = wave_sum(sum);
  if (lane_id() == 0) part[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) norm2[z] = ((part[0] + part[1]) + part[2]) + part[3];
}

// X_0 = U / (||U||_F + eps), transposed to p x q with p <= q.
__global__ __launch_bounds__(256) void ns_scale_kernel(const float* __restrict__ U, int m, int n,
                                                       const double* __restrict__ norm2, float eps,
                                                       float* __restrict__ X) {
  const int64_t size = static_cast<int64_t>(m) * n, z = blockIdx.y;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= size) return;
  const double f = sqrt(norm2[z]) + static_cast<double>(eps);
  const int64_t row = i / n, col = i % n;
  X[z * size + (m > n ? col * m + row : i)] = static_cast<float>(static_cast<double>(U[z * size + i]) / f);
}

// The result (transposed back), rounded; or the update of W.
template <typename T, bool kStep>
__global__ __launch_bounds__(256) void ns_out_kernel(const float* __restrict__ X, int m, int n, float keep, float gain,
                                                     T* __restrict__ out) {
  const int64_t size = static_cast<int64_t>(m) * n, z = blockIdx.y;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= size) return;
  const int64_t row = i / n, col = i % n;
  const float o = X[z * size + (m > n ? col * m + row : i)];
  T* p = out + z * size + i;
  *p = round_to<T>(kStep ? fmaf(keep, load_f32(p), -gain * o) : o);
}

struct NsArgs {
  int64_t batch;
  int m, n, steps;
  const float* coef;
  float eps;
};

size_t ns_workspace(int64_t batch, int32_t m, int32_t n) {
  const size_t p = m < n ? m : n, b = static_cast<size_t>(batch);
  return align_up(b * 8, 256) + 2 * align_up(b * m * n * 4, 256) + 2 * align_up(b * p * p * 4, 256);
}

template <typename T, bool kStep>
lipcache_status ns_run(const NsArgs& g, const void* G, float* M, float mu, int nesterov, float keep, float gain,
                       void* out, void* ws, hipStream_t s) {
  const int64_t p = g.m < g.n ? g.m : g.n, q = g.m < g.n ? g.n : g.m, size = p * q;
  const size_t b = static_cast<size_t>(g.batch);
  char* w = static_cast<char*>(ws);
  double* norm2 = reinterpret_cast<double*>(w);
  w += align_up(b * 8, 256);
  float* X = reinterpret_cast<float*>(w);
  w += align_up(b * size * 4, 256);
  float* Y = reinterpret_cast<float*>(w);
  w += align_up(b * size * 4, 256);
  float* P = reinterpret_cast<float*>(w);
  w += align_up(b * p * p * 4, 256);
  float* Q = reinterpret_cast<float*>(w);
  const unsigned nb = static_cast<unsigned>(g.batch);
  ns_norm_kernel<T, kStep><<<nb, 256, 0, s>>>(static_cast<const T*>(G), M, size, mu, nesterov, Y, norm2);
  LC_LAUNCHED();
  const dim3 grid(static_cast<unsigned>((size + 255) / 256), nb);
  ns_scale_kernel<<<grid, 256, 0, s>>>(Y, g.m, g.n, norm2, g.eps, X);
  LC_LAUNCHED();
  for (int k = 0; k < g.steps; ++k) {
    const float ca = g.coef[3 * k], cb = g.coef[3 * k + 1], cc = g.coef[3 * k + 2];
    LC_HIP(tile_product(
        p, p, q, static_cast<int>(nb), [=] __device__(int z, int64_t i, int64_t k_) { return X[z * size + i * q + k_]; },
        [=] __device__(int z, int64_t j, int64_t k_) { return X[z * size + j * q + k_]; },
        [=] __device__(int z, int64_t i, int64_t j, float sum) { P[(z * p + i) * p + j] = sum; }, s));
    LC_HIP(tile_product(
        p, p, p, static_cast<int>(nb), [=] __device__(int z, int64_t i, int64_t k_) { return P[(z * p + i) * p + k_]; },
        [=] __device__(int z, int64_t j, int64_t k_) { return P[(z * p + j) * p + k_]; },
        [=] __device__(int z, int64_t i, int64_t j, float sum) {
          Q[(z * p + i) * p + j] = fmaf(cc, sum, cb * P[(z * p + i) * p + j]);
        },
        s));
    LC_HIP(tile_product(
        p, q, p, static_cast<int>(nb), [=] __device__(int z, int64_t i, int64_t k_) { return Q[(z * p + i) * p + k_]; },
        [=] __device__(int z, int64_t j, int64_t k_) { return X[z * size + k_ * q + j]; },
        [=] __device__(int z, int64_t i, int64_t j, float sum) {
          Y[z * size + i * q + j] = fmaf(ca, X[z * size + i * q + j], sum);
        },
        s));
    float* t = X;
    X = Y;
    Y = t;
  }
  ns_out_kernel<T, kStep><<<grid, 256, 0, s>>>(X, g.m, g.n, keep, gain, static_cast<T*>(out));
  LC_LAUNCHED();
  return LIPCACHE_OK;
}

// The largest |s (a + b s^2 + c s^4)| over 0 <= s <= h, in float64: at h or
// where the derivative a + 3 b s^2 + 5 c s^4 vanishes.
double ns_bound(double a, double b, double c, double h) {
  auto f = [&](double s2) { return fabs(sqrt(s2) * (a + s2 * (b + s2 * c))); };
  double top = f(h * h);
  auto at = [&](double s2) {
    if (s2 > 0.0 && s2 < h * h) top = fmax(top, f(s2));
  };
  if (c != 0.0) {
    const double disc = 9.0 * b * b - 20.0 * a * c;
    if (disc >= 0.0) {
      at((-3.0 * b + sqrt(disc)) / (10.0 * c));
      at((-3.0 * b - sqrt(disc)) / (10.0 * c));
    }
  } else if (b != 0.0) {
    at(-a / (3.0 * b));
  }
  return top;
}

constexpr double kNsMost = 16.0;  // largest singular value that any step may allow

lipcache_status ns_check(int64_t batch, int32_t m, int32_t n, int32_t dtype, int32_t steps, const float* coef,
                         float eps) {
  if (batch < 0 || m < 1 || n < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16 || steps < 0 || steps > 32 ||
      !(eps >= 0.0f) || isinf(eps) || (steps > 0 && !coef))
    return LIPCACHE_EINVAL;
  for (int i = 0; i < 3 * steps; ++i)
    if (!isfinite(coef[i])) return LIPCACHE_EINVAL;
  const int32_t p = m < n ? m : n;
  if (batch > 65535 || p > 16384 || static_cast<int64_t>(m) * n > (1ll << 30)) return LIPCACHE_EUNSUPPORTED;
  double h = 1.0;
  for (int k = 0; k < steps; ++k) {
    h = ns_bound(coef[3 * k], coef[3 * k + 1], coef[3 * k + 2], h);
    if (!(h < kNsMost)) return LIPCACHE_EUNSUPPORTED;
  }
  return LIPCACHE_OK;
}

bool ns_unaligned(const void* p, int32_t dtype) {
  return !p || (reinterpret_cast<uintptr_t>(p) & (dtype == LIPCACHE_F32 ? 3u : 1u)) != 0;
}

template <bool kStep>
lipcache_status ns_dispatch(const NsArgs& g, int32_t dtype, const void* G, float* M, float mu, int nesterov, float keep,
                            float gain, void* out, void* ws, hipStream_t s) {
  switch (dtype) {
    case LIPCACHE_F32: return ns_run<float, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    case LIPCACHE_BF16: return ns_run<__bf16, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    default: return ns_run<_Float16, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
  }
}

}  // namespace lc

using namespace lc;

extern "C" size_t lipcache_orthogonalise_workspace_bytes(int64_t batch, int32_t m, int32_t n, int32_t dtype) {
  if (batch < 0 || m < 1 || n < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16) return 0;
  return ns_workspace(batch, m, n);
}

extern "C" lipcache_status lipcache_orthogonalise(const void* G, int64_t batch, int32_t m, int32_t n, int32_t dtype,
                                                  int32_t steps, const float* coef, float eps, void* out, void* ws,
                                                  size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = ns_check(batch, m, n, dtype, steps, coef, eps); st != LIPCACHE_OK) return st;
  if (batch > 0 && (ns_unaligned(G, dtype) || ns_unaligned(out, dtype))) return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < ns_workspace(batch, m, n)) return LIPCACHE_EWORKSPACE;
  if (batch == 0) return LIPCACHE_OK;
  const NsArgs g{batch, m, n, steps, coef, eps};
  return ns_dispatch<false>(g, dtype, G, nullptr, 0.0f, 0, 0.0f, 0.0f, out, ws, stream);
}

extern "C" size_t lipcache_muon_step_workspace_bytes(int64_t batch, int32_t m, int32_t n, int32_t dtype) {
  return lipcache_orthogonalise_workspace_bytes(batch, m, n, dtype);
}

extern "C" lipcache_status lipcache_muon_step(void* W, const void* G, float* M, int64_t batch, int32_t m, int32_t n,
                                              int32_t dtype, const lipcache_muon* opt, void* ws, size_t ws_bytes,
                                              lipcache_stream_t stream) {
  if (!opt) return LIPCACHE_EINVAL;
  if (lipcache_status st = ns_check(batch, m, n, dtype, opt->steps, opt->coef, opt->eps); st != LIPCACHE_OK) return st;
  if (!isfinite(opt->lr) || !isfinite(opt->momentum) || !isfinite(opt->weight_decay) || !isfinite(opt->scale))
    return LIPCACHE_EINVAL;
  if (batch > 0 && (ns_unaligned(W, dtype) || ns_unaligned(G, dtype) || ns_unaligned(M, LIPCACHE_F32)))
    return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < ns_workspace(batch, m, n)) return LIPCACHE_EWORKSPACE;
  if (batch == 0) return LIPCACHE_OK;
  const NsArgs g{batch, m, n, opt->steps, opt->coef, opt->eps};
  const float keep = static_cast<float>(1.0 - static_cast<double>(opt->lr) * opt->weight_decay);
  const float gain = static_cast<float>(static_cast<double>(opt->lr) * opt->scale);
  return ns_dispatch<true>(g, dtype, G, M, opt->momentum, opt->nesterov != 0, keep, gain, W, ws, stream);
}
