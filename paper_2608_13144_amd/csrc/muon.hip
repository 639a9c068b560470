// Orthogonalisation by Newton-Schulz products and the momentum step around it
// (see lipcache.h for the formulas).
#include <math.h>

#include "lc_common.hpp"
#include "lc_mfma.hpp"

namespace lc {

// X, P = X X^T (or X^T X) and B = b P + c P^2 go to the matrix cores as sums of
// two float16 numbers (22 bits), each times a power of two that keeps the
// largest possible entry below 2^15; the sums of the products are float32.
//
// A step may ask for single float16 numbers (LIPCACHE_MUON_SHORT_OPERANDS).  X's
// rounding is then kept in a second array and comes in with the term a X.  Small singular values grow by a = 3.4 a step
// through that term alone, and what is lost of X there is lost of them: 2e-2
// of the result for a matrix of a few strong directions over noise, 5e-4 with
// the second array.
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ float ns_load(const T* p) { return static_cast<float>(*p); }
template <typename T>
__device__ __forceinline__ T ns_round(float v) { return static_cast<T>(v); }  // to nearest even

// U of element i: G itself, or the momentum's direction (M already updated
// when kUpdate is false).
template <typename T, bool kStep, bool kUpdate>
__device__ __forceinline__ float ns_direction(const T* __restrict__ G, float* __restrict__ M, int64_t i, float mu,
                                              int nesterov) {
  float u = ns_load(G + i);
  if constexpr (kStep) {
    float m = M[i];
    if constexpr (kUpdate) {
      m = fmaf(mu, m, u);
      M[i] = m;
    }
    u = nesterov ? fmaf(mu, m, u) : m;
  }
  return u;
}

// Eight directions from element i on; whole vectors where `wide` (i and the arrays are aligned for them), else up to
// `count` of them one by one (the rest 0).
template <typename T, bool kStep, bool kUpdate>
__device__ __forceinline__ void ns_direction8(const T* __restrict__ G, float* __restrict__ M, int64_t i, int count,
                                              bool wide, float mu, int nesterov, float (&u)[8]) {
  if (wide) {
    typedef T vec __attribute__((ext_vector_type(8)));
    const vec g = *reinterpret_cast<const vec*>(G + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = static_cast<float>(g[e]);
    if constexpr (kStep) {
      f32x4 m[2] = {reinterpret_cast<const f32x4*>(M + i)[0], reinterpret_cast<const f32x4*>(M + i)[1]};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = m[e / 4][e % 4];
        if constexpr (kUpdate) v = fmaf(mu, v, u[e]);
        m[e / 4][e % 4] = v;
        u[e] = nesterov ? fmaf(mu, v, u[e]) : v;
      }
      if constexpr (kUpdate) {
        reinterpret_cast<f32x4*>(M + i)[0] = m[0];
        reinterpret_cast<f32x4*>(M + i)[1] = m[1];
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = e < count ? ns_direction<T, kStep, kUpdate>(G, M, i + e, mu, nesterov) : 0.0f;
  }
}

// Workgroups that sum one matrix's norm: 4096 elements each (two vectors a thread) up to 1024 of them.
__host__ __device__ inline int ns_chunks(int64_t size) {
  const int64_t c = (size + 4095) / 4096;
  return c < 1024 ? static_cast<int>(c) : 1024;
}

// Partial sums of U^2 in float64, in a fixed order; updates the momentum.
template <typename T, bool kStep>
__global__ __launch_bounds__(256) void ns_norm_kernel(const T* __restrict__ G, float* __restrict__ M, int64_t size,
                                                      float mu, int nesterov, int wide, double* __restrict__ part) {
  __shared__ double wave_part[256 / kWave];
  const int64_t z = blockIdx.y;
  double sum = 0.0;
#pragma unroll 2
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < size;
       i += 2048 * static_cast<int64_t>(gridDim.x)) {
    float u[8];
    ns_direction8<T, kStep, true>(G, M, z * size + i, size - i < 8 ? static_cast<int>(size - i) : 8, wide != 0, mu, nesterov, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += static_cast<double>(u[e]) * static_cast<double>(u[e]);
  }
  sum = wave_sum(sum);
  if (lane_id() == 0) wave_part[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0)
    part[z * gridDim.x + blockIdx.x] = ((wave_part[0] + wave_part[1]) + wave_part[2]) + wave_part[3];
}

// 1 / (||U||_F + eps) from the partial sums; every thread of the workgroup gets it.
__device__ __forceinline__ double ns_inverse(const double* __restrict__ part, int chunks, float eps, double* lds) {
  if (threadIdx.x < kWave) {
    double sum = 0.0;
    for (int c = threadIdx.x; c < chunks; c += kWave) sum += part[c];
    sum = wave_sum(sum);
    if (threadIdx.x == 0) *lds = sum;
  }
  __syncthreads();
  const double f = sqrt(*lds) + static_cast<double>(eps);
  return f > 0.0 || f != f ? 1.0 / f : 0.0;
}

// Element (i, j) of a matrix of _Float16 or Split numbers with `width` columns.
template <class E>
struct NsAt;
template <>
struct NsAt<_Float16> {
  static constexpr int kPad = 8;  // widths and heights are multiples of this
  static constexpr bool kLow = true;  // X's rounding is kept apart, for the term a X
  static __device__ __forceinline__ int64_t at(int64_t i, int j, int width) { return i * width + j; }
  static __device__ __forceinline__ float get(const _Float16* p) { return static_cast<float>(*p); }
  static __device__ __forceinline__ void put(_Float16* p, float v) { *p = static_cast<_Float16>(v); }
  static __device__ __forceinline__ void put4(_Float16* p, f32x4 v) {
    f16x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = static_cast<_Float16>(v[e]);
    *reinterpret_cast<f16x4*>(p) = h;
  }
};
template <>
struct NsAt<Split> {
  static constexpr int kPad = 32;
  static constexpr bool kLow = false;
  static __device__ __forceinline__ int64_t at(int64_t i, int j, int width) {
    return i * (2 * width) + (j & ~31) * 2 + (j & 31);
  }
  static __device__ __forceinline__ float get(const _Float16* p) {
    return static_cast<float>(p[0]) + static_cast<float>(p[32]);
  }
  static __device__ __forceinline__ void put(_Float16* p, float v) {
    split_f16(v, p[0], p[32]);
  }
  static __device__ __forceinline__ void put4(_Float16* p, f32x4 v) {
    f16x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 first, second;
      split_f16(v[e], first, second);
      h[e] = first;
      l[e] = second;
    }
    *reinterpret_cast<f16x4*>(p) = h;
    *reinterpret_cast<f16x4*>(p + 32) = l;
  }
};

// X_0 = U / (||U||_F + eps) on m8 x n8 (zero past m x n), scaled; eight columns a thread.
template <class E, typename T, bool kStep>
__global__ __launch_bounds__(256) void ns_start_kernel(const T* __restrict__ G, float* __restrict__ M, int m, int n,
                                                       int m8, int n8, float mu, int nesterov, int wide,
                                                       const double* __restrict__ part, int chunks, float eps,
                                                       float scale, _Float16* __restrict__ X,
                                                       _Float16* __restrict__ Xlow) {
  __shared__ double lds;
  const int64_t z = blockIdx.y, size = static_cast<int64_t>(m) * n, groups = static_cast<int64_t>(m8) * n8 / 8;
  // as mantissa and exponent: the factor itself may pass float32's range where U is tiny (or huge) and eps 0
  int up;
  const float f = static_cast<float>(frexp(ns_inverse(part + z * chunks, chunks, eps, &lds) * scale, &up));
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < groups; i += 256 * static_cast<int64_t>(gridDim.x)) {
    const int row = static_cast<int>(i / (n8 / 8)), col = static_cast<int>(i % (n8 / 8)) * 8;
    float u[8] = {};
    if (row < m && col < n)
      ns_direction8<T, kStep, false>(G, M, z * size + static_cast<int64_t>(row) * n + col, n - col, wide != 0, mu, nesterov, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = f * ldexpf(u[e], up);
    const f32x4 lo = {u[0], u[1], u[2], u[3]}, hi = {u[4], u[5], u[6], u[7]};
    const int64_t at = NsAt<E>::at(z * m8 + row, col, n8);
    if constexpr (NsAt<E>::kLow) {
      f16x8 first, second;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        _Float16 p, r;
        split_f16(u[e], p, r);
        first[e] = p;
        second[e] = r;
      }
      *reinterpret_cast<f16x8*>(X + at) = first;
      *reinterpret_cast<f16x8*>(Xlow + at) = second;
    } else {
      NsAt<E>::put4(X + at, lo);
      NsAt<E>::put4(X + at + 4, hi);
    }
  }
}

// No steps at all: the normalised matrix itself.
template <typename T, bool kStep>
__global__ __launch_bounds__(256) void ns_plain_kernel(const T* G, float* __restrict__ M, int64_t size, float mu,
                                                       int nesterov, const double* __restrict__ part, int chunks,
                                                       float eps, float keep, float gain, T* out) {
  __shared__ double lds;
  const int64_t z = blockIdx.y;
  const double f = ns_inverse(part + z * chunks, chunks, eps, &lds);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < size; i += 256 * static_cast<int64_t>(gridDim.x)) {
    const float o = static_cast<float>(f * ns_direction<T, kStep, false>(G, M, z * size + i, mu, nesterov));
    T* p = out + z * size + i;
    *p = ns_round<T>(kStep ? fmaf(keep, ns_load(p), -gain * o) : o);
  }
}

// A symmetric product: out = f_sum F F^T + f_in in  (F p8 x k8 "row", or k8 x p8 "col" with rows of `width`), the
// lower tiles computed and mirrored.  4096 wide: 215 us (0.96 PFLOP/s: three products of the triangle), 11 bits 80 us
// (0.86); 200 wide: 5.9 us, most of it the launch and one round of loads.
template <class S>
__global__ __launch_bounds__(S::kThreads) void ns_square_kernel(const _Float16* __restrict__ F, int p8, int k8,
                                                                int width, const _Float16* __restrict__ in,
                                                                float f_sum, float f_in, _Float16* __restrict__ out) {
  typedef NsAt<typename S::E> At;
  __shared__ __align__(16) char lds[S::kLds];
  const int rows = (p8 + S::BM - 1) / S::BM, tiles = rows * (rows + 1) / 2;
  const int all = xcd_order(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
  const int64_t z = all / tiles;
  const int t = all % tiles;
  int bi = static_cast<int>((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
  while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
  while (bi * (bi + 1) / 2 > t) --bi;
  const int bj = t - bi * (bi + 1) / 2;
  const int i0 = bi * S::BM, j0 = bj * S::BN;
  Side P{}, Q{};
  P.p = F + (S::PCOL ? At::at(z * k8, i0, width) : At::at(z * p8 + i0, 0, width));
  Q.p = F + (S::QCOL ? At::at(z * k8, j0, width) : At::at(z * p8 + j0, 0, width));
  P.ld = Q.ld = static_cast<int64_t>(width) * sizeof(typename S::E);
  P.rows = p8 - i0 < S::BM ? p8 - i0 : S::BM;
  Q.rows = p8 - j0 < S::BN ? p8 - j0 : S::BN;
  f32x16 acc[S::TM][S::TN] = {};
  tile_products<S>(P, Q, k8, lds, acc);
  tile_store<S>(acc, [&](int i, int j, const f32x16& v) {
    i += i0;
    j += j0;
    if (j >= p8) return;
    float add[16];
    if (in) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = i + acc_row(e) < p8 ? i + acc_row(e) : p8 - 1;
        add[e] = At::get(in + At::at(z * p8 + row, j, p8));
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (i + 8 * q >= p8) break;  // p8 is a multiple of 8, so four rows stand or fall together
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e] = f_sum * v[4 * q + e];
        if (in) o[e] = fmaf(f_in, add[4 * q + e], o[e]);
        At::put(out + At::at(z * p8 + i + 8 * q + e, j, p8), o[e]);
      }
      if (bi != bj) At::put4(out + At::at(z * p8 + j, i + 8 * q, p8), o);
    }
  });
}

// Where the result of the last step goes: [m][n], rounded, or subtracted from W.
template <typename T>
struct NsOut {
  T* out;
  int m, n;
  float keep, gain;
};

// X' = a X + B X (wide: P = B, Q = X "col") or a X + X B (tall: P = X, Q = B).  4096 x 4096: 362 us (1.14
// PFLOP/s: three products), 11 bits 147 us (0.94); three of 1000 x 777: 22 us.
template <class S, bool kWide, bool kLast, typename T, bool kStep>
__global__ __launch_bounds__(S::kThreads) void ns_apply_kernel(const _Float16* __restrict__ X,
                                                               const _Float16* __restrict__ B, int m8, int n8,
                                                               float f_sum, float f_x,
                                                               const _Float16* __restrict__ Xlow,
                                                               _Float16* __restrict__ Y, _Float16* __restrict__ Ylow,
                                                               NsOut<T> o) {
  typedef NsAt<typename S::E> At;
  __shared__ __align__(16) char lds[S::kLds];
  const int p8 = kWide ? m8 : n8;
  int bi, bj;
  const int64_t z = tile_of((m8 + S::BM - 1) / S::BM, (n8 + S::BN - 1) / S::BN, bi, bj);
  const int i0 = bi * S::BM, j0 = bj * S::BN;
  Side P{}, Q{};
  if constexpr (kWide) {
    P.p = B + At::at(z * p8 + i0, 0, p8);
    Q.p = X + At::at(z * m8, j0, n8);
  } else {
    P.p = X + At::at(z * m8 + i0, 0, n8);
    Q.p = B + At::at(z * p8 + j0, 0, p8);
  }
  P.ld = static_cast<int64_t>(kWide ? p8 : n8) * sizeof(typename S::E);
  Q.ld = static_cast<int64_t>(kWide ? n8 : p8) * sizeof(typename S::E);
  P.rows = m8 - i0 < S::BM ? m8 - i0 : S::BM;
  Q.rows = n8 - j0 < S::BN ? n8 - j0 : S::BN;
  f32x16 acc[S::TM][S::TN] = {};
  tile_products<S>(P, Q, p8, lds, acc);
  tile_store<S>(acc, [&](int i, int j, const f32x16& v) {
    i += i0;
    j += j0;
    if (j >= n8) return;
    float x[16], w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int row = i + acc_row(e) < m8 ? i + acc_row(e) : m8 - 1;
      x[e] = At::get(X + At::at(z * m8 + row, j, n8));
      if constexpr (At::kLow) x[e] += static_cast<float>(Xlow[At::at(z * m8 + row, j, n8)]);
      if constexpr (kLast && kStep)
        w[e] = ns_load(o.out + (z * o.m + (row < o.m ? row : o.m - 1)) * o.n + (j < o.n ? j : o.n - 1));
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int row = i + acc_row(e);
      const float y = fmaf(f_x, x[e], f_sum * v[e]);
      if constexpr (kLast) {
        if (row < o.m && j < o.n)
          o.out[(z * o.m + row) * o.n + j] = ns_round<T>(kStep ? fmaf(o.keep, w[e], -o.gain * y) : y);
      } else if (row < m8) {
        const int64_t at = At::at(z * m8 + row, j, n8);
        if constexpr (At::kLow) split_f16(y, Y[at], Ylow[at]);
        else At::put(Y + at, y);
      }
    }
  });
}

// ------------------------------------------------------------ short matrices
// With the shorter side p <= 64 the iteration runs on the p x p Gram matrix:
// X_k = P_k X_0 with P_k a polynomial of A_0 = X_0 X_0^T, so the long side is
// read twice and written once, whatever the number of steps:
//   A <- Q A Q, P <- Q P with Q = a I + b A + c A^2   (all commute, all symmetric).
// A_0 squares the singular values, so everything here is float64: small ones
// relative to the largest keep the digits that float32 products of X would
// give them.  Three launches: the Gram matrix in shares of the long side (and
// the momentum), the polynomial (one workgroup a matrix, in LDS), the product
// P U.
//
// Rounding leaves A eigenvalues of about -2^-53, which no X X^T has, and a step
// multiplies them by up to g^2, g the largest |a + b s + c s^2| on the spectrum;
// near -1 they would explode.  So before A's errors have grown by 2^24 (7 steps
// of the usual coefficients) a round ends: X = P U is formed in float64, and the
// next round starts from its Gram matrix, whose eigenvalues are squares again.
//
// Bound by reading and writing the long matrices, and by the chain of
// small products between: 64 of 16 x 4096 (bf16, with the momentum) 11 + 8 + 12 us
// for 84 MB; without it 26 us, 7 steps 27, 8 steps (two rounds) 56.
constexpr int kShortMost = 64;
constexpr int kShortBlock = 256;  // of the long side, in LDS at a time

typedef double f64x4 __attribute__((ext_vector_type(4)));

// A block of U in LDS as float32: element (k, c) of the short and the long index at k * sk + c * sc.
template <typename T, bool kStep>
struct ShortU {
  const T* G;
  float* M;
  int m, n;
  float mu;
  int nesterov;
  int wide;  // vectors of eight

  __device__ __forceinline__ int p() const { return m < n ? m : n; }
  __device__ __forceinline__ int q() const { return m < n ? n : m; }
  // wide matrices (m <= n) lie [k][c], tall ones [c][k] (odd strides keep the banks apart)
  __device__ __forceinline__ int sk() const { return m <= n ? kShortBlock + 4 : 1; }
  __device__ __forceinline__ int sc() const { return m <= n ? 1 : (n | 1); }
  static int room(int p, bool wide) { return wide ? p * (kShortBlock + 4) : kShortBlock * (p | 1); }

  // f(element index in the matrix, k, c, count) for groups of up to eight neighbours along a row
  template <class F>
  __device__ __forceinline__ void each(int c0, int count, F f) const {
    if (m <= n) {
      const int groups = (count + 7) / 8;
      for (int i = threadIdx.x; i < groups * m; i += 256) {
        const int k = i / groups, c = i % groups * 8;
        f(static_cast<int64_t>(k) * n + c0 + c, k, c, count - c < 8 ? count - c : 8);
      }
    } else {
      const int groups = (n + 7) / 8;
      for (int i = threadIdx.x; i < groups * count; i += 256) {
        const int c = i / groups, k = i % groups * 8;
        f(static_cast<int64_t>(c0 + c) * n + k, k, c, n - k < 8 ? n - k : 8);
      }
    }
  }

  template <bool kUpdate>
  __device__ __forceinline__ void load(int64_t z, int c0, int count, float* lds) const {
    const int64_t base = z * m * static_cast<int64_t>(n);
    const int ek = m <= n ? 0 : sk(), ec = m <= n ? sc() : 0;  // along a row
    each(c0, count, [&](int64_t at, int k, int c, int some) {
      float u[8];
      ns_direction8<T, kStep, kUpdate>(G, M, base + at, some, wide != 0, mu, nesterov, u);
      float* to = lds + k * sk() + c * sc();
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < some) to[e * (ek + ec)] = u[e];
    });
  }
};

// The tiles of a Gram matrix: the four waves' sums, added in order.
template <int N>
__device__ __forceinline__ void short_gram_store(const f64x4 (&acc)[N * (N + 1) / 2], double (&join)[4][256], double* out) {
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
#pragma unroll
  for (int t = 0; t < N * (N + 1) / 2; ++t) {
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 4; ++v) join[wave][v * 64 + lane] = acc[t][v];
    __syncthreads();
    const int i = static_cast<int>(threadIdx.x);
    out[t * 256 + i] = ((join[0][i] + join[1][i]) + join[2][i]) + join[3][i];
  }
}

// part[z][share] = sum over the share's c of U(:, c) U(:, c)^T, N x N tiles of 16 (the lower ones; zeros past p).
template <int N, typename T, bool kStep>
__global__ __launch_bounds__(256) void ns_short_gram_kernel(ShortU<T, kStep> U, int shares, double* __restrict__ part) {
  constexpr int kTiles = N * (N + 1) / 2;
  extern __shared__ __align__(16) float lds[];
  __shared__ double join[4][256];
  const int64_t z = blockIdx.y;
  const int p = U.p(), q = U.q(), sk = U.sk(), sc = U.sc();
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int row = lane & 15, quarter = lane >> 4;
  f64x4 acc[kTiles] = {};
  for (int c0 = static_cast<int>(blockIdx.x) * kShortBlock; c0 < q; c0 += shares * kShortBlock) {
    const int count = q - c0 < kShortBlock ? q - c0 : kShortBlock;
    __syncthreads();
    U.template load<true>(z, c0, count, lds);
    __syncthreads();
    for (int c = wave * 4; c < count; c += 16) {
      double f[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        f[i] = 16 * i + row < p && c + quarter < count ? static_cast<double>(lds[(16 * i + row) * sk + (c + quarter) * sc]) : 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j <= i; ++j)
          acc[i * (i + 1) / 2 + j] = __builtin_amdgcn_mfma_f64_16x16x4f64(f[i], f[j], acc[i * (i + 1) / 2 + j], 0, 0, 0);
    }
  }
  short_gram_store<N>(acc, join, part + (z * shares + blockIdx.x) * (kTiles * 256));
}

// The same for a round's X [z][q][p].
template <int N>
__global__ __launch_bounds__(256) void ns_short_regram_kernel(const double* __restrict__ X, int p, int q, int shares,
                                                              double* __restrict__ part) {
  constexpr int kTiles = N * (N + 1) / 2;
  __shared__ double join[4][256];
  const int64_t z = blockIdx.y;
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int row = lane & 15, quarter = lane >> 4;
  const double* x = X + z * q * p;
  f64x4 acc[kTiles] = {};
  for (int c0 = static_cast<int>(blockIdx.x) * kShortBlock; c0 < q; c0 += shares * kShortBlock) {
    const int count = q - c0 < kShortBlock ? q - c0 : kShortBlock;
    for (int c = wave * 4; c < count; c += 16) {
      double f[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        f[i] = 16 * i + row < p && c + quarter < count ? x[static_cast<int64_t>(c0 + c + quarter) * p + 16 * i + row] : 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j <= i; ++j)
          acc[i * (i + 1) / 2 + j] = __builtin_amdgcn_mfma_f64_16x16x4f64(f[i], f[j], acc[i * (i + 1) / 2 + j], 0, 0, 0);
    }
  }
  short_gram_store<N>(acc, join, part + (z * shares + blockIdx.x) * (kTiles * 256));
}

struct ShortCoefficients {
  float c[3 * 32];
};

// P [z][16 N][16 N] of a round's steps, in the first with the 1 / (||U||_F + eps) of X_0 in it.
template <int N>
__global__ __launch_bounds__(64 * N * N) void ns_short_poly_kernel(const double* __restrict__ part, int shares, float eps,
                                                                   int first, int steps, ShortCoefficients coef,
                                                                   double* __restrict__ out) {
  constexpr int kTiles = N * (N + 1) / 2, kSide = 16 * N, kLd = kSide + 2;
  __shared__ double A[kSide * kLd], Q[kSide * kLd], P[kSide * kLd], B[N > 3 ? 1 : kSide * kLd];
  extern __shared__ __align__(16) double more[];
  double* R = N > 3 ? more : B;  // four of them pass the static limit at N = 4
  __shared__ double scale;
  const int64_t z = blockIdx.x;
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int ti = wave / N, tj = wave % N;  // the wave's 16 x 16 tile
  const int row = lane & 15, quarter = lane >> 4;
  // rows 4 v + quarter, column `row` of the tile
  auto at = [&](int v) { return (16 * ti + 4 * v + quarter) * kLd + 16 * tj + row; };
  {
    const int i = ti > tj ? ti : tj, j = ti > tj ? tj : ti;
    const double* from = part + z * shares * (kTiles * 256) + (i * (i + 1) / 2 + j) * 256;
    int slot[4];
    double sum[4] = {};
#pragma unroll
    for (int v = 0; v < 4; ++v)  // element (r, c) of the tile, or (c, r) of its mirror image: slot (r / 4) * 64 + (r % 4) * 16 + c
      slot[v] = ti >= tj ? v * 64 + lane : (row >> 2) * 64 + (row & 3) * 16 + 4 * v + quarter;
    for (int s = 0; s < shares; s += 8) {
      double in[8][4];
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          in[u][v] = from[static_cast<int64_t>(s + u < shares ? s + u : s) * (kTiles * 256) + slot[v]];
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) sum[v] += s + u < shares ? in[u][v] : 0.0;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) A[at(v)] = sum[v];
  }
  __syncthreads();
  if (wave == 0) {
    double t = lane < kSide ? A[lane * kLd + lane] : 0.0;
    t = wave_sum(t);
    if (lane == 0) {
      const double f = sqrt(t) + static_cast<double>(eps);
      scale = !first ? 1.0 : f > 0.0 || f != f ? 1.0 / f : 0.0;
    }
  }
  __syncthreads();
  const double s = scale;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    A[at(v)] *= s * s;
    P[at(v)] = 16 * ti + 4 * v + quarter == 16 * tj + row ? s : 0.0;
  }
  __syncthreads();
  // the wave's tile of X Y, Y symmetric
  auto product = [&](const double* X, const double* Y) {
    f64x4 acc = {};
#pragma unroll
    for (int k = 0; k < kSide; k += 4)
      acc = __builtin_amdgcn_mfma_f64_16x16x4f64(X[(16 * ti + row) * kLd + k + quarter], Y[(16 * tj + row) * kLd + k + quarter], acc, 0, 0, 0);
    return acc;
  };
  for (int k = 0; k < steps; ++k) {
    const double a = coef.c[3 * k], b = coef.c[3 * k + 1], c = coef.c[3 * k + 2];
    const f64x4 square = product(A, A);
#pragma unroll
    for (int v = 0; v < 4; ++v)
      Q[at(v)] = c * square[v] + b * A[at(v)] + (16 * ti + 4 * v + quarter == 16 * tj + row ? a : 0.0);
    __syncthreads();
    if (k + 1 == steps) {  // nobody asks for the next A
      const f64x4 p = product(P, Q);
      __syncthreads();
#pragma unroll
      for (int v = 0; v < 4; ++v) P[at(v)] = p[v];
      break;
    }
    const f64x4 p = product(P, Q), qa = product(A, Q);
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      P[at(v)] = p[v];
      R[at(v)] = qa[v];
    }
    __syncthreads();
    const f64x4 next = product(R, Q);
#pragma unroll
    for (int v = 0; v < 4; ++v) A[at(v)] = next[v];
    __syncthreads();
  }
#pragma unroll
  for (int v = 0; v < 4; ++v)
    out[(z * kSide + 16 * ti + 4 * v + quarter) * kSide + 16 * tj + row] = P[at(v)];
}

// O(:, c) = P U(:, c) for 256 c, stored or subtracted from W; before the last round (kLast false) X [z][q][p] is stored.
template <int N, typename T, bool kStep, bool kLast>
__global__ __launch_bounds__(256) void ns_short_apply_kernel(ShortU<T, kStep> U, const double* __restrict__ P, float keep,
                                                             float gain, T* out, double* __restrict__ X) {
  constexpr int kSide = 16 * N;
  extern __shared__ __align__(16) float lds[];
  const int64_t z = blockIdx.y;
  const int p = U.p(), q = U.q(), sk = U.sk(), sc = U.sc();
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int row = lane & 15, quarter = lane >> 4;
  const int c0 = static_cast<int>(blockIdx.x) * kShortBlock, count = q - c0 < kShortBlock ? q - c0 : kShortBlock;
  U.template load<false>(z, c0, count, lds);
  __syncthreads();
  const double* pz = P + z * kSide * kSide;
  for (int c = wave * 16; c < count; c += 64) {
    f64x4 acc[N] = {};
    const bool in = c + row < count;
#pragma unroll 4
    for (int k = 0; k < kSide; k += 4) {
      const double u = in && k + quarter < p ? static_cast<double>(lds[(k + quarter) * sk + (c + row) * sc]) : 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        acc[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(pz[(16 * i + row) * kSide + k + quarter], u, acc[i], 0, 0, 0);
    }
    // over the columns of U that only this wave has read
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int k = 16 * i + 4 * v + quarter;
        if (!in || k >= p) continue;
        if constexpr (kLast) lds[k * sk + (c + row) * sc] = static_cast<float>(acc[i][v]);
        else X[(z * q + c0 + c + row) * p + k] = acc[i][v];
      }
  }
  if constexpr (!kLast) return;
  __syncthreads();
  const int step = U.m <= U.n ? sc : sk;
  T* oz = out + z * U.m * static_cast<int64_t>(U.n);
  U.each(c0, count, [&](int64_t at, int k, int c, int some) {
    typedef T vec __attribute__((ext_vector_type(8)));
    const float* from = lds + k * sk + c * sc;
    if (U.wide) {
      vec w{};
      if constexpr (kStep) w = *reinterpret_cast<const vec*>(oz + at);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        w[e] = static_cast<T>(kStep ? fmaf(keep, static_cast<float>(w[e]), -gain * from[e * step]) : from[e * step]);
      *reinterpret_cast<vec*>(oz + at) = w;
    } else {
      for (int e = 0; e < some; ++e)
        oz[at + e] = static_cast<T>(kStep ? fmaf(keep, static_cast<float>(oz[at + e]), -gain * from[e * step]) : from[e * step]);
    }
  });
}

// A later round's P X: X again (in place: a wave reads all of its columns before it writes them), or the result.
template <int N, typename T, bool kStep, bool kLast>
__global__ __launch_bounds__(256) void ns_short_reapply_kernel(double* X, const double* __restrict__ P, int m, int n, float keep,
                                                               float gain, T* __restrict__ out) {
  constexpr int kSide = 16 * N;
  const int64_t z = blockIdx.y;
  const int p = m < n ? m : n, q = m < n ? n : m;
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int row = lane & 15, quarter = lane >> 4;
  const int c0 = static_cast<int>(blockIdx.x) * kShortBlock, count = q - c0 < kShortBlock ? q - c0 : kShortBlock;
  const double* pz = P + z * kSide * kSide;
  for (int c = wave * 16; c < count; c += 64) {
    f64x4 acc[N] = {};
    const bool in = c + row < count;
    double* x = X + (z * q + c0 + c + (in ? row : 0)) * p;
#pragma unroll 4
    for (int k = 0; k < kSide; k += 4) {
      const double u = in && k + quarter < p ? x[k + quarter] : 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        acc[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(pz[(16 * i + row) * kSide + k + quarter], u, acc[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int k = 16 * i + 4 * v + quarter;
        if (!in || k >= p) continue;
        if constexpr (kLast) {
          const float o = static_cast<float>(acc[i][v]);
          const int64_t at = m <= n ? static_cast<int64_t>(k) * n + c0 + c + row : static_cast<int64_t>(c0 + c + row) * n + k;
          T* to = out + z * m * static_cast<int64_t>(n) + at;
          *to = static_cast<T>(kStep ? fmaf(keep, static_cast<float>(*to), -gain * o) : o);
        } else {
          x[k] = acc[i][v];
        }
      }
  }
}

// Shares of the long side of one matrix: blocks of 256, up to 256 shares and about 2048 workgroups.
inline int ns_short_shares(int64_t batch, int q) {
  int64_t n = (q + kShortBlock - 1) / kShortBlock, most = 2048 / batch;
  if (most < 1) most = 1;
  if (most > 256) most = 256;
  return static_cast<int>(n < most ? n : most);
}

inline bool ns_short(int m, int n) { return (m < n ? m : n) <= kShortMost; }

struct NsArgs {
  int64_t batch;
  int m, n, steps;
  const float* coef;
  float eps;
};

double ns_bound(double a, double b, double c, double h);

// The end of the round that starts with step k; h, the bound of the singular values, moves along.
constexpr double kShortGrowth = 1 << 24;
inline int ns_short_round(const NsArgs& g, int k, double& h) {
  double grown = 1.0;
  const int from = k;
  for (; k < g.steps && (k == from || grown <= kShortGrowth); ++k) {
    const double a = g.coef[3 * k], b = g.coef[3 * k + 1], c = g.coef[3 * k + 2];
    auto q = [&](double s) { return fabs(a + s * (b + s * c)); };
    double top = fmax(q(0.0), q(h * h));
    if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < h * h) top = fmax(top, q(-b / (2.0 * c)));
    grown *= fmax(1.0, top * top);
    h = ns_bound(a, b, c, h);
  }
  return k;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int round_up(int v, int to) { return (v + to - 1) / to * to; }

size_t ns_workspace(int64_t batch, int32_t m, int32_t n, bool split) {
  if (ns_short(m, n)) {
    const size_t tiles = ((m < n ? m : n) + 15) / 16, b = static_cast<size_t>(batch);
    return align_up(b * ns_short_shares(batch > 0 ? batch : 1, m < n ? n : m) * (tiles * (tiles + 1) / 2) * 2048, 256) +
           align_up(b * tiles * tiles * 2048, 256) + align_up(b * m * n * 8, 256);
  }
  const int pad = split ? 32 : 8;
  const size_t b = static_cast<size_t>(batch), mp = round_up(m, pad), np = round_up(n, pad), p = mp < np ? mp : np,
               e = split ? 4 : 2;
  return align_up(b * ns_chunks(static_cast<int64_t>(m) * n) * 8, 256) + 2 * align_up(b * mp * np * e, 256) + (split ? 0 : 2 * align_up(b * mp * np * 2, 256)) +
         2 * align_up(b * p * p * e, 256);
}

// A step's: for either kind of operands.
size_t ns_step_workspace(int64_t batch, int32_t m, int32_t n) {
  const size_t a = ns_workspace(batch, m, n, true), b = ns_workspace(batch, m, n, false);
  return a > b ? a : b;
}

inline int64_t tiles_of(int rows, int side) { return (rows + side - 1) / side; }

// Tile sizes.  Small products want many small tiles, large ones the arithmetic intensity of large tiles:
//   64    64 x 64, three workgroups a CU                       below 128 tiles of 128 x 128
//   128d  128 x 128, one workgroup of 8 waves, 4 steps ahead   128 to 319 such tiles (about one a CU)
//   128   128 x 128, two workgroups of 4 waves a CU            from there
//   192, 256  one workgroup a CU, where their tiles fill at least 4/5 of the rounds of 256 CUs
// One step of a square matrix in us (P, P^2, X'; 22-bit operands): 1536 wide 26 + 27 + 39 with 64, 32 + 35 + 35
// with 128d, 40 + 43 + 43 with 128; 2048 wide 48 + 49 + 67, 46 + 47 + 53, 51 + 54 + 61; four of 2048: 140 + 141 + 243,
// 135 + 139 + 200, 131 + 135 + 189.  4096 wide: P 215 with 192 against 252 with 128; 11 bits: 85 against 100, X' 152 with 256
// against 165.
enum NsTile { kNs64, kNs128Deep, kNs128, kNs192, kNs256 };

inline bool fills_chip(int64_t tiles) { return 5 * tiles >= 4 * 256 * ((tiles + 255) / 256); }

inline NsTile ns_tile(int64_t tiles128, int64_t large, NsTile large_tile) {
  if (tiles128 < 128) return kNs64;
  if (large > 0 && fills_chip(large)) return large_tile;
  return tiles128 < 320 ? kNs128Deep : kNs128;
}

constexpr int tile_side(NsTile t) { return t == kNs64 ? 64 : t == kNs192 ? 192 : t == kNs256 ? 256 : 128; }

// A tile's copies reach offsets below 2^31 bytes.  Rows along the long side of a wide matrix take smaller tiles where they
// would pass that; parts of the contraction that run across such rows (32 of 22-bit operands, 64 of 11-bit ones) do not.
constexpr int64_t kLongest = (1ll << 30) / (kShortMost + 1) + 32;  // elements, padded
static_assert(31 * 4 * kLongest + 4096 < (1ll << 31) && 63 * 2 * kLongest + 4096 < (1ll << 31), "offsets of a tile's copies");
inline bool rows_fit(int rows, int64_t ld) { return (rows - 1) * ld + 128 <= 0x7fffffff; }

struct NsPlan {
  int m8, n8;
  unsigned nb;
  hipStream_t s;

  template <class S>
  void square_with(const _Float16* F, int k8, int width, const _Float16* in, double f_sum, double f_in, _Float16* out) const {
    const int p8 = m8 < n8 ? m8 : n8;
    const unsigned t = static_cast<unsigned>(tiles_of(p8, S::BM));
    ns_square_kernel<S><<<t * (t + 1) / 2 * nb, S::kThreads, 0, s>>>(F, p8, k8, width, in, static_cast<float>(f_sum),
                                                                    static_cast<float>(f_in), out);
  }
  // out = f_sum F F^T + f_in in
  template <class E, bool kCol>
  void square(const _Float16* F, int k8, int width, const _Float16* in, double f_sum, double f_in, _Float16* out) const {
    const int p8 = m8 < n8 ? m8 : n8;
    const int64_t t128 = tiles_of(p8, 128), t192 = tiles_of(p8, 192);
    NsTile tile = ns_tile(t128 * (t128 + 1) / 2 * nb, kCol ? 0 : t192 * (t192 + 1) / 2 * nb, kNs192);
    if constexpr (!kCol) {
      const int64_t ld = static_cast<int64_t>(width) * static_cast<int64_t>(sizeof(E));
      if (!rows_fit(tile_side(tile), ld)) tile = kNs64;
      if constexpr (__is_same(E, Split))  // 64 rows of 11-bit operands always fit
        if (!rows_fit(64, ld)) return square_with<TileShape<E, 32, 32, 1, 1, 4, 4, 2, false, false>>(F, k8, width, in, f_sum, f_in, out);
    }
    switch (tile) {
      case kNs64: return square_with<TileShape<E, 64, 64, 2, 2, 1, 3, 1, kCol, kCol>>(F, k8, width, in, f_sum, f_in, out);
      case kNs128Deep: return square_with<TileShape<E, 128, 128, 2, 4, 1, 4, 1, kCol, kCol>>(F, k8, width, in, f_sum, f_in, out);
      case kNs192:
        if constexpr (!kCol) return square_with<TileShape<E, 192, 192, 2, 2, 1, 2, 1, false, false>>(F, k8, width, in, f_sum, f_in, out);
        [[fallthrough]];
      default: return square_with<TileShape<E, 128, 128, 2, 2, 1, 2, 1, kCol, kCol>>(F, k8, width, in, f_sum, f_in, out);
    }
  }

  template <class S, bool kWide, bool kLast, typename T, bool kStep>
  void apply_with(const _Float16* X, const _Float16* B, double f_sum, double f_x, const _Float16* Xl, _Float16* Y,
             _Float16* Yl, const NsOut<T>& o) const {
    const unsigned tiles = static_cast<unsigned>(tiles_of(m8, S::BM) * tiles_of(n8, S::BN));
    ns_apply_kernel<S, kWide, kLast, T, kStep><<<tiles * nb, S::kThreads, 0, s>>>(
        X, B, m8, n8, static_cast<float>(f_sum), static_cast<float>(f_x), Xl, Y, Yl, o);
  }
  // Y (or the result) = f_sum B X + f_x X, or f_sum X B + f_x X
  template <class E, bool kWide, bool kLast, typename T, bool kStep>
  void apply(const _Float16* X, const _Float16* B, double f_sum, double f_x, const _Float16* Xl, _Float16* Y,
             _Float16* Yl, const NsOut<T>& o) const {
    constexpr bool kLarge = __is_same(E, _Float16);  // the fragments of 22-bit operands do not fit beside 256 x 256 sums
    switch (ns_tile(tiles_of(m8, 128) * tiles_of(n8, 128) * nb,
                    kLarge ? tiles_of(m8, 256) * tiles_of(n8, 256) * nb : 0, kNs256)) {
      case kNs64: return apply_with<TileShape<E, 64, 64, 2, 2, 1, 3, 1, false, kWide>, kWide, kLast, T, kStep>(X, B, f_sum, f_x, Xl, Y, Yl, o);
      case kNs128Deep: return apply_with<TileShape<E, 128, 128, 2, 4, 1, 4, 1, false, kWide>, kWide, kLast, T, kStep>(X, B, f_sum, f_x, Xl, Y, Yl, o);
      case kNs256:
        if constexpr (kLarge) return apply_with<TileShape<E, 256, 256, 2, 4, 1, 2, 1, false, kWide>, kWide, kLast, T, kStep>(X, B, f_sum, f_x, Xl, Y, Yl, o);
        [[fallthrough]];
      default: return apply_with<TileShape<E, 128, 128, 2, 2, 1, 2, 1, false, kWide>, kWide, kLast, T, kStep>(X, B, f_sum, f_x, Xl, Y, Yl, o);
    }
  }
};

template <class E, bool kWide, typename T, bool kStep>
lipcache_status ns_products(const NsArgs& g, double sx, _Float16* X, _Float16* Xl, _Float16* Y, _Float16* Yl, _Float16* A, _Float16* B, float keep,
                            float gain, T* out, hipStream_t s) {
  constexpr int kPad = NsAt<E>::kPad;
  const int m8 = round_up(g.m, kPad), n8 = round_up(g.n, kPad), p8 = kWide ? m8 : n8, q8 = kWide ? n8 : m8;
  // powers of two: the largest entry of X is at most the bound h of its singular values, of P h^2, of B |b| h^2 + |c| h^4
  double h = 1.0, top_x = 1.0, top_b = 1e-30;
  for (int k = 0; k < g.steps; ++k) {
    const double b = fabs(g.coef[3 * k + 1]), c = fabs(g.coef[3 * k + 2]);
    top_b = fmax(top_b, b * h * h + c * h * h * h * h);
    if (k + 1 < g.steps) h = ns_bound(g.coef[3 * k], g.coef[3 * k + 1], g.coef[3 * k + 2], h);
    top_x = fmax(top_x, h);
  }
  const double sp = exp2(floor(log2(32768.0 / (top_x * top_x)))), sb = exp2(fmin(20.0, floor(log2(32768.0 / top_b))));
  const NsPlan plan{m8, n8, static_cast<unsigned>(g.batch), s};
  for (int k = 0; k < g.steps; ++k) {
    const double a = g.coef[3 * k], b = g.coef[3 * k + 1], c = g.coef[3 * k + 2];
    plan.square<E, !kWide>(X, q8, n8, nullptr, sp / (sx * sx), 0.0, A);
    LC_LAUNCHED();
    plan.square<E, false>(A, p8, p8, A, c * sb / (sp * sp), b * sb / sp, B);
    LC_LAUNCHED();
    if (k + 1 < g.steps)
      plan.apply<E, kWide, false, float, false>(X, B, 1.0 / sb, a, Xl, Y, Yl, NsOut<float>{});
    else
      plan.apply<E, kWide, true, T, kStep>(X, B, 1.0 / (sb * sx), a / sx, Xl, nullptr, nullptr, NsOut<T>{out, g.m, g.n, keep, gain});
    LC_LAUNCHED();
    _Float16* t = X;
    X = Y;
    Y = t;
    t = Xl;
    Xl = Yl;
    Yl = t;
  }
  return LIPCACHE_OK;
}

template <int N, typename T, bool kStep>
lipcache_status ns_short_run(const NsArgs& g, const T* G, float* M, float mu, int nesterov, float keep, float gain, T* out,
                             void* ws, hipStream_t s) {
  const bool across = g.m <= g.n;
  const int p = across ? g.m : g.n, q = across ? g.n : g.m, shares = ns_short_shares(g.batch, q);
  // eight neighbours of a row stay in it
  const int wide = g.n % 8 == 0 && aligned16(G) && aligned16(out) && (!kStep || aligned16(M));
  const ShortU<T, kStep> U{G, M, g.m, g.n, mu, nesterov, wide};
  const unsigned nb = static_cast<unsigned>(g.batch);
  const size_t lds = static_cast<size_t>(ShortU<T, kStep>::room(p, across)) * 4;
  double* part = static_cast<double*>(ws);
  double* P = reinterpret_cast<double*>(static_cast<char*>(ws) +
                                        align_up(static_cast<size_t>(g.batch) * shares * (N * (N + 1) / 2) * 2048, 256));
  double* X = reinterpret_cast<double*>(reinterpret_cast<char*>(P) + align_up(static_cast<size_t>(g.batch) * N * N * 2048, 256));
  constexpr size_t kMore = N > 3 ? 16 * N * (16 * N + 2) * 8 : 0;
  const dim3 blocks(static_cast<unsigned>((q + kShortBlock - 1) / kShortBlock), nb);
  double h = 1.0;
  for (int k = 0, first = 1;; first = 0) {
    const int end = ns_short_round(g, k, h);
    const bool last = end == g.steps;
    ShortCoefficients coef{};
    for (int i = 0; i < 3 * (end - k); ++i) coef.c[i] = g.coef[3 * k + i];
    if (first) ns_short_gram_kernel<N, T, kStep><<<dim3(shares, nb), 256, lds, s>>>(U, shares, part);
    else ns_short_regram_kernel<N><<<dim3(shares, nb), 256, 0, s>>>(X, p, q, shares, part);
    LC_LAUNCHED();
    ns_short_poly_kernel<N><<<nb, 64 * N * N, kMore, s>>>(part, shares, g.eps, first, end - k, coef, P);
    LC_LAUNCHED();
    if (first && last) ns_short_apply_kernel<N, T, kStep, true><<<blocks, 256, lds, s>>>(U, P, keep, gain, out, X);
    else if (first) ns_short_apply_kernel<N, T, kStep, false><<<blocks, 256, lds, s>>>(U, P, keep, gain, out, X);
    else if (last) ns_short_reapply_kernel<N, T, kStep, true><<<blocks, 256, 0, s>>>(X, P, g.m, g.n, keep, gain, out);
    else ns_short_reapply_kernel<N, T, kStep, false><<<blocks, 256, 0, s>>>(X, P, g.m, g.n, keep, gain, out);
    LC_LAUNCHED();
    if (last) return LIPCACHE_OK;
    k = end;
  }
}

template <class E, typename T, bool kStep>
lipcache_status ns_run(const NsArgs& g, const void* G_, float* M, float mu, int nesterov, float keep, float gain,
                       void* out_, void* ws, hipStream_t s) {
  const T* G = static_cast<const T*>(G_);
  T* out = static_cast<T*>(out_);
  if (ns_short(g.m, g.n)) {
    const int tiles = ((g.m < g.n ? g.m : g.n) + 15) / 16;
    if (tiles == 1) return ns_short_run<1, T, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    if (tiles == 2) return ns_short_run<2, T, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    if (tiles == 3) return ns_short_run<3, T, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    return ns_short_run<4, T, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
  }
  const int m8 = round_up(g.m, NsAt<E>::kPad), n8 = round_up(g.n, NsAt<E>::kPad);
  const size_t b = static_cast<size_t>(g.batch), p8 = m8 < n8 ? m8 : n8;
  const int64_t size = static_cast<int64_t>(g.m) * g.n, room = static_cast<int64_t>(m8) * n8;
  const int chunks = ns_chunks(size);
  char* w = static_cast<char*>(ws);
  auto take = [&](size_t bytes) {
    char* at = w;
    w += align_up(bytes, 256);
    return at;
  };
  double* part = reinterpret_cast<double*>(take(b * chunks * 8));
  _Float16* X = reinterpret_cast<_Float16*>(take(b * room * sizeof(E)));
  _Float16* Y = reinterpret_cast<_Float16*>(take(b * room * sizeof(E)));
  const size_t low = NsAt<E>::kLow ? b * room * 2 : 0;
  _Float16* Xl = reinterpret_cast<_Float16*>(take(low));
  _Float16* Yl = reinterpret_cast<_Float16*>(take(low));
  _Float16* A = reinterpret_cast<_Float16*>(take(b * p8 * p8 * sizeof(E)));
  _Float16* B = reinterpret_cast<_Float16*>(take(b * p8 * p8 * sizeof(E)));
  const unsigned nb = static_cast<unsigned>(g.batch);
  const dim3 grid(chunks, nb);
  const int wide = g.n % 8 == 0 && aligned16(G) && (!kStep || aligned16(M));
  ns_norm_kernel<T, kStep><<<grid, 256, 0, s>>>(G, M, size, mu, nesterov, wide, part);
  LC_LAUNCHED();
  if (g.steps == 0) {
    ns_plain_kernel<T, kStep><<<grid, 256, 0, s>>>(G, M, size, mu, nesterov, part, chunks, g.eps, keep, gain, out);
    LC_LAUNCHED();
    return LIPCACHE_OK;
  }
  double top_x = 1.0, h = 1.0;
  for (int k = 0; k + 1 < g.steps; ++k) {
    h = ns_bound(g.coef[3 * k], g.coef[3 * k + 1], g.coef[3 * k + 2], h);
    top_x = fmax(top_x, h);
  }
  const double sx = exp2(floor(log2(32768.0 / top_x)));
  const unsigned blocks = static_cast<unsigned>((room + 2047) / 2048 < 4096 ? (room + 2047) / 2048 : 4096);
  ns_start_kernel<E, T, kStep><<<dim3(blocks, nb), 256, 0, s>>>(G, M, g.m, g.n, m8, n8, mu, nesterov, wide, part, chunks,
                                                               g.eps, static_cast<float>(sx), X, Xl);
  LC_LAUNCHED();
  if (g.m <= g.n) return ns_products<E, true, T, kStep>(g, sx, X, Xl, Y, Yl, A, B, keep, gain, out, s);
  return ns_products<E, false, T, kStep>(g, sx, X, Xl, Y, Yl, A, B, keep, gain, out, s);
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

template <class E, bool kStep>
lipcache_status ns_dispatch(const NsArgs& g, int32_t dtype, const void* G, float* M, float mu, int nesterov, float keep,
                            float gain, void* out, void* ws, hipStream_t s) {
  switch (dtype) {
    case LIPCACHE_F32: return ns_run<Split, float, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    case LIPCACHE_BF16: return ns_run<E, __bf16, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
    default: return ns_run<E, _Float16, kStep>(g, G, M, mu, nesterov, keep, gain, out, ws, s);
  }
}

}  // namespace lc

using namespace lc;

extern "C" size_t lipcache_orthogonalise_workspace_bytes(int64_t batch, int32_t m, int32_t n, int32_t dtype) {
  if (batch < 0 || m < 1 || n < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16) return 0;
  return ns_workspace(batch, m, n, true);
}

extern "C" lipcache_status lipcache_orthogonalise(const void* G, int64_t batch, int32_t m, int32_t n, int32_t dtype,
                                                  int32_t steps, const float* coef, float eps, void* out, void* ws,
                                                  size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = ns_check(batch, m, n, dtype, steps, coef, eps); st != LIPCACHE_OK) return st;
  if (batch > 0 && (ns_unaligned(G, dtype) || ns_unaligned(out, dtype))) return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < ns_workspace(batch, m, n, true)) return LIPCACHE_EWORKSPACE;
  if (batch == 0) return LIPCACHE_OK;
  const NsArgs g{batch, m, n, steps, coef, eps};
  return ns_dispatch<Split, false>(g, dtype, G, nullptr, 0.0f, 0, 0.0f, 0.0f, out, ws, stream);
}

extern "C" size_t lipcache_muon_step_workspace_bytes(int64_t batch, int32_t m, int32_t n, int32_t dtype) {
  if (batch < 0 || m < 1 || n < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16) return 0;
  return ns_step_workspace(batch, m, n);
}

extern "C" lipcache_status lipcache_muon_step(void* W, const void* G, float* M, int64_t batch, int32_t m, int32_t n,
                                              int32_t dtype, const lipcache_muon* opt, void* ws, size_t ws_bytes,
                                              lipcache_stream_t stream) {
  if (!opt) return LIPCACHE_EINVAL;
  if (lipcache_status st = ns_check(batch, m, n, dtype, opt->steps, opt->coef, opt->eps); st != LIPCACHE_OK) return st;
  if (!isfinite(opt->lr) || !isfinite(opt->momentum) || !isfinite(opt->weight_decay) || !isfinite(opt->scale))
    return LIPCACHE_EINVAL;
  const bool nesterov = (opt->nesterov & 1) != 0, few_bits = (opt->nesterov & LIPCACHE_MUON_SHORT_OPERANDS) != 0;
  if ((opt->nesterov & ~(1 | LIPCACHE_MUON_SHORT_OPERANDS)) != 0 || (few_bits && dtype == LIPCACHE_F32)) return LIPCACHE_EINVAL;
  if (batch > 0 && (ns_unaligned(W, dtype) || ns_unaligned(G, dtype) || ns_unaligned(M, LIPCACHE_F32)))
    return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < ns_step_workspace(batch, m, n)) return LIPCACHE_EWORKSPACE;
  if (batch == 0) return LIPCACHE_OK;
  const NsArgs g{batch, m, n, opt->steps, opt->coef, opt->eps};
  const float keep = static_cast<float>(1.0 - static_cast<double>(opt->lr) * opt->weight_decay);
  const float gain = static_cast<float>(static_cast<double>(opt->lr) * opt->scale);
  if (few_bits) return ns_dispatch<_Float16, true>(g, dtype, G, M, opt->momentum, nesterov, keep, gain, W, ws, stream);
  return ns_dispatch<Split, true>(g, dtype, G, M, opt->momentum, nesterov, keep, gain, W, ws, stream);
}
