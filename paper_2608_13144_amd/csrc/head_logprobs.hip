// Log probabilities straight from features and a head: the product W x + bias
// goes from the matrix cores' sums into each class tile's largest value and sums
// of exponentials, and no logit is written (see lipcache.h).
//
// The classes lie along the accumulators' rows, the features' rows along their
// columns: a lane holds 16 classes of one row in each 32 x 32 tile, so the sums over classes are sums over its registers, and only
// the two halves of a wave meet at the end.  Every wave of a tile leaves
// (largest value, sum, sum of the exponents weighted) of its classes; a second
// launch joins them in order.
#include <type_traits>

#include "lc_common.hpp"
#include "lc_mfma.hpp"

namespace lc {

constexpr int64_t kHlMostClasses = 1 << 20;
constexpr int64_t kHlMostWidth = 1 << 20;
constexpr float kHlLn2 = 0.6931471805599453f;
constexpr float kHlLog2e = 1.4426950408889634f;
constexpr float kHlInf = __builtin_huge_valf();
constexpr float kHlLeast = -1000.0f;  // exponents below add nothing: 2^-1000 is zero, and -inf times zero is not

inline int64_t hl_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Matrices whose own rows are not whole 16-byte vectors, as rows that are, zeros past the width: what the tiles are copied
// from.  Both operands in one launch (z); a lane takes a vector of a row, read from any element's address.  Bound by
// memory: 128192 x 294 float32 in 77 us (3.9 TB/s).
struct HlCopy {
  const void* from;
  void* to;
  int64_t ld, rows;  // of the source; 0 rows: nothing to do
};
struct HlCopies {
  HlCopy of[2];
};
template <class E>
__global__ __launch_bounds__(256) void hl_copy_kernel(HlCopies copies, int width) {
  constexpr int V = 16 / static_cast<int>(sizeof(E));
  typedef u32x4 __attribute__((aligned(2))) vec;
  const HlCopy c = copies.of[blockIdx.z];
  const int vectors = (width + V - 1) / V, at = static_cast<int>(blockIdx.x) * 64 + (static_cast<int>(threadIdx.x) & 63);
  if (at >= vectors) return;
  const int left = width - at * V;
  const int64_t step = static_cast<int64_t>(gridDim.y) * 4;
  const E* from = static_cast<const E*>(c.from) + at * V;
  E* to = static_cast<E*>(c.to) + at * V;
  const int64_t to_ld = static_cast<int64_t>(vectors) * V;
  int64_t row = static_cast<int64_t>(blockIdx.y) * 4 + (threadIdx.x >> 6);
  if (left >= V) {
    // four rows' loads under way at a time
    for (; row + 3 * step < c.rows; row += 4 * step) {
      u32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const vec*>(from + (row + i * step) * c.ld);
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(to + (row + i * step) * to_ld) = v[i];
    }
    for (; row < c.rows; row += step)
      *reinterpret_cast<u32x4*>(to + row * to_ld) = *reinterpret_cast<const vec*>(from + row * c.ld);
  } else {
    for (; row < c.rows; row += step)
#pragma unroll
      for (int e = 0; e < V; ++e) to[row * to_ld + e] = e < left ? from[row * c.ld + e] : static_cast<E>(0.0f);
  }
}

// (largest value, sum of 2^(scale (x - m)), sum of those times their exponents) of some classes.
struct HlPart {
  float m, s, mean;
};
__device__ __forceinline__ HlPart hl_join(const HlPart& a, const HlPart& b, float scale) {
  const float m = fmaxf(a.m, b.m);
  if (m == -kHlInf) return {m, a.s + b.s, a.mean + b.mean};  // no class yet (sums are zero, or NaN)
  const float da = (a.m - m) * scale, db = (b.m - m) * scale;
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  return {m, fmaf(a.s, fa, b.s * fb),
          fa * fmaf(fmaxf(da, kHlLeast), a.s, a.mean) + fb * fmaf(fmaxf(db, kHlLeast), b.s, b.mean)};
}

// The same sums about m, which is no smaller.
__device__ __forceinline__ void hl_move(HlPart& p, float m, float scale) {
  const float d = (p.m - (m == -kHlInf ? 0.0f : m)) * scale, f = __builtin_amdgcn_exp2f(d);
  p.mean = f * fmaf(fmaxf(d, kHlLeast), p.s, p.mean);
  p.s *= f;
  p.m = m;
}

struct HlOut {
  const int32_t* label;
  float *logp, *lse, *entropy;
  float scale, temperature;  // log2(e) / temperature
  __device__ __forceinline__ void write(int t, const HlPart& sum, bool labelled, float logit) const {
    const float m = sum.m == -kHlInf ? 0.0f : sum.m, log_s = __builtin_amdgcn_logf(sum.s);
    if (logp) logp[t] = !labelled ? 0.0f : sum.s == 0.0f ? -kHlInf : (logit - m) / temperature - log_s * kHlLn2;
    if (lse) lse[t] = m / temperature + log_s * kHlLn2;
    if (entropy) entropy[t] = sum.s == 0.0f ? 0.0f : (log_s - sum.mean / sum.s) * kHlLn2;
  }
};

// A tile of W x + bias with classes along the accumulators' rows (a lane holds 16 classes of a row of x in each 32 x 32 of it), and
// from the accumulators its share of every row's softmax: the largest logit, the sum and the sum for the entropy, joined across
// the lane's pair; 16 bytes a row and wave leave the chip instead of the logits.  4096 x 4096 -> 32768 bfloat16 871 us,
// bound by the product (1.26 PFLOP/s with its sums, 5 % of it); one row of 4096 -> 131072 179 us, bound by reading W (6 TB/s).
// kAll: the tile holds all classes and each wave those of its rows, which it finishes itself.  32768 x 256 -> 200
// float32 38 us, of which 24 are the products at the float32 matrix rate; the rest is one tile's start and end a CU.
// Registers for two waves a SIMD, or for as many as the ring leaves.
template <class S>
inline constexpr int kHlWaves = S::kThreads > 256 || 2 * S::kLds <= 160 * 1024 ? 2 : 1;
template <class S, bool kAll>
__global__ __launch_bounds__(S::kThreads, kHlWaves<S>) void hl_tile_kernel(const typename S::E* __restrict__ W, int64_t ldw, int C,
                                                              const typename S::E* __restrict__ x, int64_t ldx, int T,
                                                              int K, const float* __restrict__ bias, HlOut out, int parts,
                                                              float4* __restrict__ part, float* __restrict__ at) {
  typedef typename S::E E;
  static_assert(!kAll || S::WM == 1, "one wave for all classes of a row");
  __shared__ __align__(16) char lds[S::kLds];
  int bi, bj;
  tile_of(static_cast<int>((C + S::BM - 1) / S::BM), static_cast<int>((T + S::BN - 1) / S::BN), bi, bj);
  const int i0 = bi * S::BM, j0 = bj * S::BN;
  Side p{}, q{};
  p.p = W + i0 * ldw;
  p.ld = ldw * sizeof(E);
  p.rows = C - i0 < S::BM ? C - i0 : S::BM;
  q.p = x + j0 * ldx;
  q.ld = ldx * sizeof(E);
  q.rows = T - j0 < S::BN ? T - j0 : S::BN;
  f32x16 acc[S::TM][S::TN] = {};
  tile_products<S>(p, q, K, lds, acc);
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  if (S::WK > 1 && wave >= S::WM * S::WN) return;
  const int wm = wave / S::WN, wn = wave % S::WN, half = 4 * (lane >> 5);
  HlPart sum[S::TN];
  int y[S::TN];  // the label as a row of the wave's, counted from the lane's first
  float logit[S::TN];
  bool labelled[S::TN];
#pragma unroll
  for (int b = 0; b < S::TN; ++b) {
    const int t = j0 + (wn * S::TN + b) * 32 + (lane & 31);
    const int label = out.label && t < T ? out.label[t] : -1;
    labelled[b] = label >= 0 && label < C;
    y[b] = labelled[b] ? label - (i0 + wm * S::TM * 32 + half) : -1;
    logit[b] = 0.0f;
    sum[b] = {-kHlInf, 0.0f, 0.0f};
  }
#pragma unroll
  for (int a = 0; a < S::TM; ++a) {
    const int base = i0 + (wm * S::TM + a) * 32 + half;
    float add[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) add[v] = bias && base + acc_row(v) < C ? bias[base + acc_row(v)] : 0.0f;
#pragma unroll
    for (int b = 0; b < S::TN; ++b) {
      float x16[16], m = -kHlInf;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        x16[v] = base + acc_row(v) < C ? acc[a][b][v] + add[v] : -kHlInf;
        m = fmaxf(m, x16[v]);
      }
      hl_move(sum[b], fmaxf(m, sum[b].m), out.scale);
      const float from = sum[b].m == -kHlInf ? 0.0f : sum[b].m;
      float s = 0.0f, mean = 0.0f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float e = (x16[v] - from) * out.scale, w = __builtin_amdgcn_exp2f(e);
        s += w;
        mean = fmaf(fmaxf(e, kHlLeast), w, mean);
      }
      sum[b].s += s;
      sum[b].mean += mean;
      const int row = y[b] - a * 32;
      if (__ballot(row >= 0 && row < 32) != 0) {
#pragma unroll
        for (int v = 0; v < 16; ++v) logit[b] = row == acc_row(v) ? x16[v] : logit[b];
      }
      __builtin_amdgcn_sched_barrier(0);  // one tile's numbers at a time beside the accumulators
    }
  }
#pragma unroll
  for (int b = 0; b < S::TN; ++b) {
    const int t = j0 + (wn * S::TN + b) * 32 + (lane & 31);
    const HlPart other{__shfl_xor(sum[b].m, 32, kWave), __shfl_xor(sum[b].s, 32, kWave), __shfl_xor(sum[b].mean, 32, kWave)};
    const HlPart both = hl_join(sum[b], other, out.scale);
    const bool mine = y[b] >= 0 && y[b] < S::TM * 32 && (y[b] & 4) == 0;
    if constexpr (kAll) {
      const float across = __shfl_xor(logit[b], 32, kWave);
      const int there = __shfl_xor(mine ? 1 : 0, 32, kWave);
      if (lane < 32 && t < T) out.write(t, both, labelled[b], there ? across : logit[b]);
    } else {
      if (mine) at[t] = logit[b];
      if (lane < 32 && t < T) part[static_cast<int64_t>(t) * parts + bi * S::WM + wm] = {both.m, both.s, both.mean, 0.0f};
    }
  }
}

// WAVES waves join a row's parts: four rows a workgroup, or one.  Bound by latency: 7 us for one row of 131072 classes.
template <int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void hl_join_kernel(int T, int C, int parts, const float4* __restrict__ part,
                                                      const float* __restrict__ at, HlOut out) {
  __shared__ HlPart room[WAVES];
  const int wave = static_cast<int>(threadIdx.x) / kWave, lane = lane_id();
  const int t = WAVES == 1 ? static_cast<int>(blockIdx.x) * 4 + wave : static_cast<int>(blockIdx.x);
  HlPart sum{-kHlInf, 0.0f, 0.0f};
  if (t < T) {
#pragma unroll 4
    for (int i = lane + (WAVES == 1 ? 0 : wave * kWave); i < parts; i += WAVES * kWave) {
      const float4 p = part[static_cast<int64_t>(t) * parts + i];
      sum = hl_join(sum, {p.x, p.y, p.z}, out.scale);
    }
  }
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1)
    sum = hl_join(sum, {__shfl_xor(sum.m, o, kWave), __shfl_xor(sum.s, o, kWave), __shfl_xor(sum.mean, o, kWave)}, out.scale);
  if constexpr (WAVES > 1) {
    if (lane == 0) room[wave] = sum;
    __syncthreads();
    sum = room[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum = hl_join(sum, room[w], out.scale);
  }
  if (lane != 0 || (WAVES > 1 && wave != 0) || t >= T) return;
  const int y = out.label ? out.label[t] : -1;
  const bool labelled = y >= 0 && y < C;
  out.write(t, sum, labelled, labelled ? at[t] : 0.0f);
}

// ----------------------------------------------------------------- host side
template <class E>
inline constexpr int kHlVector = 16 / static_cast<int>(sizeof(E));

struct HlSpace {
  char* at;
  size_t used = 0;
  template <class T>
  T* take(int64_t n) {
    T* p = reinterpret_cast<T*>(at + used);
    used = align_up(used + static_cast<size_t>(n) * sizeof(T), 256);
    return p;
  }
};

inline int64_t hl_parts(int C) { return hl_ceil(C, 256) * 8; }  // at most, of any tile shape
// Rows of a pass: their parts stay below 256 MiB.
constexpr int64_t kHlPartBytes = 1 << 28;
static_assert(kHlPartBytes / (kHlMostClasses / 256 * 8 * 16) >= 256, "some rows a pass");
inline int64_t hl_rows(int64_t T, int C) {
  const int64_t most = kHlPartBytes / (hl_parts(C) * 16) / 256 * 256;
  return T < most ? T : most;
}

template <class E>
bool hl_aligned(const void* p, int64_t ld, int K) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % kHlVector<E> == 0 && K % kHlVector<E> == 0 &&
         ld * static_cast<int64_t>(sizeof(E)) <= (4 << 20);
}

// Parts, label's logits, and copies of the operands whose rows are not whole 16-byte vectors.
template <class E>
struct HlBuffers {
  float4* part;
  float* at;
  E *x = nullptr, *W = nullptr;
  HlBuffers(HlSpace& ws, const void* x_, int64_t ldx, int64_t T, const void* W_, int64_t ldw, int K, int C) {
    const int64_t rows = hl_rows(T, C), K8 = hl_ceil(K, kHlVector<E>) * kHlVector<E>;
    part = ws.take<float4>(rows * hl_parts(C));
    at = ws.take<float>(rows);
    if (!hl_aligned<E>(x_, ldx, K)) x = ws.take<E>(T * K8);
    if (!hl_aligned<E>(W_, ldw, K)) W = ws.take<E>(C * K8);
  }
};

// The operands, or their copies in the workspace.
template <class E>
lipcache_status hl_vectors(const E*& x, int64_t& ldx, int64_t T, const E*& W, int64_t& ldw, int64_t C, int K,
                           const HlBuffers<E>& ws, hipStream_t s) {
  if (!ws.x && !ws.W) return LIPCACHE_OK;
  const int64_t to = hl_ceil(K, kHlVector<E>) * kHlVector<E>, across = hl_ceil(to / kHlVector<E>, 64);
  // about 4096 workgroups an operand
  const int64_t most = hl_ceil(T > C ? T : C, 4), some = 4096 / across < 64 ? 64 : 4096 / across;
  const HlCopies copies{{{x, ws.x, ldx, ws.x ? T : 0}, {W, ws.W, ldw, ws.W ? C : 0}}};
  const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>(most < some ? most : some), 2);
  hl_copy_kernel<E><<<grid, 256, 0, s>>>(copies, K);
  LC_LAUNCHED();
  if (ws.x) {
    x = ws.x;
    ldx = to;
  }
  if (ws.W) {
    W = ws.W;
    ldw = to;
  }
  return LIPCACHE_OK;
}

// Heads of up to 256 classes and many rows: one tile has all classes, and a row is finished where its sums are.  float32 products
// are what bounds such a call, so their tiles come in steps of 32 classes; 16-bit ones wait for the features.  Fewer rows
// leave CUs idle that way (64 rows of 256 -> 200 float32: 20 us against 12 of the tiles below and the join).
inline bool hl_whole(int64_t T, int C) { return C <= 256 && T > 64 * 128; }

template <class E>
lipcache_status hl_all(const E* x, int64_t ldx, int64_t T, const E* W, int64_t ldw, const float* bias, int K, int C,
                       const HlOut& out, hipStream_t s) {
  auto run = [&](auto shape) {
    typedef decltype(shape) S;
    hl_tile_kernel<S, true><<<static_cast<unsigned>(hl_ceil(T, S::BN)), S::kThreads, 0, s>>>(
        W, ldw, C, x, ldx, static_cast<int>(T), K, bias, out, 0, nullptr, nullptr);
    return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
  };
  // 128 rows a workgroup where that fills the CUs, else 64, whose waves share the contraction two by two.  32768 x 256 ->
  // 200 float32: 38 us of 128 rows, 44 of 64 (the shares are joined in LDS), 78 of 32.
  auto sized = [&](auto tm) {
    constexpr int BM = 32 * decltype(tm)::value;
    if (T > 128 * 192) return run(TileShape<E, BM, 128, 1, 4, 1, 3, 1, false, false>{});
    return run(TileShape<E, BM, 64, 1, 2, 2, 2, 1, false, false>{});
  };
  const int tiles = static_cast<int>(hl_ceil(C, 32));
  if constexpr (sizeof(E) == 4) {
    switch (tiles) {
      case 1: return sized(std::integral_constant<int, 1>{});
      case 2: return sized(std::integral_constant<int, 2>{});
      case 3: return sized(std::integral_constant<int, 3>{});
      case 4: return sized(std::integral_constant<int, 4>{});
      case 5: return sized(std::integral_constant<int, 5>{});
      case 6: return sized(std::integral_constant<int, 6>{});
      case 7: return sized(std::integral_constant<int, 7>{});
      default: return sized(std::integral_constant<int, 8>{});
    }
  } else {
    if (tiles <= 1) return sized(std::integral_constant<int, 1>{});
    if (tiles <= 4) return sized(std::integral_constant<int, 4>{});
    return sized(std::integral_constant<int, 8>{});
  }
}

template <class E>
lipcache_status hl_run(const E* x, int64_t ldx, int64_t T, const E* W, int64_t ldw, const float* bias, int K, int C,
                       HlOut out, void* ws_, hipStream_t s) {
  HlSpace space{static_cast<char*>(ws_)};
  const HlBuffers<E> ws(space, x, ldx, T, W, ldw, K, C);
  lipcache_status st;
  if ((st = hl_vectors(x, ldx, T, W, ldw, C, K, ws, s)) != LIPCACHE_OK) return st;
  const int64_t pass = hl_rows(T, C);
  for (int64_t t = 0; t < T; t += pass) {
    const int n = static_cast<int>(T - t < pass ? T - t : pass);
    HlOut o = out;
    if (out.label) o.label = out.label + t;
    if (out.logp) o.logp = out.logp + t;
    if (out.lse) o.lse = out.lse + t;
    if (out.entropy) o.entropy = out.entropy + t;
    if (hl_whole(n, C)) {
      if ((st = hl_all<E>(x + t * ldx, ldx, n, W, ldw, bias, K, C, o, s)) != LIPCACHE_OK) return st;
      continue;
    }
    int parts = 0;
    auto run = [&](auto shape) {
      typedef decltype(shape) S;
      parts = static_cast<int>(hl_ceil(C, S::BM)) * S::WM;
      const int64_t tiles = hl_ceil(C, S::BM) * hl_ceil(n, S::BN);
      hl_tile_kernel<S, false><<<static_cast<unsigned>(tiles), S::kThreads, 0, s>>>(W, ldw, C, x + t * ldx, ldx, n, K, bias, o,
                                                                                  parts, ws.part, ws.at);
      return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
    };
    const int64_t t128 = hl_ceil(C, 128) * hl_ceil(n, 128), t256 = hl_ceil(C, 256) * hl_ceil(n, 256);
    if (n <= 32) {
      // bound by reading W: tiles of 32 classes until they fill the CUs
      st = hl_ceil(C, 128) >= 256 ? run(TileShape<E, 128, 32, 4, 1, 1, 4, 1, false, false>{})
                                  : run(TileShape<E, 32, 32, 1, 1, 4, 4, 1, false, false>{});
    } else if (hl_ceil(C, 128) >= 256 && (n <= 64 || (sizeof(E) == 4 && n < 512 && hl_ceil(n, 64) % 2 == 1))) {
      // 64 rows of 4096 -> 131072 bfloat16: 240 us with tiles of 128 rows.  float32, bound by its products, takes 64 rows
      // also where 128 would leave half of the last tile empty: 300 rows of 1024 -> 65536 356 us (403), 171 of 296 ->
      // 128192 168 (201); bfloat16 loses by it (300 rows: 83 us, 75 with 128).
      st = run(TileShape<E, 128, 64, 4, 1, 1, 3, 1, false, false>{});
    } else if (hl_ceil(C, 64) * hl_ceil(n, 64) < (sizeof(E) == 4 ? 512 : 128)) {
      // tiles of 64 x 64 that leave CUs idle, or float32 matrix cores waiting: 32 x 32, whose four waves share the contraction.
      // 64 rows of 4096 -> 1000 float32 25 us (68 with 64 x 64), 189 of 3528 -> 440 24 (61), 64 of 4096 -> 20000 134 (244),
      // 2000 of 1000 -> 500 26 (24); bfloat16 loses by it past 128 tiles (700 rows of 4096 -> 1500 35 us, 28 with 64 x 64).
      st = run(TileShape<E, 32, 32, 1, 1, 4, 4, 1, false, false>{});
    } else if (t128 < 128) {
      // 128 x 128 would leave half of the CUs idle: 1024 rows of 4096 -> 1920 bfloat16 (120 such tiles) 28 us, 32 with 128 x 128;
      // 1280 -> 2048 (160) 40 and 32
      st = run(TileShape<E, 64, 64, 2, 2, 1, 3, 1, false, false>{});
    } else if (sizeof(E) == 2 && 5 * t256 >= 4 * 256 * hl_ceil(t256, 256)) {
      // 256 x 256, one a CU, where they fill four fifths of their rounds: 2048 rows of 4096 -> 6656 (208 of 256) 98 us, 119 with
      // 128 x 128 of four waves, 4096 -> 32768 876 and 1047; 2048 -> 9216 (288 of 512) 189 and 156
      if constexpr (sizeof(E) == 2) st = run(TileShape<E, 256, 256, 2, 4, 1, 2, 1, false, false>{});
    } else if (t128 < 320) {
      // about one tile a CU: eight waves and a longer ring.  2048 rows of 4096 -> 2048 (256 tiles) bfloat16 39 us, 45 with four
      // waves, float32 244 and 253; -> 3200 (400) 68 and 60
      st = run(TileShape<E, 128, 128, 2, 4, 1, 4, 1, false, false>{});
    } else {
      st = run(TileShape<E, 128, 128, 2, 2, 1, 2, 1, false, false>{});
    }
    if (st != LIPCACHE_OK) return st;
    // a wave a row, or more where a row has many parts (4096 of one row: 10 us by four waves)
    if (parts <= 256) hl_join_kernel<1><<<static_cast<unsigned>(hl_ceil(n, 4)), 256, 0, s>>>(n, C, parts, ws.part, ws.at, o);
    else if (parts <= 1024) hl_join_kernel<4><<<static_cast<unsigned>(n), 256, 0, s>>>(n, C, parts, ws.part, ws.at, o);
    else hl_join_kernel<16><<<static_cast<unsigned>(n), 1024, 0, s>>>(n, C, parts, ws.part, ws.at, o);
    LC_LAUNCHED();
  }
  return LIPCACHE_OK;
}

bool hl_sizes_bad(int64_t T, int32_t K, int32_t C, int32_t dtype) {
  return T < 0 || K < 1 || C < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16;
}
bool hl_unaligned(const void* p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

}  // namespace lc

using namespace lc;

extern "C" size_t lipcache_head_logprobs_workspace_bytes(const void* x, int64_t ldx, int64_t T, const void* W, int64_t ldw,
                                                         int32_t K, int32_t C, int32_t dtype) {
  if (hl_sizes_bad(T, K, C, dtype) || T == 0) return 0;
  HlSpace space{nullptr};
  if (dtype == LIPCACHE_F32) HlBuffers<float>(space, x, ldx, T, W, ldw, K, C);
  else HlBuffers<__bf16>(space, x, ldx, T, W, ldw, K, C);
  return space.used;
}

extern "C" lipcache_status lipcache_head_logprobs(const void* x, int64_t ldx, int64_t T, const void* W, int64_t ldw,
                                                  const float* bias, int32_t K, int32_t C, int32_t dtype,
                                                  float temperature, const int32_t* label, float* logp, float* lse,
                                                  float* entropy, void* ws, size_t ws_bytes, lipcache_stream_t stream) {
  if (hl_sizes_bad(T, K, C, dtype) || ldx < K || ldw < K) return LIPCACHE_EINVAL;
  if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f)) return LIPCACHE_EINVAL;
  if (T > 0 && (!W || !x)) return LIPCACHE_EINVAL;
  const uintptr_t size = dtype == LIPCACHE_F32 ? 4 : 2;
  if (hl_unaligned(x, size) || hl_unaligned(W, size) || hl_unaligned(bias, 4) || hl_unaligned(label, 4) ||
      hl_unaligned(logp, 4) || hl_unaligned(lse, 4) || hl_unaligned(entropy, 4))
    return LIPCACHE_EINVAL;
  if (C > kHlMostClasses || K > kHlMostWidth || T > 0x7fffffff) return LIPCACHE_EUNSUPPORTED;
  if (T == 0) return LIPCACHE_OK;
  if (!ws || !aligned256(ws) || ws_bytes < lipcache_head_logprobs_workspace_bytes(x, ldx, T, W, ldw, K, C, dtype))
    return LIPCACHE_EWORKSPACE;
  const HlOut out{label, logp, lse, entropy, kHlLog2e / temperature, temperature};
  auto run = [&](auto type) {
    typedef decltype(type) E;
    return hl_run<E>(static_cast<const E*>(x), ldx, T, static_cast<const E*>(W), ldw, bias, K, C, out, ws, stream);
  };
  switch (dtype) {
    case LIPCACHE_F32: return run(float{});
    case LIPCACHE_BF16: return run(__bf16{});
    default: return run(_Float16{});
  }
}
