// Log probabilities of rows of logits: labels, sums, entropies and the most
// likely classes (see lipcache.h for the formulas).
#include "lc_rows.hpp"

namespace lc {

constexpr int kTopMost = LIPCACHE_MOST_TOP;
// Candidates that a row's list holds, and the groups of threads whose largest values give the threshold.
template <class S>
inline constexpr int kTopList = S::G >= 64 ? 512 : 32;
template <class S>
inline constexpr int kTopGroups = S::G >= 64 ? 64 : 16;

struct LpScore {
  float temperature;
  const int32_t* label;
  int k;
  float *logp, *lse, *entropy;
  int32_t* top_index;
  float* top_logp;
};

struct TopCandidate {
  float v;
  int j;
};

template <class S>
struct TopSpace {
  float maxima[S::kRows][kTopGroups<S>];
  float least[S::kRows];
  int count[S::kRows];
  TopCandidate list[S::kRows][kTopList<S>];
};
template <class S>
struct TopRoom {
  float value[2][S::kWaves];
};

__device__ __forceinline__ bool top_before(float v, int j, float w, int i) { return v > w || (v == w && j < i); }

// A row's k largest, one after another: each the largest of those behind the one before.  each(f) calls f(value,
// index) for the thread's elements by rising index.
template <class S, class Each, class Put>
__device__ __forceinline__ void top_rounds(int k, TopRoom<S>& room, Each each, Put put) {
  float last = kRowInf;
  int last_at = -1;
  for (int i = 0; i < k; ++i) {
    float best = -kRowInf;
    int at = kRowMostClasses;
    each([&](float v, int j) {
      const bool left = v < last || (v == last && j > last_at);
      if (left && v > best) {
        best = v;
        at = j;
      }
    });
    float top = lanes_max<S::kLanes>(best), where;
    auto least = [](float a, float b) { return fminf(a, b); };
    if constexpr (S::kWaves > 1) {
      const int w = lane_id() & 15;
      __syncthreads();
      if (lane_id() == 0) room.value[0][threadIdx.x / kWave] = top;
      __syncthreads();
      top = lanes_max<16>(w < S::kWaves ? room.value[0][w] : -kRowInf);
      where = lanes_join<64>(best == top ? static_cast<float>(at) : static_cast<float>(kRowMostClasses), least);
      if (lane_id() == 0) room.value[1][threadIdx.x / kWave] = where;
      __syncthreads();
      where = lanes_join<16>(w < S::kWaves ? room.value[1][w] : static_cast<float>(kRowMostClasses), least);
    } else {
      where = lanes_join<S::kLanes>(best == top ? static_cast<float>(at) : static_cast<float>(kRowMostClasses), least);
    }
    last = top;
    last_at = static_cast<int>(where);  // below 2^24: exact
    put(i, top, last_at);
  }
}

// A row's k largest by a threshold: the largest value that k of the groups of threads reach.  What reaches it
// is a list of little more than k, each of which finds its place by counting: reaching(least, f) calls f(index) for
// the thread's elements that do, logit_of(index) gives the value.  Rows whose list would be longer (many equal
// values, or all large ones in few threads) go round by round.
template <class S, class Each, class Reaching, class Logit, class Put>
__device__ __forceinline__ void top_listed(int k, float own, const RowPlace<S>& at, TopSpace<S>& top, TopRoom<S>& room,
                                           Each each, Reaching reaching, Logit logit_of, Put put) {
  constexpr int kGroups = kTopGroups<S>;
  if (S::kWaves == 1 || threadIdx.x < kWave) {
    const float v = top.maxima[at.row][at.g % kGroups];
    int n = 0;
#pragma unroll
    for (int j = 0; j < kGroups; ++j) n += (kGroups == 64 ? lane_f32(v, j) : top.maxima[at.row][j]) >= v ? 1 : 0;
    const float least = lanes_max<kGroups>(n >= k ? v : -kRowInf);
    if (at.g == 0) {
      top.least[at.row] = least;
      top.count[at.row] = 0;
    }
  }
  RowPlace<S>::sync();
  const float least = top.least[at.row];
  if (own >= least && own > -kRowInf)
    reaching(least, [&](int j) {
      const int n = atomicAdd(&top.count[at.row], 1);
      if (n < kTopList<S>) top.list[at.row][n] = {logit_of(j), j};
    });
  RowPlace<S>::sync();
  const int n = top.count[at.row];
  if (n > kTopList<S>) {
    top_rounds<S>(k, room, each, [&](int i, float v, int j) {
      if (at.g == 0) put(i, v, j);
    });
    return;
  }
  for (int c = at.g; c < n || c < k; c += S::G) {
    if (c < n) {
      const TopCandidate mine = top.list[at.row][c];
      int place = 0;
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const TopCandidate other = top.list[at.row][i];
        place += top_before(other.v, other.j, mine.v, mine.j) ? 1 : 0;
      }
      if (place < k) put(place, mine.v, mine.j);
    } else {
      put(c, -kRowInf, 0);
    }
  }
}

template <class E, class S, bool kWhole>
__global__ __launch_bounds__(S::kThreads) void lp_score_kernel(const E* __restrict__ logits, int64_t ldx, int64_t T, int C,
                                                               LpScore a) {
  typedef RowData<E, S> Data;
  constexpr int kSegment = S::G * S::N;
  __shared__ RowSums room[2][S::kWaves];
  __shared__ TopSpace<S> top;
  __shared__ TopRoom<S> top_room;
  const RowPlace<S> at;
  const RowScale scale{kRowLog2e / a.temperature, 0.0f};
  const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows;
  const int full = C / Data::V;
  auto row_of = [&](int64_t t) { return logits + (t < T ? t : T - 1) * ldx; };
  auto label_of = [&](int64_t t) { return a.label && t < T ? a.label[t] : -1; };
  auto checked = [&](int y) { return y < C ? y : -1; };
  auto logit_of = [&](int64_t t, int y) { return y >= 0 ? static_cast<float>(row_of(t)[y]) : 0.0f; };
  Data data;
  int64_t t = static_cast<int64_t>(blockIdx.x) * S::kRows + at.row;
  int y = checked(label_of(t));
  float logit = logit_of(t, y);
  data.load(row_of(t), 0, C, at.g);
  for (int turn = 0; t - at.row < T; t += step, turn ^= 1) {
    const E* x = row_of(t);
    int next_y = label_of(t + step);
    RowSums r;
    data.template add<RowWants::kMean, true>(r, scale);
    if constexpr (!kWhole) {
      for (int first = kSegment; first < full; first += kSegment) {
#pragma unroll
        for (int i = 0; i < S::N; ++i) data.load_chunk(i, x, first, full, at.g);
        data.template add<RowWants::kMean, false>(r, scale);
      }
    }
    const float own = r.m;
    next_y = checked(next_y);
    const float next_logit = logit_of(t + step, next_y);
    if (a.k > 0) {
      float m = own;
      if constexpr (S::G >= 128) m = fmaxf(m, dpp_f32<kDppQuadXor1>(m));
      if constexpr (S::G >= 256) m = fmaxf(m, dpp_f32<kDppQuadXor2>(m));
      if constexpr (S::G >= 512) m = fmaxf(m, dpp_f32<kDppHalfMirror>(m));
      if constexpr (S::G >= 1024) m = fmaxf(m, dpp_f32<kDppMirror>(m));
      constexpr int kEach = S::G / kTopGroups<S>;
      if (at.g % kEach == 0) top.maxima[at.row][at.g / kEach] = m;
    }
    auto next = [&] { data.load(row_of(t + step), 0, C, at.g); };
    if (kWhole && a.k == 0) next();
    if constexpr (S::G <= 64) wave_sync();  // the join of longer rows has a barrier
    row_join<S, RowWants::kMean>(r, scale, room[turn]);
    const float from = row_from(r.m), log_s = row_log2(r.s);
    auto logp = [&](float v) { return r.s == 0.0f ? -kRowInf : (v - from) / a.temperature - log_s * kRowLn2; };
    if (t < T && at.g == 0) {
      if (a.logp) a.logp[t] = y >= 0 ? logp(logit) : 0.0f;
      if (a.lse) a.lse[t] = from / a.temperature + log_s * kRowLn2;
      if (a.entropy) a.entropy[t] = r.s == 0.0f ? 0.0f : (log_s - r.more / r.s) * kRowLn2;
    }
    if (a.k > 0) {
      auto put = [&](int i, float v, int j) {
        if (t >= T) return;
        a.top_index[t * a.k + i] = v == -kRowInf ? -1 : j;
        a.top_logp[t * a.k + i] = v == -kRowInf ? -kRowInf : logp(v);
      };
      // the rare ways through the row read it again
      auto each = [&](auto f) {
#pragma unroll 1
        for (int c = at.g; c < full; c += S::G) {
          const u32x4 raw = *reinterpret_cast<const typename Data::Type::vec*>(x + static_cast<int64_t>(c) * Data::V);
#pragma unroll
          for (int e = 0; e < Data::V; ++e) f(Data::Type::get(raw, e), c * Data::V + e);
        }
        f(data.tail, full * Data::V + at.g);
      };
      auto reaching = [&](float least, auto f) {
        if constexpr (kWhole) {
          data.reaching(least, 0, at.g, f);
        } else {
          for (int first = 0; first < full; first += kSegment) {
#pragma unroll
            for (int i = 0; i < S::N; ++i) data.load_chunk(i, x, first, full, at.g);
            data.reaching(least, first, at.g, f);
          }
        }
        if (data.tail >= least && data.tail > -kRowInf) f(full * Data::V + at.g);
      };
      if (a.k <= kTopGroups<S>) {
        top_listed<S>(a.k, own, at, top, top_room, each, reaching, [&](int j) { return static_cast<float>(x[j]); }, put);
      } else {
        top_rounds<S>(a.k, top_room, each, [&](int i, float v, int j) {
          if (at.g == 0) put(i, v, j);
        });
      }
    }
    if (!kWhole || a.k > 0) next();
    y = next_y;
    logit = next_logit;
  }
}

}  // namespace lc

using namespace lc;

extern "C" lipcache_status lipcache_logprobs(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                             float temperature, const int32_t* label, int32_t k, float* logp,
                                             float* lse, float* entropy, int32_t* top_index, float* top_logp,
                                             lipcache_stream_t stream) {
  if (lipcache_status st = row_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || (T > 0 && k > 0 && (!top_index || !top_logp))) return LIPCACHE_EINVAL;
  if (row_unaligned4(label) || row_unaligned4(logp) || row_unaligned4(lse) || row_unaligned4(entropy) ||
      row_unaligned4(top_index) || row_unaligned4(top_logp))
    return LIPCACHE_EINVAL;
  if (k > kTopMost) return LIPCACHE_EUNSUPPORTED;
  if (T == 0) return LIPCACHE_OK;
  const LpScore a{temperature, label, k, logp, lse, entropy, top_index, top_logp};
  return row_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    return row_shaped<E>(C, [&](auto shape, auto whole) {
      typedef decltype(shape) S;
      lp_score_kernel<E, S, decltype(whole)::value><<<row_blocks<S>(T), S::kThreads, 0, stream>>>(static_cast<const E*>(x), ldx, T, C, a);
      LC_LAUNCHED();
      return LIPCACHE_OK;
    });
  });
}
