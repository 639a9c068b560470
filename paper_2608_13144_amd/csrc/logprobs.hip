// Log probabilities of rows of logits: labels, sums, entropies and the most
// likely classes (see lipcache.h for the formulas).
#include "lc_rows.hpp"

namespace lc {

constexpr int kTopMost = LIPCACHE_MOST_TOP;
// Groups of a row's first segment whose largest values give the threshold: 16 for up to 8 alternatives (about 1.4 each reach
// it in what the groups have seen).  For more, four of every thread where a row has up to 64 threads, else 256 (1.1 to 1.2 each,
// up to 5 for 64 of 64 groups: 1024 x 131072 bfloat16 with 12 takes 65 us with 256 groups, 79 with 16).
constexpr int kTopFew = 8;
template <class S>
inline constexpr int kTopGroups = S::G <= 64 ? 16 : 256;

struct LpScore {
  float temperature;
  const int32_t* label;
  int k;
  float *logp, *lse, *entropy;
  int32_t* top_index;
  float* top_logp;
};

// A candidate: larger values first, equal ones by rising index (-0 is 0).
__device__ __forceinline__ uint64_t top_key(float v, int j) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
  return static_cast<uint64_t>(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | ~static_cast<uint32_t>(j);
}
__device__ __forceinline__ float top_value(uint64_t key) {
  const uint32_t b = static_cast<uint32_t>(key >> 32);
  return __builtin_bit_cast(float, b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int top_index(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }

// Every wave of a row (its lanes, where a wave holds several) has a list of its own.
template <class S>
inline constexpr int kTopList = S::G < 64 ? 64 : S::G == 64 ? 512 : S::G == 256 ? 256 : 128;
template <class S>
struct TopSpace {
  float maxima[2][S::kRows][kTopGroups<S>];  // of this call of top_least and of the one before, which waves may still read
  int count[S::kRows][S::kWaves];
  union {
    uint64_t list[S::kRows][S::kWaves][kTopList<S>];
    uint32_t bins[S::kRows][2 * S::kWaves * kTopList<S>];  // where a list ran over
  };
};

// A number in the order of the floats; 0x007fffff is -inf.
__device__ __forceinline__ uint32_t top_order(float v) { return static_cast<uint32_t>(top_key(v, 0) >> 32); }
// The largest number whose last 16 bits are zero that k of those of L lanes reach, found bit by bit.
template <int L, int N>
__device__ __forceinline__ uint32_t top_reached(int k, const uint32_t (&v)[N]) {
  uint32_t found = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t with = found | 1u << bit;
    if constexpr (L == 64) {
      int reach = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) reach += __builtin_popcountll(__ballot(v[i] >= with));
      found = reach >= k ? with : found;
    } else {
      float reach = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) reach += v[i] >= with ? 1.0f : 0.0f;
      found = lanes_sum<L>(reach) >= static_cast<float>(k) ? with : found;
    }
  }
  return found;
}
// The number of the type that is next to it, up (below -inf: nothing but -inf or less, which is no candidate).
template <class E>
__device__ __forceinline__ float top_float(uint32_t found) {
  if (found <= 0x007fffffu) return -kRowInf;
  constexpr uint32_t kMore = sizeof(E) == 4 ? 0 : std::is_same<E, __bf16>::value ? 0xffffu : 0x1fffu;  // bits that the type lacks
  return top_value(static_cast<uint64_t>(found & 0x80000000u ? found : found | kMore) << 32);
}

// A value that k of the groups of a row's threads reach, `own` being what a thread has: the largest such with 16 groups, with
// 256 the largest whose last 16 bits are zero.  At least k elements of what the threads have seen reach it.  The row's
// threads meet here; each wave counts for itself.
template <class E, class S>
__device__ __forceinline__ float top_least(int k, float own, const RowPlace<S>& at, TopSpace<S>& top, int& turn) {
  constexpr int G = S::G, kMany = kTopGroups<S>;
  const bool few = G <= 64 || k <= kTopFew;
  float m = own;
  turn ^= 1;
  float* maxima = top.maxima[turn][at.row];
  if (few) {
    if constexpr (G >= 32) m = fmaxf(m, dpp_f32<kDppQuadXor1>(m));
    if constexpr (G >= 64) m = fmaxf(m, dpp_f32<kDppQuadXor2>(m));
    if constexpr (G >= 128) m = fmaxf(m, dpp_f32<kDppHalfMirror>(m));
    if constexpr (G >= 256) m = fmaxf(m, dpp_f32<kDppMirror>(m));
    if constexpr (G >= 512) m = fmaxf(m, __shfl_xor(m, 16, kWave));
    if constexpr (G >= 1024) m = fmaxf(m, __shfl_xor(m, 32, kWave));
    if (at.g % (G / 16) == 0) maxima[at.g / (G / 16)] = m;
  } else {
    if constexpr (G >= 2 * kMany) m = fmaxf(m, dpp_f32<kDppQuadXor1>(m));
    if constexpr (G >= 4 * kMany) m = fmaxf(m, dpp_f32<kDppQuadXor2>(m));
    if (at.g % (G / kMany) == 0) maxima[at.g / (G / kMany)] = m;
  }
  RowPlace<S>::sync();
  if (few) {
    // a group's place is the number of groups that reach its value
    const float v = maxima[lane_id() & 15];
    int n = 1;
    auto count = [&](float other) { n += other >= v ? 1 : 0; };
    count(dpp_f32<0x121>(v));  // row_ror: the 15 other lanes of 16
    count(dpp_f32<0x122>(v));
    count(dpp_f32<0x123>(v));
    count(dpp_f32<0x124>(v));
    count(dpp_f32<0x125>(v));
    count(dpp_f32<0x126>(v));
    count(dpp_f32<0x127>(v));
    count(dpp_f32<0x128>(v));
    count(dpp_f32<0x129>(v));
    count(dpp_f32<0x12a>(v));
    count(dpp_f32<0x12b>(v));
    count(dpp_f32<0x12c>(v));
    count(dpp_f32<0x12d>(v));
    count(dpp_f32<0x12e>(v));
    count(dpp_f32<0x12f>(v));
    return lanes_max<16>(n >= k ? v : -kRowInf);
  }
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = G > 64 ? top_order(maxima[lane_id() + 64 * i]) : 0;
  return top_float<E>(top_reached<64>(k, v));
}

// The list that a wave's lanes fill: a place is the number of the lanes before and of what is there already, so
// nothing waits for an atomic.
template <class S>
struct TopList {
  uint64_t* list;
  int n = 0;  // may pass what the list holds; what does not fit is not written
  // All lanes of the row in this wave.
  __device__ __forceinline__ void push(bool hit, float v, int j) {
    uint64_t all = __ballot(hit);
    int before;
    if constexpr (S::G < 64) {
      all = all >> (lane_id() & ~(S::G - 1)) & ((1ull << S::G) - 1);
      before = __builtin_popcount(static_cast<uint32_t>(all) & ((1u << (lane_id() & (S::G - 1))) - 1));
    } else {
      before = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(all >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(all), 0));
    }
    if (hit && n + before < kTopList<S>) list[n + before] = top_key(v, j);
    n += __builtin_popcountll(all);
  }
};

// A candidate's place in the order of all: what top_key joins.
struct TopLeast {
  uint32_t order, index;
  __device__ __forceinline__ bool reached(float v, int j) const {
    const uint32_t o = top_order(v);
    return o > order || (o == order && ~static_cast<uint32_t>(j) >= index);
  }
};

// A key that at least k of a row's elements reach, and no more than one list holds, whatever the values; k elements reach `least`, and
// none is past `most`.  Those past `least` are counted first, fewer than k where many are equal to it.  Else those of the value's
// first bits are counted, then those that share the k-th's by their next bits; then, among the equal ones, by the bits of ~index,
// until few enough are left.  Keys differ, so the last bits leave k.  each(f) calls f(value, index) for the thread's
// elements, whole waves at a time.  Up to eight readings of the row, most often two; the row's threads meet here, and its
// lists are overwritten.  64 alternatives of rows that rise, or hold one value: 2100 x 16384 bfloat16 100 and 136 us (random ones
// 35), 4096 x 32768 304 and 432 (94), 1024 x 131072 303 and 513 (74); one alternative after another 1964 to 4500.
template <class S, class Each>
__device__ __forceinline__ TopLeast top_select(int k, float least, float most, int C, uint32_t* bins, Each each) {
  constexpr int L = S::kLanes, kBits = S::G < 64 ? 7 : 8, kBins = 1 << kBits, kOwn = kBins / L;
  static_assert(kBins <= 2 * S::kWaves * kTopList<S> && kTopList<S> >= kTopMost, "room for bins, and for k in one list");
  auto same = [](auto v) { return L == 64 ? uniform(static_cast<int>(v)) : static_cast<int>(v); };  // of all lanes of a row
  const uint32_t lo = same(top_order(least)), hi = same(top_order(most));
  const int index_bits = C > 1 ? 32 - __builtin_clz(C - 1) : 1;
  int beyond = 0;  // keys past all that share the found one's bits: fewer than k
  if (lo != hi) {
    float past = 0.0f;  // (below 2^24: exact)
    each([&](float v, int) { past += v > least ? 1.0f : 0.0f; });
    beyond = same(lanes_sum<L>(past));
    if constexpr (S::kWaves > 1) {
      if (lane_id() == 0) bins[threadIdx.x / kWave] = static_cast<uint32_t>(beyond);
      __syncthreads();
      beyond = 0;
      for (int w = 0; w < S::kWaves; ++w) beyond += same(bins[w]);
      __syncthreads();
    }
  }
  bool values = beyond >= k;
  int bits = values ? 32 - __builtin_clz(lo ^ hi) : index_bits;
  TopLeast found{lo, ~0u << index_bits};
  if (values) {
    found = {hi >> (bits - 1) >> 1 << (bits - 1) << 1, 0};
    beyond = 0;
  }
  for (;;) {
    const int shift = bits > kBits ? bits - kBits : 0;
    const uint32_t known = ~0u << (bits - 1) << 1, mask = (1u << (bits - shift)) - 1;
    // (the thread's place as a new number: what follows from it would be kept in registers from row to row)
    int thread = static_cast<int>(threadIdx.x);
    asm volatile("" : "+v"(thread));
    const int lane = thread % L;
    for (int b = thread % S::G; b < kBins; b += S::G) bins[b] = 0;
    RowPlace<S>::sync();
    each([&](float v, int j) {
      const uint32_t o = top_order(v), word = values ? o : ~static_cast<uint32_t>(j);
      const bool in = v >= least && v > -kRowInf &&
                      (values ? ((o ^ found.order) & known) == 0 : o == found.order && ((word ^ found.index) & known) == 0);
      const int bin = static_cast<int>(word >> shift & mask);
      if constexpr (S::G >= 64) {
        // (most of a wave's are often of one bin)
        const uint64_t all = __ballot(in);
        if (all == 0) return;
        const int first = __builtin_ctzll(all), one = __builtin_amdgcn_readlane(bin, first);
        if (__ballot(in && bin == one) == all) {
          if (lane == first) atomicAdd(&bins[one], static_cast<uint32_t>(__builtin_popcountll(all)));
          return;
        }
      }
      if (in) atomicAdd(&bins[bin], 1u);
    });
    RowPlace<S>::sync();
    int mine = 0;
#pragma unroll 1
    for (int b = 0; b < kOwn; ++b) mine += static_cast<int>(bins[lane * kOwn + b]);
    int past = mine;  // with the lanes' behind, whose bins are of larger keys
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      const int other = __builtin_amdgcn_ds_bpermute((thread + o) * 4, past);
      past += lane + o < L ? other : 0;
    }
    past += beyond - mine;
    float bin = 0.0f, over = 0.0f, with = 0.0f;  // of the one bin that holds the k-th: below 2^24, exact
#pragma unroll 1
    for (int b = kOwn - 1; b >= 0; --b) {
      const int reach = past + static_cast<int>(bins[lane * kOwn + b]);
      if (past < k && reach >= k) {
        bin = static_cast<float>(lane * kOwn + b);
        over = static_cast<float>(past);
        with = static_cast<float>(reach);
      }
      past = reach;
    }
    const uint32_t more = static_cast<uint32_t>(same(lanes_max<L>(bin))) << shift;
    const int reach = same(lanes_max<L>(with));
    beyond = same(lanes_max<L>(over));
    RowPlace<S>::sync();  // the bins are read
    if (values) found.order |= more;
    else found.index |= more;
    bits = shift;
    if (reach <= kTopList<S> || (bits == 0 && !values)) break;
    if (bits == 0) {
      values = false;
      bits = index_bits;
      found.index = ~0u << bits;
    }
  }
  return found;
}

// Scores of rows, one pass: with a thread's own largest value m, s = sum 2^(c (x - m)) and the exponents' sum weighted by
// what they add, c = log2(e) / temperature; joined, lse = m / temperature + ln s and entropy = ln s - ln 2 sum / s.
//
// Alternatives: a threshold that k elements of the row's first segment reach (the largest values of its threads give
// it), then every block of the row whose largest value reaches it puts its elements that do on a list, a few times k of
// them, each of which finds its place by counting.  Where a list is too short for them (the first segment holds
// little of what is large, or many values are equal), a threshold from the threads' largest values of the whole row
// and another pass follow, and where that is not enough either, a key found by counting (top_select) and another.
//
// Bound by memory without alternatives (4096 x 32768 bfloat16 50 us, 5.4 TB/s; 1024 x 131072 46 us, 5.8 TB/s), by vector
// instructions with them (eight 72 and 58 us, 64 92 and 73; without the threshold, one after another, each costs a reading
// of the row).  32768 x 200 float32, 13.6 us with five: the joins of so short rows.
//
// kWhole: a row is one segment.  kShare: a workgroup takes a share of a row, and leaves its sums and its k largest (keys
// in falling order, 0 where there are fewer) for lp_score_join_kernel.
template <class E, class S, bool kWhole, bool kShare>
__global__ __launch_bounds__(S::kThreads) void lp_score_kernel(const E* __restrict__ logits, int64_t ldx, int64_t T, int C,
                                                               LpScore a, RowShares shares, RowSums* __restrict__ sums,
                                                               uint64_t* __restrict__ keys) {
  static_assert(!kShare || (!kWhole && S::kRows == 1), "a share goes in segments");
  typedef RowData<E, S> Data;
  constexpr int kSegment = S::G * S::N;
  __shared__ RowSums room[2][S::kWaves];
  __shared__ TopSpace<S> top;
  const RowPlace<S> at;
  const RowScale scale{kRowLog2e / a.temperature, 0.0f};
  const int64_t step = kShare ? T : static_cast<int64_t>(gridDim.x) * S::kRows;
  const int full = C / Data::V;
  const int share = kShare ? static_cast<int>(blockIdx.x) % shares.count : 0;
  const bool last = !kShare || share == shares.count - 1;
  const int begin = kShare ? share * shares.each : 0, end = last ? full : begin + shares.each;
  auto row_of = [&](int64_t t) { return logits + (t < T ? t : T - 1) * ldx; };
  auto label_of = [&](int64_t t) { return a.label && t < T ? a.label[t] : -1; };
  auto checked = [&](int y) { return y < C ? y : -1; };
  auto logit_of = [&](int64_t t, int y) { return y >= 0 ? static_cast<float>(row_of(t)[y]) : 0.0f; };
  Data data(at.g);
  int64_t t = kShare ? static_cast<int>(blockIdx.x) / shares.count : static_cast<int64_t>(blockIdx.x) * S::kRows + at.row;
  int y = kShare ? -1 : checked(label_of(t));
  float logit = logit_of(t, y);
  data.tail = -kRowInf;
  if (last) data.load_tail(row_of(t), C, at.g);
#pragma unroll
  for (int i = 0; i < S::N; ++i) data.load_chunk(i, row_of(t), begin, end, at.g);
  const int wave = S::kWaves > 1 ? static_cast<int>(threadIdx.x) / kWave : 0;  // of the row
  int top_turn = 0;
  for (int turn = 0; t - at.row < T; t += step, turn ^= 1) {
    const E *x = row_of(t), *following = row_of(t + step);
    int next_y = kShare ? -1 : label_of(t + step);
    const float tail = data.tail;
    TopList<S> list{top.list[at.row][wave]};
    float least = kRowInf;
    auto hits = [&](float v) { return v >= least && v > -kRowInf; };
    if (a.k > 0) {
      bool found = false;
      if constexpr (S::G <= 64) {
        if (a.k > kTopFew) {
          // four groups a lane
          float m[4];
          uint32_t v[4];
          data.largest(begin, end, at.g, m);
#pragma unroll
          for (int p = 0; p < 4; ++p) v[p] = top_order(m[p]);
          least = top_float<E>(top_reached<S::G>(a.k, v));
          found = true;
        }
      }
      if (!found) {
        float m[1];
        data.largest(begin, end, at.g, m);
        least = top_least<E, S>(a.k, m[0], at, top, top_turn);
      }
      list.push(hits(tail), tail, full * Data::V + at.g);
    }
    RowSums r = data.template begin<RowWants::kMean>(scale);
    float next_logit = 0.0f;
    auto next = [&] {
      next_y = checked(next_y);
      next_logit = logit_of(t + step, next_y);
      data.load_tail(following, C, at.g);
    };
    auto seen = [&](float m, auto each) {
      if (a.k > 0 && __ballot(hits(m)) != 0) each(hits, [&](bool any, float v, int j) { list.push(any, v, j); });
    };
    // a threshold from all that the threads have seen, which no more than a few times k of the lists reach; past its barrier
    // the waves have read the counts
    auto cut = [&](float own) {
      least = top_least<E, S>(a.k, own, at, top, top_turn);
      const int mine = list.n < kTopList<S> ? list.n : kTopList<S>;
      if (list.n > mine) return;  // (some are lost already)
      list.n = 0;
      for (int i = lane_id(); i - lane_id() < mine; i += kWave) {
        const uint64_t key = i < mine ? list.list[i] : 0;
        list.push(key != 0 && top_value(key) >= least, top_value(key), top_index(key));  // (no place behind what is read)
      }
    };
    // a segment's chunks are asked for as the one before is used, the next row's behind the row's last
    int first = begin;
    if constexpr (!kWhole) {
      for (int done = 1; first + kSegment < end; first += kSegment, ++done) {
        data.template add<RowWants::kMean>(first, end, at.g, r, scale, seen,
                                           [&](int i) { data.load_chunk(i, x, first + kSegment, end, at.g); });
        // lists of long rows stay short: 1943 x 103064 float32 with 64 alternatives 164 us, 272 without
        if constexpr (S::kWaves > 1) {
          if (a.k > 0 && done > 1 && (done & (done - 1)) == 0) cut(r.m);
        }
      }
    }
    if constexpr (kShare) {
      data.template add<RowWants::kMean>(first, end, at.g, r, scale, seen, RowNothing{});
    } else {
      next();
      data.template add<RowWants::kMean>(first, full, at.g, r, scale, seen,
                                         [&](int i) { data.load_chunk(i, following, 0, full, at.g); });
    }
    const float own = r.m;
    if (a.k > 0 && at.g % S::kLanes == 0) top.count[at.row][wave] = list.n;
    if constexpr (S::G <= 64) wave_sync();  // the join of longer rows has a barrier
    row_join<S, RowWants::kMean>(r, scale, room[turn]);
    const float from = row_from(r.m), log_s = row_log2(r.s);
    auto logp = [&](float v) { return r.s == 0.0f ? -kRowInf : (v - from) / a.temperature - log_s * kRowLn2; };
    if (kShare) {
      if (at.g == 0) sums[blockIdx.x] = r;
    } else if (t < T && at.g == 0) {
      if (a.logp) a.logp[t] = y >= 0 ? logp(logit) : 0.0f;
      if (a.lse) a.lse[t] = from / a.temperature + log_s * kRowLn2;
      if (a.entropy) a.entropy[t] = r.s == 0.0f ? 0.0f : (log_s - r.more / r.s) * kRowLn2;
    }
    if (a.k > 0) {
      auto put = [&](int i, float v, int j) {
        if (t >= T) return;
        if constexpr (kShare) {
          keys[static_cast<int64_t>(blockIdx.x) * a.k + i] = v == -kRowInf ? 0 : top_key(v, j);
          return;
        }
        a.top_index[t * a.k + i] = v == -kRowInf ? -1 : j;
        a.top_logp[t * a.k + i] = v == -kRowInf ? -kRowInf : logp(v);
      };
      // what is on the row's lists, -1 where one is too short
      auto listed = [&] {
        int n = 0;
        bool fits = true;
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) {
          const int c = top.count[at.row][w];
          fits = fits && c <= kTopList<S>;
          n += c;
        }
        n = fits ? n : -1;
        return S::G < 64 ? n : uniform(n);
      };
      int n = listed();
      if constexpr (S::kWaves > 1) {
        if (n > 128) {
          // (n candidates take n steps, by G at a time: 1024 x 131072 bfloat16 with 64 alternatives 73 us, 138 without the cut)
          cut(own);
          if (lane_id() == 0) top.count[at.row][wave] = list.n;
          __syncthreads();
          n = listed();
        }
      }
      // (the same in a row held by a wave, most often of equal values: 32768 x 500 bfloat16, 488 of each row's classes masked by the
      // lowest value, with 64 alternatives 116 us, 907 on lists of all)
      if (S::G == 64 && kWhole && n > 128) n = -1;
      if (n < 0) {
        // the rare ways read the row again
        auto each = [&](auto f) {
#pragma unroll 1
          for (int c = begin + at.g - at.g % S::kLanes; c < end; c += S::G) {  // (whole waves)
            const int mine = c + at.g % S::kLanes;
            u32x4 raw = Data::fill();
            if (mine < end) raw = *reinterpret_cast<const typename Data::Type::vec*>(x + static_cast<int64_t>(mine) * Data::V);
#pragma unroll
            for (int e = 0; e < Data::V; ++e) f(Data::Type::get(raw, e), mine * Data::V + e);
          }
          f(tail, full * Data::V + at.g);
        };
        auto relisted = [&](auto take) {
          list.n = 0;
          each([&](float v, int j) { list.push(take(v, j), v, j); });
          if (at.g % S::kLanes == 0) top.count[at.row][wave] = list.n;
          RowPlace<S>::sync();
          return listed();
        };
        if constexpr (!kWhole) {
          // (a row of one segment had its whole row's threshold at first; 16 groups never give one for more than 16)
          if (S::G == 64 && a.k > kTopFew) {
            const uint32_t v[1] = {top_order(own)};
            least = fmaxf(least, top_float<E>(top_reached<64>(a.k, v)));
          } else {
            least = top_least<E, S>(a.k, own, at, top, top_turn);  // (past its barrier the counts are read)
          }
          n = relisted([&](float v, int) { return hits(v); });
        }
        if (n < 0) {
          const TopLeast from = top_select<S>(a.k, least, r.m, C, top.bins[at.row], each);
          n = relisted([&](float v, int j) { return hits(v) && from.reached(v, j); });
        }
      }
      for (int c = at.g; c < n || c < a.k; c += S::G) {
        if (c >= n) {
          put(c, -kRowInf, 0);
          continue;
        }
        int w = 0, i = c;
        while (S::kWaves > 1 && i >= top.count[at.row][w]) i -= top.count[at.row][w++];
        const uint64_t key = top.list[at.row][w][i];
        int place = 0;
#pragma unroll 1
        for (int o = 0; o < S::kWaves; ++o) {
          const int m = top.count[at.row][o];
#pragma unroll 4
          for (int e = 0; e < m; ++e) place += top.list[at.row][o][e] > key ? 1 : 0;
        }
        if (place < a.k) put(place, top_value(key), top_index(key));
      }
    }
    y = next_y;
    logit = next_logit;
  }
}

// Joins a row's shares.  The k-th of what the shares' m-th alternatives reach, m = k over the shares, is a threshold: what
// reaches it is a list whose entries find their places by counting.  One row of 131072 with 20 alternatives: 5 us, of which
// most is the chain of load, threshold, list and places.
template <class E>
__global__ __launch_bounds__(256) void lp_score_join_kernel(const E* __restrict__ logits, int64_t ldx, int C, LpScore a,
                                                            RowShares shares, const RowSums* __restrict__ sums,
                                                            const uint64_t* __restrict__ keys) {
  typedef RowShape<256, 1> S;
  __shared__ RowSums room[S::kWaves];
  __shared__ uint64_t list[kRowShares * kTopMost];
  __shared__ int count;
  const RowPlace<S> at;
  const int64_t t = blockIdx.x;
  const RowScale scale{kRowLog2e / a.temperature, 0.0f};
  int y = a.label ? a.label[t] : -1;
  if (y >= C) y = -1;
  const float logit = y >= 0 ? static_cast<float>(logits[t * ldx + y]) : 0.0f;
  RowSums r = at.g < shares.count ? sums[t * shares.count + at.g] : RowSums{-kRowInf, 0.0f, 0.0f};
  if (at.g == 0) count = 0;
  row_join<S, RowWants::kMean>(r, scale, room);
  const float from = row_from(r.m), log_s = row_log2(r.s);
  auto logp = [&](float v) { return r.s == 0.0f ? -kRowInf : (v - from) / a.temperature - log_s * kRowLn2; };
  if (at.g == 0) {
    if (a.logp) a.logp[t] = y >= 0 ? logp(logit) : 0.0f;
    if (a.lse) a.lse[t] = from / a.temperature + log_s * kRowLn2;
    if (a.entropy) a.entropy[t] = r.s == 0.0f ? 0.0f : (log_s - r.more / r.s) * kRowLn2;
  }
  if (a.k == 0) return;
  const uint64_t* mine = keys + t * shares.count * a.k;
  const int m = (a.k + shares.count - 1) / shares.count;
  uint64_t least = lane_id() < shares.count ? mine[lane_id() * a.k + m - 1] : ~0ull;  // each wave for itself
#pragma unroll
  for (int o = 1; o < kRowShares; o <<= 1) {
    const uint64_t other = __shfl_xor(static_cast<unsigned long long>(least), o, kWave);
    least = other < least ? other : least;
  }
  least = __shfl(static_cast<unsigned long long>(least), 0, kWave);
  for (int i = at.g; i < shares.count * a.k; i += S::G) {
    const uint64_t key = mine[i];
    if (key >= least && key != 0) list[atomicAdd(&count, 1)] = key;
  }
  __syncthreads();
  const int n = count;
  for (int c = at.g; c < n || c < a.k; c += S::G) {
    int place = c;
    const uint64_t key = c < n ? list[c] : 0;
    if (c < n) {
      place = 0;
#pragma unroll 4
      for (int i = 0; i < n; ++i) place += list[i] > key ? 1 : 0;
    }
    if (place >= a.k) continue;
    a.top_index[t * a.k + place] = c < n ? top_index(key) : -1;
    a.top_logp[t * a.k + place] = c < n ? logp(top_value(key)) : -kRowInf;
  }
}

// Without alternatives one workgroup is as fast as two launches up to 16384 chunks (131072 bfloat16: 12 us and 15).
inline RowShares score_shares(int64_t T, int C, int k, int32_t dtype) {
  const RowShares shares = row_shares(T, C, dtype);
  const int chunks = C / (dtype == LIPCACHE_F32 ? 4 : 8);
  return k == 0 && chunks <= 16384 ? RowShares{1, chunks} : shares;
}

inline size_t score_bytes(int64_t T, int k, const RowShares& shares) {
  if (shares.count == 1) return 0;
  const size_t n = static_cast<size_t>(T) * shares.count;
  return align_up(n * sizeof(RowSums), 256) + align_up(n * k * sizeof(uint64_t), 256);
}

// Threads of a row.  Rows of up to 64 chunks are held by 16 lanes, of up to 256 by a wave.  Longer ones go through in
// segments: by a wave up to 2048 chunks where the rows fill the chip with waves (2560 where several times), by 256 threads, or
// by 1024 where there are few.  With five alternatives a wave and 256 threads a row: 24261 x 9399 bfloat16 134 and 197 us,
// 6001 x 16384 51 and 63, 2100 x 9399 21 and 23, 6001 x 20480 62 and 75, 4096 x 32768 with eight 81 and 72; 8192 x 32768 with 20
// alternatives 172 and 158.  A wave's list grows with the alternatives and, as its first segment is the smaller part of it, with
// the row, and is ranked by 64 lanes.  With 64 alternatives: 2100 x 5003 bfloat16 20 and 26 us, 2100 x 16384 79 to 90 and 34,
// 6001 x 10000 float32 187 and 74.  Where there are many rows the others' work hides it longer: 24261 x 9399 230 and 262,
// 13048 x 18112 float16 with 40 alternatives 191 and 201, with 48 218 and 204.
// The 64 groups of 16 lanes give a threshold for up to 32 alternatives, about 44 of 32 on a list of 64: 32768 x 200 float32 with 16
// takes 20 us, 37 with a wave a row, with 32 28 and 41.
template <class E, class F>
lipcache_status score_shaped(int64_t T, int C, int k, F f) {
  const int chunks = C / RowType<E>::V;
  if (k <= 32) {
    if (chunks <= 16) return f(RowShape<16, 1>{}, std::true_type{});
    if (chunks <= 32) return f(RowShape<16, 2>{}, std::true_type{});
    if (chunks <= 64) return f(RowShape<16, 4>{}, std::true_type{});
  }
  if (chunks <= 256) return f(RowShape<64, 4>{}, std::true_type{});
  const bool few = k * chunks <= (T >= 12000 ? 98304 : 57344);  // alternatives, for a wave
  if (T >= 2048 && few && chunks <= (T >= 6000 ? 2560 : 2048)) return f(RowShape<64, 8>{}, std::false_type{});
  if (chunks <= 1024 || T >= 768) return f(RowShape<256, 8>{}, std::false_type{});
  return f(RowShape<1024, 4>{}, std::false_type{});
}

}  // namespace lc

using namespace lc;

extern "C" lipcache_status lipcache_logprobs(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                             float temperature, const int32_t* label, int32_t k, float* logp,
                                             float* lse, float* entropy, int32_t* top_index, float* top_logp,
                                             void* ws, size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = row_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || (T > 0 && k > 0 && (!top_index || !top_logp))) return LIPCACHE_EINVAL;
  if (row_unaligned4(label) || row_unaligned4(logp) || row_unaligned4(lse) || row_unaligned4(entropy) ||
      row_unaligned4(top_index) || row_unaligned4(top_logp))
    return LIPCACHE_EINVAL;
  if (k > kTopMost) return LIPCACHE_EUNSUPPORTED;
  if (T == 0) return LIPCACHE_OK;
  const RowShares shares = score_shares(T, C, k, dtype);
  if (const size_t need = score_bytes(T, k, shares); need > 0 && (!ws || !aligned256(ws) || ws_bytes < need))
    return LIPCACHE_EWORKSPACE;
  const LpScore a{temperature, label, k, logp, lse, entropy, top_index, top_logp};
  return row_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    const E* logits = static_cast<const E*>(x);
    if (shares.count > 1) {
      typedef RowShape<256, 4> S;
      RowSums* sums = static_cast<RowSums*>(ws);
      uint64_t* keys = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + align_up(T * shares.count * sizeof(RowSums), 256));
      lp_score_kernel<E, S, false, true>
          <<<static_cast<unsigned>(T * shares.count), S::kThreads, 0, stream>>>(logits, ldx, T, C, a, shares, sums, keys);
      LC_LAUNCHED();
      lp_score_join_kernel<E><<<static_cast<unsigned>(T), 256, 0, stream>>>(logits, ldx, C, a, shares, sums, keys);
      LC_LAUNCHED();
      return LIPCACHE_OK;
    }
    return score_shaped<E>(T, C, k, [&](auto shape, auto whole) {
      typedef decltype(shape) S;
      lp_score_kernel<E, S, decltype(whole)::value, false>
          <<<row_blocks<S>(T), S::kThreads, 0, stream>>>(logits, ldx, T, C, a, shares, nullptr, nullptr);
      LC_LAUNCHED();
      return LIPCACHE_OK;
    });
  });
}

extern "C" size_t lipcache_logprobs_workspace_bytes(int64_t T, int32_t C, int32_t k, int32_t dtype) {
  return row_sizes_bad(T, C, k, dtype) ? 0 : score_bytes(T, k, score_shares(T, C, k, dtype));
}
