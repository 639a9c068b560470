// Distillation: losses of rows of logits against labels and a teacher's top
// logits, and their gradient (see lipcache.h for the formulas).
#include "lc_rows.hpp"

namespace lc {

struct LpDistill {
  float temperature, hard, soft;
  float scale, second;  // log2(e) over the temperature of the first sum (the teacher's, where there are two), of the second
  const int32_t* label;
  const float* weight;
  int k;
  const float* teacher;
  const int32_t* index;
  float *ce, *kl;
  int bits;  // of the entries' index
};

struct LpShares {
  float hard, soft;  // of the row, with its weight; zero where it has no label, no entry
};

// The row's sums at one temperature or both from one reading; meanwhile its first wave has the teacher's softmax over the
// entries; then the gradient from the same registers, and the named places behind it.  Bound by memory: 4096 x 131072 bfloat16 with 64
// entries 456 us (4.7 TB/s), 4096 x 32768 with one temperature 116 (4.6) and two 129 (another exponential an element: vector pipe).
// Small calls are one row's chain of loads, joins and entries: 4096 x 200 float32 with all 200 entries 13 us.
// kSplit: a workgroup takes a share of a row whose sums are there already.
template <class E, class S, bool kWhole, bool kTwo, bool kSplit>
__global__ __launch_bounds__(S::kThreads) void lp_distill_kernel(const E* logits, int64_t ldx, int64_t T, int C,
                                                                 LpDistill a, E* grad, int64_t ldd, RowSplit split) {
  static_assert(!kSplit || (!kWhole && S::kRows == 1), "a share goes in segments");
  typedef RowData<E, S> Data;
  constexpr RowWants kWants = kTwo ? RowWants::kTwo : RowWants::kSum;
  constexpr int kSegment = S::G * S::N, kLanes = S::kLanes;
  __shared__ RowSums room[2][S::kWaves];
  __shared__ LpShares shares[2][S::kRows];
  extern __shared__ __align__(16) char lds[];
  const RowPlace<S> at;
  const int lane = at.g;  // (of the row's first wave, where it matters)
  const bool keeps = at.g < kLanes;
  RowEntries<kLanes> entries(lds + at.row * entry_bytes(a.k, a.bits), a.k, a.bits);
  const RowScale scale{a.scale, a.second};
  const float hot_scale = kRowLog2e / a.temperature;
  const int64_t step = kSplit ? T : static_cast<int64_t>(gridDim.x) * S::kRows;
  const int full = C / Data::V;
  const int share = kSplit ? static_cast<int>(blockIdx.x) % split.shares.count : 0;
  const bool last = !kSplit || share == split.shares.count - 1;
  const int begin = kSplit ? share * split.shares.each : 0, end = last ? full : begin + split.shares.each;
  auto row_of = [&](int64_t t) { return logits + (t < T ? t : T - 1) * ldx; };
  auto entry_of = [&](int64_t t, int i) {
    RowEntry e{-1, 0.0f};
    if (t < T && i < a.k) e = {a.index[t * a.k + i], a.teacher[t * a.k + i]};
    return e;
  };
  auto label_of = [&](int64_t t) { return t < T && a.label ? a.label[t] : -1; };
  auto inside = [&](int c) { return c < C ? c : -1; };
  // of entry i (a.k: the label), which names class c
  auto logit_of = [&](int64_t t, int i, int c) {
    if constexpr (kSplit) return t < T && i <= a.k ? split.logits[t * (a.k + 1) + i] : 0.0f;
    else return c >= 0 ? static_cast<float>(row_of(t)[c]) : 0.0f;
  };
  Data data(at.g);
  int64_t t = kSplit ? static_cast<int>(blockIdx.x) / split.shares.count : static_cast<int64_t>(blockIdx.x) * S::kRows + at.row;
  RowEntry mine{-1, 0.0f};
  int y = -1;
  float logit = 0.0f, y_logit = 0.0f;
  if (keeps) {
    mine = entry_of(t, lane);
    mine.at = inside(mine.at);
    y = inside(label_of(t));
    logit = logit_of(t, lane, mine.at);
    y_logit = logit_of(t, a.k, y);
  }
  if constexpr (!kSplit) data.load(row_of(t), 0, C, at.g);
  else data.load_tail(row_of(t), C, at.g);
  for (int turn = 0; t - at.row < T; t += step, turn ^= 1) {
    const E* x = row_of(t);
    RowEntry next_entry{-1, 0.0f};
    int next_y = -1;
    float w = 1.0f;
    if (keeps) {
      next_entry = entry_of(t + step, lane);
      next_y = label_of(t + step);
      if (a.weight && t < T) w = a.weight[t];
    }
    RowSums r = data.template begin<kWants>(scale);
    if constexpr (kSplit) {
      r = at.g < split.shares.count ? split.sums[t * split.shares.count + at.g] : RowSums{-kRowInf, 0.0f, 0.0f};
    } else if constexpr (kWhole) {
      data.template add<kWants>(0, full, at.g, r, scale, RowNothing{}, RowNothing{});
    } else {
      // a segment's chunks are asked for as the one before is used
      for (int first = 0; first < full; first += kSegment)
        data.template add<kWants>(first, full, at.g, r, scale, RowNothing{}, [&](int i) { data.load_chunk(i, x, first + kSegment, full, at.g); });
    }
    next_entry.at = inside(next_entry.at);
    next_y = inside(next_y);
    float top = -kRowInf, sum = 0.0f, some = 0.0f;
    if (keeps) {
      auto loaded = [&](int i) {
        RowEntry e = entry_of(t, i);
        e.at = inside(e.at);
        return e;
      };
      entries.keep(lane, mine, logit, loaded, [&](int i, int c) { return logit_of(t, i, c); });
      for (int i = lane; i < a.k; i += kLanes)
        if (entries.at[i] >= 0) {
          const float v = entries.value[i];
          top = fmaxf(top, v);
          some = v == -kRowInf ? some : 1.0f;  // (a NaN is an entry)
        }
      top = row_from(lanes_max<kLanes>(top));
      some = lanes_max<kLanes>(some);
      for (int i = lane; i < a.k; i += kLanes)
        if (entries.at[i] >= 0) sum += row_exp2((entries.value[i] - top) * hot_scale);
      sum = lanes_sum<kLanes>(sum);
      if (lane == 0) shares[turn][at.row] = {y >= 0 ? w * a.hard : 0.0f, some != 0.0f ? w * a.soft / a.temperature : 0.0f};
      wave_sync();
    }
    row_join<S, kWants>(r, scale, room[turn]);
    const LpShares part = shares[turn][at.row];
    const float from = row_from(r.m);
    const bool any = (part.hard != 0.0f || part.soft != 0.0f) && r.s != 0.0f;
    // what an element adds: one exponential with both parts' factor, or one for each
    const float one = (kTwo ? part.soft : part.hard + part.soft) / r.s, two = kTwo ? part.hard / r.more : 0.0f;
    auto smooth = [&](float v) {
      const float d = v - from;
      float g = row_exp2(d * scale.scale) * one;
      if constexpr (kTwo) g = fmaf(row_exp2(d * scale.second), two, g);
      return g;
    };
    const int now_y = y;
    const float now_logit = y_logit;
    if (keeps) {
      float kl = 0.0f;
      for (int i = lane; i < a.k; i += kLanes) {
        if (entries.at[i] < 0) continue;
        const float b = entries.value[i] - top, q = some != 0.0f ? row_exp2(b * hot_scale) / sum : 0.0f;
        if (!(q == 0.0f)) kl += q * ((b - (entries.logit[i] - from)) * hot_scale);
        const float mass = part.soft * q;
        entries.value[i] = mass;
        if (mass == 0.0f) entries.at[i] = -1;
      }
      kl = lanes_sum<kLanes>(kl);
      if (lane == 0 && t < T && share == 0) {
        if (a.ce)
          a.ce[t] = y < 0 ? 0.0f : r.s == 0.0f ? kRowInf : row_log2(kTwo ? r.more : r.s) * kRowLn2 - (y_logit - from);
        if (a.kl) a.kl[t] = some == 0.0f ? 0.0f : r.s == 0.0f ? kRowInf : (kl + row_log2(r.s) - row_log2(sum)) * kRowLn2;
      }
      wave_sync();
      mine = next_entry;
      y = next_y;
      logit = logit_of(t + step, lane, mine.at);
      y_logit = logit_of(t + step, a.k, y);
    }
    const E* following = row_of(t + step);
    if (!grad) {
      if constexpr (!kSplit) data.load(following, 0, C, at.g);
      continue;
    }
    E* dx = grad + (t < T ? t : T - 1) * ldd;
    const bool live = t < T;
    if (kWhole) {
#pragma unroll
      for (int i = 0; i < S::N; ++i) {
        data.store_chunk(i, dx, 0, full, at.g, live, any, smooth);
        data.load_chunk(i, following, 0, full, at.g);
      }
    } else {
      for (int first = begin; first < end; first += kSegment) {
#pragma unroll
        for (int i = 0; i < S::N; ++i) data.load_chunk(i, x, first, end, at.g);
#pragma unroll
        for (int i = 0; i < S::N; ++i)
          data.store_chunk(i, dx, first, end, at.g, live, any, smooth);
      }
      if constexpr (!kSplit) {
#pragma unroll
        for (int i = 0; i < S::N; ++i) data.load_chunk(i, following, 0, full, at.g);
      }
    }
    data.store_tail(dx, C, at.g, live && last, any, smooth);
    if constexpr (!kSplit) data.load_tail(following, C, at.g);
    RowPlace<S>::sync();  // the row is written before its entries are
    if (keeps && any && t < T) {
      const int from_class = begin * Data::V, to_class = last ? C : end * Data::V;
      auto here = [&](int c) { return c >= from_class && c < to_class; };
      const bool named = now_y >= 0 && part.hard != 0.0f, met = named && entries.add(lane, now_y, part.hard);
      entries.index(lane);
      entries.firsts(lane, [&](int i, float q) {
        if (here(entries.at[i])) dx[entries.at[i]] = static_cast<E>(smooth(entries.logit[i]) - q);
      });
      if (lane == 0 && named && !met && here(now_y)) dx[now_y] = static_cast<E>(smooth(now_logit) - part.hard);
    }
  }
}

}  // namespace lc

using namespace lc;

extern "C" lipcache_status lipcache_distill(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                            float temperature, float hard, float soft, int32_t k,
                                            const float* teacher, const int32_t* index, const int32_t* label,
                                            const float* weight, float* ce, float* kl, void* dx, int64_t lddx,
                                            void* ws, size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = row_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || (dx && lddx < C) || (T > 0 && k > 0 && (!teacher || !index))) return LIPCACHE_EINVAL;
  if (!(__builtin_fabsf(hard) < kRowInf) || !(__builtin_fabsf(soft) < kRowInf)) return LIPCACHE_EINVAL;
  if (row_unaligned(dx, dtype) || row_unaligned4(teacher) || row_unaligned4(index) || row_unaligned4(label) ||
      row_unaligned4(weight) || row_unaligned4(ce) || row_unaligned4(kl))
    return LIPCACHE_EINVAL;
  if (k > LIPCACHE_MOST_ENTRIES) return LIPCACHE_EUNSUPPORTED;
  if (T == 0) return LIPCACHE_OK;
  const RowShares shares = row_shares(T, C, dtype);
  if (const size_t need = row_share_bytes(T, k, shares); need > 0 && (!ws || !aligned256(ws) || ws_bytes < need))
    return LIPCACHE_EWORKSPACE;
  const int bits = entry_bits(C);
  // which sums there are: the label's at temperature 1, the teacher's at its own, one where they are the same
  const bool cold = label && (hard != 0.0f || ce), hot = k > 0 && (soft != 0.0f || kl);
  const bool two = cold && hot && temperature != 1.0f;
  const float at_one = kRowLog2e, at_own = kRowLog2e / temperature;
  const LpDistill a{temperature, hard, soft, hot ? at_own : at_one, at_one, label, weight, k,
                    teacher, index, ce, kl, bits};
  RowSplit split{shares, nullptr, nullptr};
  if (shares.count > 1) {
    RowSums* sums = static_cast<RowSums*>(ws);
    float* named = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(T * shares.count * sizeof(RowSums), 256));
    if (lipcache_status st = row_share_sums(x, ldx, T, C, dtype, two ? RowWants::kTwo : RowWants::kSum, RowScale{a.scale, a.second},
                                            shares, k, index, label, sums, named, stream);
        st != LIPCACHE_OK)
      return st;
    split.sums = sums;
    split.logits = named;
  }
  return row_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    auto run = [&](auto shape, auto whole, auto cut, unsigned blocks) {
      typedef decltype(shape) S;
      auto both = [&](auto with) {
        lp_distill_kernel<E, S, decltype(whole)::value, decltype(with)::value, decltype(cut)::value>
            <<<blocks, S::kThreads, S::kRows * entry_bytes(k, bits), stream>>>(static_cast<const E*>(x), ldx, T, C, a,
                                                                              static_cast<E*>(dx), lddx, split);
        return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
      };
      return two ? both(std::true_type{}) : both(std::false_type{});
    };
    if (shares.count > 1)
      return run(RowShape<256, 4>{}, std::false_type{}, std::true_type{}, static_cast<unsigned>(T * shares.count));
    // losses alone keep no row for a gradient: long ones go in segments by more workgroups of fewer registers (2048 x 131072
    // bfloat16 with two temperatures 117 us, 151 held; 1024 x 65536 float32 49, 61; 4096 x 32768 bfloat16 73, 72)
    if (!dx && C / RowType<E>::V > 8192)
      return run(RowShape<512, 4>{}, std::false_type{}, std::false_type{}, row_blocks<RowShape<512, 4>>(T));
    return row_shaped_entries<E>(T, C, k, [&](auto shape, auto whole) {
      return run(shape, whole, std::false_type{}, row_blocks<decltype(shape)>(T));
    });
  });
}

extern "C" size_t lipcache_distill_workspace_bytes(int64_t T, int32_t C, int32_t k, int32_t dtype) {
  return row_sizes_bad(T, C, k, dtype) ? 0 : row_share_bytes(T, k, row_shares(T, C, dtype));
}
