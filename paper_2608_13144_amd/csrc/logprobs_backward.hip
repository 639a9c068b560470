// The gradient of log probabilities, sums, entropies and alternatives with
// regard to the logits (see lipcache.h for the formulas).
#include "lc_rows.hpp"

namespace lc {

struct LpBackward {
  float temperature;
  const int32_t* label;
  const float *g_logp, *g_lse, *g_entropy;
  int k;
  const int32_t* top_index;
  const float* g_top;
  int bits;  // of the entries' index
};

// What a row's elements share: dx = 2^a (flat + slope a), a the exponent to base 2.
struct LpSlope {
  float mass;  // gl - sum of the entries' gradients
  float ge;
  int some;    // any gradient that is not zero
};

// A row's sums, then dx = 2^a (flat + slope a) of every element from the same registers, then the places that label and
// alternatives name, each written once with all that it gets.  Bound by memory, with the vector pipe at 74 % where the
// entropy's gradient is wanted (two sums, about 23 instructions an element): 4096 x 32768 bfloat16 116 us with entropy
// and eight alternatives (4.6 TB/s), 109 without (4.9); float32 203 us (5.3 TB/s).  Rows too long for the registers are read
// twice: 1024 x 131072 float32 275 us.
// kSplit: a workgroup takes a share of a row whose sums are there already.
template <class E, class S, bool kWhole, bool kEntropy, bool kSplit>
__global__ __launch_bounds__(S::kThreads) void lp_backward_kernel(const E* logits, int64_t ldx, int64_t T, int C,
                                                                  LpBackward a, E* grad, int64_t ldd, RowSplit split) {
  static_assert(!kSplit || (!kWhole && S::kRows == 1), "a share goes in segments");
  typedef RowData<E, S> Data;
  constexpr RowWants kWants = kEntropy ? RowWants::kMean : RowWants::kSum;
  constexpr int kSegment = S::G * S::N, kLanes = S::kLanes;
  __shared__ RowSums room[S::kWaves];
  __shared__ LpSlope slope[S::kRows];
  extern __shared__ __align__(16) char lds[];
  const RowPlace<S> at;
  const int lane = at.g;  // (of the row's first wave, where it matters)
  const bool keeps = at.g < kLanes;
  RowEntries<kLanes> entries(lds + at.row * entry_bytes(a.k, a.bits), a.k, a.bits);
  const RowScale scale{kRowLog2e / a.temperature, 0.0f};
  const float inv_t = 1.0f / a.temperature;
  const int64_t step = kSplit ? T : static_cast<int64_t>(gridDim.x) * S::kRows;
  const int full = C / Data::V;
  const int share = kSplit ? static_cast<int>(blockIdx.x) % split.shares.count : 0;
  const bool last = !kSplit || share == split.shares.count - 1;
  const int begin = kSplit ? share * split.shares.each : 0, end = last ? full : begin + split.shares.each;
  auto row_of = [&](int64_t t) { return logits + (t < T ? t : T - 1) * ldx; };
  auto entry_of = [&](int64_t t, int i) {
    RowEntry e{-1, 0.0f};
    if (t < T && i < a.k) e = {a.top_index[t * a.k + i], a.g_top[t * a.k + i]};
    return e;
  };
  auto label_of = [&](int64_t t) {
    RowEntry e{-1, 0.0f};
    if (t < T && a.g_logp) e = {a.label[t], a.g_logp[t]};
    return e;
  };
  auto checked = [&](RowEntry e) {
    if (e.at < 0 || e.at >= C || e.value == 0.0f) e = {-1, 0.0f};
    return e;
  };
  // of entry i (a.k: the label), which names class c
  auto logit_of = [&](int64_t t, int i, int c) {
    if constexpr (kSplit) return t < T && i <= a.k ? split.logits[t * (a.k + 1) + i] : 0.0f;
    else return c >= 0 ? static_cast<float>(row_of(t)[c]) : 0.0f;
  };
  Data data(at.g);
  int64_t t = kSplit ? static_cast<int>(blockIdx.x) / split.shares.count : static_cast<int64_t>(blockIdx.x) * S::kRows + at.row;
  RowEntry mine{-1, 0.0f}, label{-1, 0.0f};
  float logit = 0.0f, label_logit = 0.0f;
  if (keeps) {
    mine = checked(entry_of(t, lane));
    label = checked(label_of(t));
    logit = logit_of(t, lane, mine.at);
    label_logit = logit_of(t, a.k, label.at);
  }
  if constexpr (!kSplit) data.load(row_of(t), 0, C, at.g);
  else data.load_tail(row_of(t), C, at.g);
  for (; t - at.row < T; t += step) {
    const E* x = row_of(t);
    E* dx = grad + (t < T ? t : T - 1) * ldd;
    RowEntry next_entry{-1, 0.0f}, next_label{-1, 0.0f};
    float gl = 0.0f, ge = 0.0f;
    if (keeps) {
      next_entry = entry_of(t + step, lane);
      next_label = label_of(t + step);
      if (a.g_lse && t < T) gl = a.g_lse[t];
      if (kEntropy && t < T) ge = a.g_entropy[t];
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
    next_entry = checked(next_entry);
    next_label = checked(next_label);
    if (keeps) {
      entries.keep(lane, mine, logit, [&](int i) { return checked(entry_of(t, i)); }, [&](int i, int c) { return logit_of(t, i, c); });
      float mass = 0.0f, any = gl != 0.0f || ge != 0.0f || label.value != 0.0f ? 1.0f : 0.0f;
      for (int i = lane; i < a.k; i += kLanes) {
        const float v = entries.value[i];
        mass += v;
        any = v != 0.0f ? 1.0f : any;
      }
      mass = lanes_sum<kLanes>(mass) + label.value;
      any = lanes_max<kLanes>(any);
      if (lane == 0) slope[at.row] = {gl - mass, ge, any != 0.0f ? 1 : 0};
      wave_sync();
    }
    row_join<S, kWants>(r, scale, room);
    const LpSlope k = slope[at.row];
    const bool some = k.some != 0 && r.s != 0.0f;  // (true for NaN)
    const float from = row_from(r.m), inv = inv_t / r.s, steep = kEntropy ? -k.ge * kRowLn2 * inv : 0.0f,
                flat = k.mass * inv - steep * (r.more / r.s);
    auto smooth = [&](float v) {
      const float e = (v - from) * scale.scale;
      if constexpr (kEntropy) return row_exp2(e) * fmaf(steep, fmaxf(e, kRowLeast), flat);
      else return row_exp2(e) * flat;
    };
    const bool live = t < T;
    const E* following = row_of(t + step);
    const RowEntry now = label;
    const float now_logit = label_logit;
    if (keeps) {
      mine = next_entry;
      label = next_label;
      logit = logit_of(t + step, lane, mine.at);
      label_logit = logit_of(t + step, a.k, label.at);
    }
    if (kWhole) {
#pragma unroll
      for (int i = 0; i < S::N; ++i) {
        data.store_chunk(i, dx, 0, full, at.g, live, some, smooth);
        data.load_chunk(i, following, 0, full, at.g);
      }
    } else {
      for (int first = begin; first < end; first += kSegment) {
#pragma unroll
        for (int i = 0; i < S::N; ++i) data.load_chunk(i, x, first, end, at.g);
#pragma unroll
        for (int i = 0; i < S::N; ++i)
          data.store_chunk(i, dx, first, end, at.g, live, some, smooth);
      }
      if constexpr (!kSplit) {
#pragma unroll
        for (int i = 0; i < S::N; ++i) data.load_chunk(i, following, 0, full, at.g);
      }
    }
    data.store_tail(dx, C, at.g, live && last, some, smooth);
    if constexpr (!kSplit) data.load_tail(following, C, at.g);
    RowPlace<S>::sync();  // the row is written before its entries are
    if (keeps && some && t < T) {
      const int from_class = begin * Data::V, to_class = last ? C : end * Data::V;
      auto here = [&](int c) { return c >= from_class && c < to_class; };
      const bool met = now.at >= 0 && entries.add(lane, now.at, now.value);
      entries.index(lane);
      entries.firsts(lane, [&](int i, float g) {
        if (here(entries.at[i])) dx[entries.at[i]] = static_cast<E>(fmaf(g, inv_t, smooth(entries.logit[i])));
      });
      if (lane == 0 && now.at >= 0 && !met && here(now.at)) dx[now.at] = static_cast<E>(fmaf(now.value, inv_t, smooth(now_logit)));
    }
  }
}

}  // namespace lc

using namespace lc;

extern "C" lipcache_status lipcache_logprobs_backward(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                                      float temperature, const int32_t* label, const float* g_logp,
                                                      const float* g_lse, const float* g_entropy, int32_t k,
                                                      const int32_t* top_index, const float* g_top, void* dx,
                                                      int64_t lddx, void* ws, size_t ws_bytes,
                                                      lipcache_stream_t stream) {
  if (lipcache_status st = row_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || lddx < C || (T > 0 && !dx) || (T > 0 && k > 0 && (!top_index || !g_top)) || (g_logp && !label))
    return LIPCACHE_EINVAL;
  if (row_unaligned(dx, dtype) || row_unaligned4(label) || row_unaligned4(g_logp) || row_unaligned4(g_lse) ||
      row_unaligned4(g_entropy) || row_unaligned4(top_index) || row_unaligned4(g_top))
    return LIPCACHE_EINVAL;
  if (k > LIPCACHE_MOST_ENTRIES) return LIPCACHE_EUNSUPPORTED;
  if (T == 0) return LIPCACHE_OK;
  const RowShares shares = row_shares(T, C, dtype);
  if (const size_t need = row_share_bytes(T, k, shares); need > 0 && (!ws || !aligned256(ws) || ws_bytes < need))
    return LIPCACHE_EWORKSPACE;
  const int bits = entry_bits(C);
  const LpBackward a{temperature, label, g_logp, g_lse, g_entropy, k, top_index, g_top, bits};
  const RowScale scale{kRowLog2e / temperature, 0.0f};
  RowSplit split{shares, nullptr, nullptr};
  if (shares.count > 1) {
    RowSums* sums = static_cast<RowSums*>(ws);
    float* named = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(T * shares.count * sizeof(RowSums), 256));
    if (lipcache_status st = row_share_sums(x, ldx, T, C, dtype, g_entropy ? RowWants::kMean : RowWants::kSum, scale, shares, k,
                                            top_index, label, sums, named, stream);
        st != LIPCACHE_OK)
      return st;
    split.sums = sums;
    split.logits = named;
  }
  return row_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    auto run = [&](auto shape, auto whole, auto cut, unsigned blocks) {
      typedef decltype(shape) S;
      auto entropy = [&](auto with) {
        lp_backward_kernel<E, S, decltype(whole)::value, decltype(with)::value, decltype(cut)::value>
            <<<blocks, S::kThreads, S::kRows * entry_bytes(k, bits), stream>>>(static_cast<const E*>(x), ldx, T, C, a,
                                                                              static_cast<E*>(dx), lddx, split);
        return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
      };
      return g_entropy ? entropy(std::true_type{}) : entropy(std::false_type{});
    };
    if (shares.count > 1)
      return run(RowShape<256, 4>{}, std::false_type{}, std::true_type{}, static_cast<unsigned>(T * shares.count));
    return row_shaped_entries<E>(T, C, k, [&](auto shape, auto whole) {
      return run(shape, whole, std::false_type{}, row_blocks<decltype(shape)>(T));
    });
  });
}

extern "C" size_t lipcache_logprobs_backward_workspace_bytes(int64_t T, int32_t C, int32_t k, int32_t dtype) {
  return row_sizes_bad(T, C, k, dtype) ? 0 : row_share_bytes(T, k, row_shares(T, C, dtype));
}
