// The sums of a row's shares, for few rows of many classes (lc_rows.hpp).
#include "lc_rows.hpp"

namespace lc {

// Bound by the latency of a share's few loads: one row of 131072 bfloat16, this launch and the gradient by shares 12 us (20 as
// one workgroup).
template <class E, RowWants W>
__global__ __launch_bounds__(256) void row_share_kernel(const E* __restrict__ logits, int64_t ldx, int C, RowScale scale,
                                                        RowShares shares, int k, const int32_t* __restrict__ index,
                                                        const int32_t* __restrict__ label, RowSums* __restrict__ sums,
                                                        float* __restrict__ named) {
  typedef RowShape<256, 4> S;
  typedef RowData<E, S> Data;
  constexpr int kSegment = S::G * S::N;
  __shared__ RowSums room[S::kWaves];
  const RowPlace<S> at;
  const int t = static_cast<int>(blockIdx.x) / shares.count, share = static_cast<int>(blockIdx.x) % shares.count;
  const E* x = logits + t * ldx;
  const int full = C / Data::V, begin = share * shares.each, end = begin + shares.each < full ? begin + shares.each : full;
  if (share == 0)
    for (int i = at.g; i <= k; i += S::G) {
      const int c = i < k ? index[static_cast<int64_t>(t) * k + i] : label ? label[t] : -1;
      named[static_cast<int64_t>(t) * (k + 1) + i] = c >= 0 && c < C ? static_cast<float>(x[c]) : 0.0f;
    }
  Data data(at.g);
  data.tail = -kRowInf;
  if (share == shares.count - 1) data.load_tail(x, C, at.g);
#pragma unroll
  for (int i = 0; i < S::N; ++i) data.load_chunk(i, x, begin, end, at.g);
  RowSums r = data.template begin<W>(scale);
  for (int first = begin; first < end; first += kSegment)
    data.template add<W>(first, end, at.g, r, scale, RowNothing{},
                         [&](int i) { data.load_chunk(i, x, first + kSegment, end, at.g); });
  row_join<S, W>(r, scale, room);
  if (at.g == 0) sums[blockIdx.x] = r;
}

lipcache_status row_share_sums(const void* x, int64_t ldx, int64_t T, int C, int32_t dtype, RowWants wants, RowScale scale,
                               RowShares shares, int k, const int32_t* index, const int32_t* label, RowSums* sums,
                               float* logits, hipStream_t s) {
  return row_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    auto run = [&](auto w) {
      row_share_kernel<E, decltype(w)::value><<<static_cast<unsigned>(T * shares.count), 256, 0, s>>>(
          static_cast<const E*>(x), ldx, C, scale, shares, k, index, label, sums, logits);
      return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
    };
    if (wants == RowWants::kSum) return run(std::integral_constant<RowWants, RowWants::kSum>{});
    if (wants == RowWants::kMean) return run(std::integral_constant<RowWants, RowWants::kMean>{});
    return run(std::integral_constant<RowWants, RowWants::kTwo>{});
  });
}

}  // namespace lc
