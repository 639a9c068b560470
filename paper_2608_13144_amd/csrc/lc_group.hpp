// The arithmetic of grouping rows by pair, apart from the kernel that uses it
// (constexpr, so the device takes it as it is and a host program can check it).
//
// T < 2^31 rows; offsets may be anything, so a round's rows are counted with
// sums that stop at T: in a valid batch they never reach past it, and whatever
// the offsets hold every place gets a row that exists.
#pragma once

#include <stdint.h>

namespace lc {

struct GroupRows {
  uint32_t first, count;  // from the first row of the chunk on
};

// The rows of [begin, end) among the T from t0 on.
constexpr GroupRows group_clamp(int64_t begin, int64_t end, int64_t t0, uint32_t T) {
  const int64_t last = t0 + T, lo = begin < t0 ? t0 : begin, hi = end > last ? last : end;
  return hi > lo ? GroupRows{static_cast<uint32_t>(lo - t0), static_cast<uint32_t>(hi - lo)} : GroupRows{0, 0};
}

// a, b <= T.  Associative, as a scan needs it.
constexpr uint32_t group_add(uint32_t a, uint32_t b, uint32_t T) { return a + b < T ? a + b : T; }

// The p-th row of a round.  Entry i has the rows first[2 i] .. + some[i] and those from first[2 i + 1] on; sums[i] is the number of
// rows of the entries up to i (p < sums[count - 1]).
constexpr uint32_t group_row(const uint32_t* sums, const uint32_t* some, const uint32_t* first, int count, uint32_t p, uint32_t T) {
  int a = 0, b = count - 1;  // the first entry whose sum passes p
  while (a < b) {
    const int mid = (a + b) >> 1;
    if (sums[mid] > p) b = mid; else a = mid + 1;
  }
  const uint32_t in = p - (a > 0 ? sums[a - 1] : 0);
  const uint32_t row = in < some[a] ? first[2 * a] + in : first[2 * a + 1] + (in - some[a]);
  return row < T ? row : 0;
}

}  // namespace lc
