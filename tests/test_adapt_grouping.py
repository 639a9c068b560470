"""The arithmetic of grouping rows by pair (csrc/lc_group.hpp), run on the CPU in the kernel's order of work.

A host program walks the requests as the workgroups of the kernel do, with the same functions, and looks at every place:
whatever the offsets hold, each must get a row that exists."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_13144_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("clang++")
pytestmark = pytest.mark.skipif(CXX is None, reason="no host compiler")

PROGRAM = r"""
#include <stdint.h>
#include <stdio.h>
#include <vector>
#include "lc_group.hpp"
constexpr int kThreads = 1024, kRound = 2048;
int main(int argc, char** argv) {
  // in: T, S, R, wrap, offsets[R + 1], adapter[R]; out: order[T], pair[T] (-2: never written)
  FILE* f = fopen(argv[1], "rb");
  int64_t head[4];
  if (!f || fread(head, 8, 4, f) != 4) return 1;
  const int64_t T = head[0];
  const int S = head[1], R = head[2];
  const bool wrap = head[3];  // sums as plain 32-bit numbers, as a mistake would have them
  std::vector<int32_t> offsets(R + 1), adapter(R + 1), order(T, -2), pair(T, -2);
  if (fread(offsets.data(), 4, R + 1, f) != size_t(R + 1) || fread(adapter.data(), 4, R, f) != size_t(R)) return 1;
  fclose(f);
  const uint32_t all = T;
  auto add = [&](uint32_t a, uint32_t b) { return wrap ? a + b : lc::group_add(a, b, all); };
  auto request = [&](int i, uint32_t& lo, int& key) -> uint32_t {
    int64_t a = i >= 0 ? offsets[i < R ? i : R] : 0, b = i < R ? offsets[i + 1] : T;
    if (i > R) return 0;
    const lc::GroupRows rows = lc::group_clamp(a, b, 0, all);
    lo = rows.first;
    key = i >= 0 && i < R && adapter[i] >= 0 && adapter[i] < S ? adapter[i] : S;
    return rows.count;
  };
  std::vector<uint32_t> count(S + 1, 0);
  for (int i = -1; i <= R; ++i) {
    uint32_t lo = 0; int key = S;
    const uint32_t n = request(i, lo, key);
    count[key] += n;
  }
  std::vector<uint32_t> sums(kThreads), first(kRound), some(kThreads);
  uint64_t place0 = 0;
  for (int s = 0; s <= S; place0 += count[s++]) {
    uint64_t place = place0;
    for (int i0 = -1; i0 <= R && count[s] > 0 && place < all; i0 += kRound) {
      uint32_t before = 0;
      for (int t = 0; t < kThreads; ++t) {
        uint32_t n[2];
        for (int e = 0; e < 2; ++e) {
          uint32_t lo = 0; int key = S;
          const uint32_t rows = request(i0 + 2 * t + e, lo, key);
          n[e] = key == s ? rows : 0;
          first[2 * t + e] = lo;
        }
        some[t] = n[0];
        sums[t] = before = add(before, add(n[0], n[1]));
      }
      const uint32_t total = sums[kThreads - 1];
      const int64_t most = wrap ? int64_t(int32_t(total)) : int64_t(total);
      for (int64_t p = 0; p < most && place + p < all; ++p) {
        order[place + p] = lc::group_row(sums.data(), some.data(), first.data(), kThreads, p, all);
        pair[place + p] = s;
      }
      place += most > 0 ? most : 0;
    }
    if (s == S)
      for (uint64_t p = place; p < all; ++p) { order[p] = 0; pair[p] = S; }
  }
  f = fopen(argv[2], "wb");
  fwrite(order.data(), 4, T, f);
  fwrite(pair.data(), 4, T, f);
  fclose(f);
  return 0;
}
"""


@pytest.fixture(scope="module")
def group(tmp_path_factory):
    d = tmp_path_factory.mktemp("group")
    (d / "group.cpp").write_text(PROGRAM)
    subprocess.run([CXX, "-O2", "-std=c++17", f"-I{CSRC}", str(d / "group.cpp"), "-o", str(d / "group")], check=True)

    def run(T, S, offsets, adapter, wrap=False):
        offsets, adapter = np.asarray(offsets, dtype=np.int32), np.asarray(adapter, dtype=np.int32)
        with open(d / "in", "wb") as f:
            f.write(np.array([T, S, len(adapter), int(wrap)], dtype=np.int64).tobytes() + offsets.tobytes() + adapter.tobytes())
        subprocess.run([str(d / "group"), str(d / "in"), str(d / "out")], check=True, timeout=100)
        both = np.fromfile(d / "out", dtype=np.int32)
        return both[:T], both[T:]
    return run


@pytest.mark.parametrize("T,S,R", [(1, 1, 1), (37, 3, 5), (500, 7, 4100), (8300, 4, 60), (3000, 1, 2049)])
def test_batches_are_grouped_in_order(group, T, S, R):
    g = np.random.default_rng(T + R)
    for _ in range(4):
        offsets = np.sort(g.integers(-3, T + 4, R + 1))
        adapter = g.integers(-1, S + 1, R)
        order, pair = group(T, S, offsets, adapter)
        rows = np.full(T, S)
        for i in range(R):
            if 0 <= adapter[i] < S:
                rows[max(0, offsets[i]):max(0, offsets[i + 1])] = adapter[i]
        expect = np.argsort(rows, kind="stable")
        assert np.array_equal(order, expect) and np.array_equal(pair, rows[expect])


BIG = 1 << 21
DECREASING = {
    "up and down": (BIG, 1, np.tile([0, BIG], 1024), np.zeros(2047)),
    "two rounds": (BIG, 1, np.tile([0, BIG], 2050), np.zeros(4099)),
    "two pairs": (BIG + 5, 2, np.tile([0, BIG + 5], 1025), np.arange(2049) // 2 % 2),
    "none": (BIG, 2, np.tile([0, BIG], 1024), np.full(2047, -1)),
    "count of 2^32": (BIG, 3, np.tile([0, BIG], 2049), np.arange(4097) // 2 % 2 * 0),
    "extremes": (BIG, 2, np.tile([2 ** 31 - 1, -2 ** 31, 7], 700), np.arange(2099) % 2),
    "small": (400, 3, np.array([9, 3, 400, 0, 400, 2, 400]), np.arange(6) % 3),
}


@pytest.mark.parametrize("name", DECREASING)
def test_offsets_that_decrease_leave_no_place_out(group, name):
    T, S, offsets, adapter = DECREASING[name]
    order, pair = group(T, S, offsets, adapter)
    assert order.min() >= 0 and order.max() < T
    assert pair.min() >= 0 and pair.max() <= S


def test_sums_of_32_bits_would_leave_places_out(group):
    """What the sums that stop at T are for: the same walk with plain ones."""
    T, S, offsets, adapter = DECREASING["up and down"]
    order, _ = group(T, S, offsets, adapter, wrap=True)
    assert order.min() == -2
