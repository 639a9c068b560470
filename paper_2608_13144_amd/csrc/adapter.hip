// Low-rank adapters of many requests beside a shared projection, forward and
// backward (see lipcache.h for the formulas).
//
// Rows of one pair go together: a first kernel sorts the rows by their pair
// (stable, so every sum has one order), and everything after it works on
// sorted rows, gathered as they are read.  The low-rank part of the result
// joins the projection's sums in registers before they are stored, so y (dx)
// is written once.
//
// Rows of one output tile may belong to several pairs.  Each pair multiplies
// only its own rows and adds only to them by selection, never by a product
// with zero: what one request's pair or rows hold that is not finite stays
// with it.
#include <type_traits>

#include "lc_common.hpp"
#include "lc_group.hpp"
#include "lc_mfma.hpp"

namespace lc {

constexpr int kAdMaxRank = 128;
constexpr int kAdMaxPairs = 8192;
constexpr int kAdMaxRequests = 1 << 30;
constexpr int64_t kAdMaxWidth = 1 << 20;
constexpr int kThinRows = 32;  // sorted rows of one pair that a workgroup of the thin products takes

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// A launch holds fewer than 2^32 threads.  Kernels whose workgroups may be more take the first one's number, a pass after another.
constexpr int64_t kMostBlocks = 1 << 23;
template <class F>
lipcache_status in_passes(int64_t blocks, F launch) {
  for (int64_t first = 0; first < blocks; first += kMostBlocks) {
    launch(first, static_cast<unsigned>(blocks - first < kMostBlocks ? blocks - first : kMostBlocks));
    LC_LAUNCHED();
  }
  return LIPCACHE_OK;
}

// ---------------------------------------------------------------- grouping
// Rows sorted by pair (rows without one last), and the table of the thin
// products' tiles: up to kThinRows sorted rows of one pair each.
struct AdGroups {
  int32_t* order;      // [T] sorted place -> row
  int32_t* pair;       // [T] sorted place -> pair, S where none
  int32_t* start;      // [S + 2] first place of each pair, of none, and T
  int32_t* tile_pair;  // [tiles]
  int32_t* tile_row;   // [tiles] first sorted place
  int32_t* tile_rows;  // [tiles] rows
  int32_t* tile_start; // [S + 1] first tile of each pair, and the number of tiles
  uint32_t* zeros;     // 16 bytes of zero
};

__host__ __device__ inline int64_t ad_tiles(int64_t T, int S) { return T / kThinRows + (S < T ? S : T); }

constexpr int kGroupThreads = 1024;
constexpr int kGroupRound = 2 * kGroupThreads;  // requests that the workgroup takes at a time

// Inclusive sums over the workgroup's threads, at most T, in LDS (`sums`, one word a
// thread; `waves`, one a wave).  Ends with a barrier.
__device__ __forceinline__ void group_scan(uint32_t v, uint32_t T, uint32_t* sums, uint32_t* waves) {
  const int tid = static_cast<int>(threadIdx.x), lane = lane_id(), wave = tid / kWave;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t u = __shfl_up(v, o, kWave);
    if (lane >= o) v = group_add(v, u, T);
  }
  if (lane == kWave - 1) waves[wave] = v;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < kGroupThreads / kWave; ++w) before = group_add(before, w < wave ? waves[w] : 0, T);
  sums[tid] = group_add(before, v, T);
  __syncthreads();
}

// Workgroup s places the rows of pair s.  Every workgroup counts all pairs'
// rows (integer sums in LDS: any order gives the same), then walks the
// requests in order, 2048 at a time, two neighbours a thread (whose loads go
// out together).  Request -1 is the rows before the first offset, request R
// those after the last.  Offsets that decrease place rows
// wrongly or not at all: counts may wrap and pairs' places overlap, but a pair fills at least the places up to the next one's
// first, the last workgroup the rest, with rows below T (sums stop there), so whatever they are no access leaves the arrays.  Bound
// by latency (one round of loads, then scans and a search in LDS): 6 us for 64 pairs and 1024 requests, 9 us for four
// pairs of 2048 rows each.
__global__ __launch_bounds__(kGroupThreads) void ad_group_kernel(int64_t t0, int T, const int32_t* __restrict__ offsets,
                                                                 const int32_t* __restrict__ adapter, int R, int S,
                                                                 AdGroups g) {
  extern __shared__ uint32_t count[];       // [S + 1] rows of each pair, then scratch
  uint32_t* sums = count + S + 1;           // [kGroupThreads]
  uint32_t* first = sums + kGroupThreads;   // [kGroupRound]
  uint32_t* some = first + kGroupRound;     // [kGroupThreads] rows of a thread's first request
  uint32_t* waves = some + kGroupThreads;   // [kGroupThreads / kWave]
  __shared__ unsigned long long base_rows, base_tiles;
  const int tid = static_cast<int>(threadIdx.x), s = static_cast<int>(blockIdx.x);
  const uint32_t all = static_cast<uint32_t>(T), last = static_cast<uint32_t>(ad_tiles(T, S));
  // rows of request i >= -1 (none past R).  Three loads that wait for nothing, least of all each other.
  auto request = [&](int i, uint32_t& lo, int& key) {
    int64_t a = t0, b = t0 + T;
    int p = -1;
    if (R > 0) {
      const int at = i < 0 ? 0 : i < R ? i : R, next = i + 1 < R ? i + 1 : R;
      const int32_t begin = offsets[at], end = offsets[next], named = adapter[at < R ? at : R - 1];
      if (i >= 0) a = begin;
      if (i < R) b = end;
      if (i >= 0 && i < R) p = named;
    } else if (i < 0) {
      b = t0;
    }
    const GroupRows rows = group_clamp(a, b, t0, all);
    lo = rows.first;
    key = p >= 0 && p < S ? p : S;
    return i <= R ? rows.count : 0;
  };
  int key[2];
  uint32_t lo[2], n[2];  // this thread's requests among the first 2048
#pragma unroll
  for (int e = 0; e < 2; ++e) n[e] = request(2 * tid + e - 1, lo[e], key[e]);
  for (int i = tid; i <= S; i += kGroupThreads) count[i] = 0;
  if (tid == 0) base_rows = base_tiles = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (n[e] > 0) atomicAdd(&count[key[e]], n[e]);
  for (int i = tid - 1 + kGroupRound; i <= R; i += kGroupThreads) {
    int k;
    uint32_t l;
    const uint32_t rows = request(i, l, k);
    if (rows > 0) atomicAdd(&count[k], rows);
  }
  __syncthreads();
  unsigned long long rows = 0, tiles = 0;
  for (int i = tid; i < s; i += kGroupThreads) {
    const uint32_t n = count[i];
    rows += n;
    tiles += ((n < all ? n : all) + kThinRows - 1) / kThinRows;  // as many as the pair writes below
  }
  if (uniform(tid / kWave) * kWave < s) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      rows += __shfl_xor(rows, o, kWave);
      tiles += __shfl_xor(tiles, o, kWave);
    }
    if (lane_id() == 0 && rows > 0) {
      atomicAdd(&base_rows, rows);
      atomicAdd(&base_tiles, tiles);
    }
  }
  __syncthreads();
  const uint64_t place0 = base_rows;
  const uint32_t mine = count[s];
  if (tid == 0) {
    g.start[s] = static_cast<int32_t>(place0 < all ? place0 : all);
    g.tile_start[s] = static_cast<int32_t>(base_tiles < last ? base_tiles : last);
    if (s == S) g.start[S + 1] = T;
  }
  if (s == S && tid < 4) g.zeros[tid] = 0;
  if (s < S) {
    for (uint64_t i = tid; i * kThinRows < (mine < all ? mine : all); i += kGroupThreads) {
      const uint64_t at = base_tiles + i, row = place0 + i * kThinRows;
      if (at < last) {
        g.tile_pair[at] = s;
        g.tile_row[at] = static_cast<int32_t>(row < all ? row : all);
        const uint64_t end = place0 + mine < all ? place0 + mine : all, left = row < end ? end - row : 0;
        g.tile_rows[at] = static_cast<int32_t>(left < kThinRows ? left : kThinRows);
      }
    }
  }
  uint64_t place = place0;
  for (int i0 = -1; i0 <= R && mine > 0 && place < all; i0 += kGroupRound) {
    if (i0 >= 0) {
#pragma unroll
      for (int e = 0; e < 2; ++e) n[e] = request(i0 + 2 * tid + e, lo[e], key[e]);
      __syncthreads();  // the last round's readers are done
    }
    const uint32_t n0 = key[0] == s ? n[0] : 0, n1 = key[1] == s ? n[1] : 0;
    first[2 * tid] = lo[0];
    first[2 * tid + 1] = lo[1];
    some[tid] = n0;
    group_scan(group_add(n0, n1, all), all, sums, waves);
    const uint32_t total = sums[kGroupThreads - 1];
    for (uint32_t p = tid; p < total && place + p < all; p += kGroupThreads) {
      g.order[place + p] = static_cast<int32_t>(group_row(sums, some, first, kGroupThreads, p, all));
      g.pair[place + p] = s;
    }
    place += total;
  }
  if (s == S)
    for (uint64_t p = place + tid; p < all; p += kGroupThreads) {
      g.order[p] = 0;
      g.pair[p] = S;
    }
}

// ------------------------------------------------------------ element types
template <class E>
struct Vec16;  // 16 bytes of elements
template <>
struct Vec16<float> {
  static constexpr int kCount = 4;
  typedef f32x4 type;
};
template <>
struct Vec16<__bf16> {
  static constexpr int kCount = 8;
  typedef bf16x8 type;
};
template <>
struct Vec16<_Float16> {
  static constexpr int kCount = 8;
  typedef f16x8 type;
};

// A matrix whose rows are read as 16-byte vectors: itself, or its copy in the workspace.
template <class E>
struct AdRows {
  const E* p;
  int64_t ld;
};

// A float32 factor as what the matrix cores take: itself, or a sum of 16-bit
// numbers, an instruction each: three bfloat16 (all 24 bits) or two float16 (22).
// What is not finite, or rounds to infinity, is the first part alone.
template <class E>
inline constexpr int kFactorParts = std::is_same_v<E, float> ? 1 : std::is_same_v<E, __bf16> ? 3 : 2;
template <class E>
__device__ __forceinline__ void factor_parts(float v, E (&part)[kFactorParts<E>]) {
#pragma unroll
  for (int h = 0; h < kFactorParts<E>; ++h) {
    asm("" : "+v"(v));
    part[h] = static_cast<E>(v);
    v -= static_cast<float>(part[h]);
    v = fabsf(v) < __builtin_huge_valf() ? v : 0.0f;
  }
}

// float16 ends at 65504 and loses digits below 2^-14, where A_a x and B_a^T dy
// may lie (gradients of a mean over many rows, outliers of a wide sum).  Such
// factors go to the matrix cores times 2^e, which brings the largest finite one
// of a row (in the pairs' gradients, of a tile) to [2^14, 2^15), and what comes out is taken back by 2^-e in float32.
// Rows keep exponents of their own, so that one request's size costs another's rows no digits.
// bfloat16 has float32's range and takes them as they are.
template <class E>
inline constexpr bool kScaledFactors = std::is_same_v<E, _Float16>;
__device__ __forceinline__ float finite_size(float v) {
  const float a = fabsf(v);
  return a < __builtin_huge_valf() ? a : 0.0f;
}
__device__ __forceinline__ int factor_exponent(float peak) {  // of a peak > 0
  return 15 - __builtin_amdgcn_frexp_expf(peak);
}
template <class E>
__device__ __forceinline__ float two_to(float v, int e) {
  if constexpr (kScaledFactors<E>) return __builtin_amdgcn_ldexpf(v, e);
  else return v;
}

// ------------------------------------------------------- copies and transposes
// Matrices moved into the workspace: padded with zeros to a width of whole
// 16-byte vectors, as they are or transposed; all of a call in one launch.
struct AdCopy {
  const void* from;
  void* to;
  int64_t ld_from, ld_to;     // elements
  int64_t from_next, to_next; // elements between matrices of a stack
  int rows, width;            // of the source
  int to_rows, to_width;      // written, zeros outside the source
  int stack;
  int transpose;
};
constexpr int kAdCopies = 6;
struct AdCopies {
  AdCopy c[kAdCopies];
  int64_t end[kAdCopies];  // first workgroup past each (none of a copy that is not there)
};

template <typename T>
__global__ __launch_bounds__(256) void ad_copy_kernel(AdCopies all, int64_t first) {
  __shared__ T tile[32][33];
  const int x = static_cast<int>(threadIdx.x) & 31, y = static_cast<int>(threadIdx.x) >> 5;
  const int64_t number = first + blockIdx.x;
  int64_t block = number;
  AdCopy c = all.c[0];
#pragma unroll
  for (int i = 1; i < kAdCopies; ++i)
    if (number >= all.end[i - 1]) {
      c = all.c[i];
      block = number - all.end[i - 1];
    }
  // tiles of the result
  const int64_t tiles_w = ceil_div(c.to_width, 32), tiles = tiles_w * ceil_div(c.to_rows, 32);
  const int64_t z = block / tiles, t = block % tiles;
  const int64_t i0 = t / tiles_w * 32;
  const int j0 = static_cast<int>(t % tiles_w) * 32;
  const T* from = static_cast<const T*>(c.from) + z * c.from_next;
  T* to = static_cast<T*>(c.to) + z * c.to_next;
  if (c.transpose) {
#pragma unroll
    for (int k = y; k < 32; k += 8) {
      const int row = j0 + k;  // of the source
      const int64_t col = i0 + x;
      tile[k][x] = row < c.rows && col < c.width ? from[row * c.ld_from + col] : static_cast<T>(0.0f);
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = y; k < 32; k += 8) {
    const int64_t row = i0 + k;
    const int col = j0 + x;
    if (row >= c.to_rows || col >= c.to_width) continue;
    T v;
    if (c.transpose) v = tile[x][k];
    else v = row < c.rows && col < c.width ? from[row * c.ld_from + col] : static_cast<T>(0.0f);
    to[row * c.ld_to + col] = v;
  }
}

struct AdCopyList {
  AdCopies all{};
  int count = 0;
  int64_t blocks = 0;
  void add(const AdCopy& c) {
    const int64_t n = ceil_div(c.to_width, 32) * ceil_div(c.to_rows, 32) * c.stack;
    if (n <= 0) return;
    blocks += n;
    all.c[count] = c;
    for (int i = count++; i < kAdCopies; ++i) all.end[i] = blocks;
  }
  template <typename T>
  lipcache_status launch(hipStream_t s) const {
    return in_passes(blocks, [&](int64_t first, unsigned n) { ad_copy_kernel<T><<<n, 256, 0, s>>>(all, first); });
  }
};

// ------------------------------------------------------------ thin products
// out[row][rho] = F_a[rho] . x[row] for the up to 32 sorted rows of one tile
// of the table (F is [S][r][ldf]), the contraction shared by four waves.  The
// workgroups past the table write zeros to the rows without a pair.  peak[row]
// (or NULL): the largest finite |out| of a row with one.  Bound by reading x
// once, and F_a once a tile: 8192 rows of 4096 bf16, rank 32, 24 us (2.8 TB/s
// of x); short batches by three dependent rounds of loads, 7 us (float16, with the rows' largest values, 12).
template <class S>
__global__ __launch_bounds__(S::kThreads) void ad_thin_kernel(const typename S::E* __restrict__ x, int64_t ldx, int width,
                                                              const typename S::E* __restrict__ F, int64_t ldf, int r,
                                                              int pairs, int T, AdGroups g, float* __restrict__ out,
                                                              float* __restrict__ peak) {
  typedef typename S::E E;
  __shared__ __align__(16) char lds[S::kLds];
  const int t = static_cast<int>(blockIdx.x), table = static_cast<int>(ad_tiles(T, pairs));
  if (t >= table) {
    const int first = g.start[pairs];
    const int64_t all = static_cast<int64_t>(T - first) * r, step = static_cast<int64_t>(gridDim.x - table) * S::kThreads;
    for (int64_t i = static_cast<int64_t>(t - table) * S::kThreads + threadIdx.x; i < all; i += step)
      out[static_cast<int64_t>(g.order[first + i / r]) * r + i % r] = 0.0f;
    return;
  }
  // together: past the last tile they are not used
  const int last = g.tile_start[pairs], a = g.tile_pair[t], row0 = g.tile_row[t], rows = g.tile_rows[t];
  if (static_cast<uint32_t>(t) >= static_cast<uint32_t>(last) || rows <= 0) return;
  Side p{}, q{};
  p.p = x;
  p.ld = ldx * sizeof(E);
  p.rows = rows;
  p.pick = g.order + row0;
  q.p = F + static_cast<int64_t>(a) * r * ldf;
  q.ld = ldf * sizeof(E);
  q.rows = r;
  f32x16 acc[S::TM][S::TN] = {};
  tile_products<S>(p, q, width, lds, acc);
  float size[16] = {};
  tile_store<S>(acc, [&](int i, int j, const f32x16& v) {
    if (j >= r) return;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (i + acc_row(e) < rows) out[static_cast<int64_t>(g.order[row0 + i + acc_row(e)]) * r + j] = v[e];
      if constexpr (kScaledFactors<E>) size[e] = fmaxf(size[e], finite_size(v[e]));
    }
  });
  if constexpr (kScaledFactors<E>) {
    // each lane has a column of 16 rows: halve the rows and double the columns, four times
    if (!peak || threadIdx.x >= kWave) return;  // the first wave has the sums
    const int lane = lane_id();
#pragma unroll
    for (int b = 0, n = 8; b < 4; ++b, n >>= 1)
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const bool upper = (lane >> b & 1) != 0;
        const float mine = upper ? size[e + n] : size[e], other = upper ? size[e] : size[e + n];
        size[e] = fmaxf(mine, __shfl_xor(other, 1 << b, kWave));
      }
    const float top = fmaxf(size[0], __shfl_xor(size[0], 16, kWave));
    const int e = (lane & 1) << 3 | (lane & 2) << 1 | (lane & 4) >> 1 | (lane & 8) >> 3;
    const int i = acc_row(e) + 4 * (lane >> 5);
    if ((lane & 16) == 0 && i < rows) peak[g.order[row0 + i]] = top;
  }
}

// ------------------------------------------------------------- main product
// The fragment (one 16-byte vector) of lane's row or column from `p`, the
// `count` valid elements of which start at p (others 0); whole vectors where `wide`.
template <class E>
__device__ __forceinline__ typename Vec16<E>::type load_some(const E* p, int count, bool wide) {
  typedef typename Vec16<E>::type V;
  constexpr int kV = Vec16<E>::kCount;
  if (wide && count >= kV) return *reinterpret_cast<const V*>(p);
  V v{};
#pragma unroll
  for (int e = 0; e < kV; ++e)
    if (e < count) v[e] = p[e];
  return v;
}

struct AdLow {
  const void* F;       // [S][width][ldf]: B (forward) or A transposed (backward)
  int64_t ldf;         // elements between its rows
  const float* v;      // [T][r]
  const float* peak;   // [T]: the thin product's (float16 only)
  const float* scale;  // [S]
  int r, S, width;
  int wide;            // F's rows and r allow whole vectors
  int wide_v;          // v's
};

// The rows of a wave's accumulators: lane l has row l % 32 of each 32, loaded before the main loop.
template <class S>
struct AdTileRows {
  int pair[S::TM], row[S::TM];
  float peak[S::TM], scale[S::TM];
  __device__ __forceinline__ void load(const AdGroups& g, const AdLow& low, int i0, int rows) {
    const int wave = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int wm = wave % (S::WM * S::WN) / S::WN;
#pragma unroll
    for (int tm = 0; tm < S::TM; ++tm) {
      const int i = (wm * S::TM + tm) * 32 + (lane_id() & 31);
      const bool in = i < rows;
      pair[tm] = in ? g.pair[i0 + i] : low.S;
      row[tm] = g.order[i0 + (in ? i : 0)];
      scale[tm] = pair[tm] < low.S ? low.scale[pair[tm]] : 0.0f;
      if constexpr (kScaledFactors<typename S::E>) peak[tm] = pair[tm] < low.S ? low.peak[row[tm]] : 0.0f;
    }
  }
};

// acc += scale_a F_a v for the tile's rows of every pair among them: one pair
// of a 32-row accumulator at a time, its rows a mask.
template <class S, class E>
__device__ __forceinline__ void add_low_rank(const AdLow& low, const AdTileRows<S>& rows, int j0,
                                             f32x16 (&acc)[S::TM][S::TN]) {
  constexpr int kV = Vec16<E>::kCount;
  typedef typename Vec16<E>::type V;
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int wn = wave % S::WN;
  const int li = lane & 31, half = lane >> 5;
  const E* F = static_cast<const E*>(low.F);
#pragma unroll
  for (int tm = 0; tm < S::TM; ++tm) {
    uint32_t todo = static_cast<uint32_t>(__ballot(rows.pair[tm] < low.S));
    const float* v = low.v + static_cast<int64_t>(rows.row[tm]) * low.r;
    while (todo) {
      const int a = __builtin_amdgcn_readlane(rows.pair[tm], __builtin_ctz(todo));
      const bool mine = rows.pair[tm] == a;
      const uint32_t mask = static_cast<uint32_t>(__ballot(mine));
      todo &= ~mask;
      const float scale = rows.scale[tm];  // of this lane's row: its own where `mine`
      int up = 0, up_of[16];  // of this lane's row; of the accumulators' rows
      if constexpr (kScaledFactors<E>) {
        const float top = mine ? finite_size(scale * rows.peak[tm]) : 0.0f;
        up = top > 0.0f ? factor_exponent(top) : 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) up_of[e] = __shfl(up, acc_row(e) + 4 * half, kWave);
      }
#pragma unroll
      for (int tn = 0; tn < S::TN; ++tn) {
        const int j = j0 + (wn * S::TN + tn) * 32 + li;
        const E* f = F + (static_cast<int64_t>(a) * low.width + (j < low.width ? j : low.width - 1)) * low.ldf;
        f32x16 sum = {};
#pragma unroll 1
        for (int k = 0; k < low.r; k += 2 * kV) {
          const int at_k = k + half * kV, left = low.r - at_k;
          const V vf = load_some<E>(f + at_k, left, low.wide != 0);
          float w[kV];
#pragma unroll
          for (int e = 0; e < kV; e += 4) {
            const f32x4 u = load_some<float>(v + at_k + e, mine ? left - e : 0, low.wide_v != 0);
#pragma unroll
            for (int o = 0; o < 4; ++o) w[e + o] = mine ? two_to<E>(scale * u[o], up) : 0.0f;
          }
          if constexpr (std::is_same_v<E, float>) {
            sum = MfmaType<E>::mul(V{w[0], w[1], w[2], w[3]}, vf, sum);
          } else {
            V part[kFactorParts<E>];
#pragma unroll
            for (int e = 0; e < kV; ++e) {
              E p[kFactorParts<E>];
              factor_parts(w[e], p);
#pragma unroll
              for (int h = 0; h < kFactorParts<E>; ++h) part[h][e] = p[h];
            }
#pragma unroll
            for (int h = kFactorParts<E> - 1; h >= 0; --h) sum = MfmaType<E>::mul(part[h], vf, sum);
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (mask >> (acc_row(e) + 4 * half) & 1) acc[tm][tn][e] += two_to<E>(sum[e], kScaledFactors<E> ? -up_of[e] : 0);
      }
    }
  }
}

// out[row] = P[row] Q^T + bias + the low-rank part, for the sorted rows of this tile.  Bound by the matrix cores: 8192
// x 4096 -> 8192 bf16 with rank 64 590 to 615 us (0.93 PFLOP/s), 4096 -> 4096 backward 280 us (0.98).
template <class S>
__global__ __launch_bounds__(S::kThreads) void ad_main_kernel(const typename S::E* __restrict__ P, int64_t ldp,
                                                              const typename S::E* __restrict__ Q, int64_t ldq, int T,
                                                              int width, int K, const float* __restrict__ bias,
                                                              AdLow low, AdGroups g, typename S::E* __restrict__ out,
                                                              int64_t ldo) {
  typedef typename S::E E;
  __shared__ __align__(16) char lds[S::kLds];
  int bi, bj;
  tile_of(static_cast<int>(ceil_div(T, S::BM)), static_cast<int>(ceil_div(width, S::BN)), bi, bj);
  const int i0 = bi * S::BM, j0 = bj * S::BN;
  Side p{}, q{};
  p.p = P;
  p.ld = ldp * sizeof(E);
  p.rows = T - i0 < S::BM ? T - i0 : S::BM;
  p.pick = g.order + i0;
  q.p = Q + (S::QCOL ? static_cast<int64_t>(j0) : j0 * ldq);
  q.ld = ldq * sizeof(E);
  q.rows = width - j0 < S::BN ? width - j0 : S::BN;
  AdTileRows<S> rows;
  rows.load(g, low, i0, p.rows);
  f32x16 acc[S::TM][S::TN] = {};
  tile_products<S>(p, q, K, lds, acc);
  if (S::WK > 1 && static_cast<int>(threadIdx.x) / kWave >= S::WM * S::WN) return;  // their sums are added
  add_low_rank<S, E>(low, rows, j0, acc);
  tile_store<S>(acc, [&](int i, int j, const f32x16& v) {
    j += j0;
    if (j >= width) return;
    const float b = bias ? bias[j] : 0.0f;
    int row[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) row[e] = g.order[i0 + (i + acc_row(e) < p.rows ? i + acc_row(e) : p.rows - 1)];
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (i + acc_row(e) < p.rows) out[row[e] * ldo + j] = static_cast<E>(v[e] + b);
  });
}

// Tile size by the number of 128 x 128 tiles, as the CUs fill (256 of them).
template <class E, bool kCol>
lipcache_status ad_main(const void* P, int64_t ldp, const void* Q, int64_t ldq, int T, int width, int K,
                        const float* bias, const AdLow& low, const AdGroups& g, void* out, int64_t ldo, hipStream_t s) {
  auto run = [&](auto shape) {
    typedef decltype(shape) S;
    const int64_t tiles = ceil_div(T, S::BM) * ceil_div(width, S::BN);
    ad_main_kernel<S><<<static_cast<unsigned>(tiles), S::kThreads, 0, s>>>(
        static_cast<const E*>(P), ldp, static_cast<const E*>(Q), ldq, T, width, K, bias, low, g, static_cast<E*>(out), ldo);
    return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
  };
  const int64_t t128 = ceil_div(T, 128) * ceil_div(width, 128), t256 = ceil_div(T, 256) * ceil_div(width, 256);
  // float32 products of one wave's 32 x 32 tile take 3.4 us at K = 256: two waves share them where workgroups are few
  // (1024 x 256 -> 200: 13.0 -> 10.9 us; with 256 tiles of 64 x 64 the larger tile is ahead, 12.4 to 14.0)
  if constexpr (sizeof(E) == 4)
    if (ceil_div(T, 64) * ceil_div(width, 64) <= 128) return run(TileShape<E, 32, 64, 1, 2, 2, 4, 1, false, kCol>{});
  if (t128 < 128) return run(TileShape<E, 64, 64, 2, 2, 1, 3, 1, false, kCol>{});
  if constexpr (sizeof(E) == 2)
    if (5 * t256 >= 4 * 256 * ceil_div(t256, 256)) return run(TileShape<E, 256, 256, 2, 4, 1, 2, 1, false, kCol>{});
  if (t128 < 320) return run(TileShape<E, 128, 128, 2, 4, 1, 4, 1, false, kCol>{});
  return run(TileShape<E, 128, 128, 2, 2, 1, 2, 1, false, kCol>{});
}

// ------------------------------------------------------------- few rows
// A decode batch is bound by reading W once, a batch of single queries of a
// small head by launches.  Neither is sorted.  One launch does two independent
// things: some workgroups multiply a tile of rows with 64 rows of W over a share
// of the contraction each (so that W comes through all CUs, and x in shares), the
// others find each row's pair and A_a x, a wave a row and one or four ranks.  A
// second launch adds the shares in order, the bias and scale_a B_a v, a dot
// product of r an output.  32 MiB of W: 8 us for one row, where one launch after
// another took 13.
constexpr int kFewRows = 64;

// Up to 64 rows always; up to 8192 where what every row reads of its pair for itself (sorted rows share it) and the
// projection's float32 sums stay below 60 MiB.  In us, few against sorted: 1024 x 256 -> 200 (float32, rank 8, 16 MiB)
// 9 to 22, 128 x 4096 -> 4096 (bf16, rank 16, 36 MiB) 20 to 41, 256 x 4096 -> 4096 (rank 8, 40 MiB) 30 to 40, 4096 x 256
// -> 200 (bf16, rank 16, 63 MiB) 24 to 23, 8192 x 64 -> 64 (float32, rank 16, 68 MiB) 37 to 29, 512 x 4096 -> 4096 (bf16,
// rank 8, 80 MiB) 52 to 52, 1024 x 1024 -> 1024 (bf16, rank 64, 264 MiB) 55 to 30.
inline bool few_rows(int64_t T, int64_t K, int64_t N, int r, size_t size) {
  if (T <= kFewRows) return true;
  const int64_t e = static_cast<int64_t>(size);
  return T <= 8192 && T * (r * K * e + N * (r * e + 8)) <= (60 << 20);
}

// The pair of row t (-1: none), by the whole wave: 64 offsets a round.
__device__ __forceinline__ int pair_of_row(int64_t t, const int32_t* __restrict__ offsets,
                                           const int32_t* __restrict__ adapter, int R, int S) {
  int lo = 0, n = R + 1;  // the first offset past t lies in [lo, lo + n]
  while (n > 0) {
    const int step = (n + kWave - 1) / kWave, at = lo + (lane_id() + 1) * step - 1;
    const bool before = at < lo + n && offsets[at] <= t;
    const int passed = __builtin_popcountll(__ballot(before));
    lo += passed * step;
    n = step > 1 ? (n - passed * step < step ? n - passed * step : step - 1) : 0;
  }
  if (lo < 1 || lo > R) return -1;
  const int a = adapter[lo - 1];
  return a >= 0 && a < S ? a : -1;
}

// A_a x of a row at kRanks ranks, by one wave.
template <class E, int kRanks>
__device__ __forceinline__ void few_low(int w, const E* __restrict__ x, int64_t ldx, int K, const E* __restrict__ A,
                                        int64_t lda, const lipcache_adapters& ad, int32_t* __restrict__ pair,
                                        float* __restrict__ v) {
  constexpr int kV = Vec16<E>::kCount;
  typedef typename Vec16<E>::type V;
  const int groups = (ad.r + kRanks - 1) / kRanks;
  const int t = w / groups, rho = w % groups * kRanks, lane = lane_id();
  const int a = ad.R > 0 ? uniform(pair_of_row(t, ad.offsets, ad.adapter, ad.R, ad.S)) : -1;
  float sum[kRanks] = {};
  if (a >= 0) {
    const E* px = x + t * ldx;
    const E* pa[kRanks];
#pragma unroll
    for (int i = 0; i < kRanks; ++i)
      pa[i] = A + (static_cast<int64_t>(a) * ad.r + (rho + i < ad.r ? rho + i : ad.r - 1)) * lda;
#pragma unroll(kRanks > 1 ? 2 : 4)
    for (int k = lane * kV; k < K; k += kWave * kV) {
      const V vx = *reinterpret_cast<const V*>(px + k);
#pragma unroll
      for (int i = 0; i < kRanks; ++i) {
        const V va = *reinterpret_cast<const V*>(pa[i] + k);
#pragma unroll
        for (int e = 0; e < kV; ++e)
          sum[i] = fmaf(k + e < K ? static_cast<float>(vx[e]) : 0.0f, k + e < K ? static_cast<float>(va[e]) : 0.0f, sum[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRanks; ++i) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum[i] += __shfl_xor(sum[i], o, kWave);
    if (lane == 0 && rho + i < ad.r) v[static_cast<int64_t>(t) * ad.r + rho + i] = sum[i];
  }
  if (lane == 0 && rho == 0) pair[t] = a;
}

// The first `products` workgroups: part[share][t][j] of the projection; the others: v and the pairs.
template <class S, int kRanks>
__global__ __launch_bounds__(S::kThreads) void ad_few_kernel(const typename S::E* __restrict__ x, int64_t ldx, int T,
                                                             const typename S::E* __restrict__ W, int64_t ldw, int K,
                                                             int N, int row_tiles, int tiles, int products, int each,
                                                             float* __restrict__ part,
                                                             const typename S::E* __restrict__ A, int64_t lda,
                                                             lipcache_adapters ad, int32_t* __restrict__ pair,
                                                             float* __restrict__ v) {
  typedef typename S::E E;
  __shared__ __align__(16) char lds[S::kLds];
  const int block = static_cast<int>(blockIdx.x);
  if (block >= products) {
    const int w = uniform((block - products) * S::kWaves + static_cast<int>(threadIdx.x) / kWave);
    if (w < T * ((ad.r + kRanks - 1) / kRanks)) few_low<E, kRanks>(w, x, ldx, K, A, lda, ad, pair, v);
    return;
  }
  const int share = block / tiles, tile = block % tiles, i0 = tile % row_tiles * S::BM, j0 = tile / row_tiles * S::BN;
  const int k0 = share * each, count = K - k0 < each ? K - k0 : each;
  Side p{}, q{};
  p.p = x + i0 * ldx + k0;
  p.ld = ldx * sizeof(E);
  p.rows = T - i0 < S::BM ? T - i0 : S::BM;
  q.p = W + j0 * ldw + k0;
  q.ld = ldw * sizeof(E);
  q.rows = N - j0 < S::BN ? N - j0 : S::BN;
  f32x16 acc[S::TM][S::TN] = {};
  tile_products<S>(p, q, count, lds, acc);
  tile_store<S>(acc, [&](int i, int j, const f32x16& u) {
    i += i0;
    j += j0;
    if (j >= N) return;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (i + acc_row(e) < T) part[(static_cast<int64_t>(share) * T + i + acc_row(e)) * N + j] = u[e];
  });
}

template <class E>
__global__ __launch_bounds__(256) void ad_few_join_kernel(int T, int N, int shares, const float* __restrict__ part,
                                                          const float* __restrict__ bias, AdLow low,
                                                          const int32_t* __restrict__ pair, E* __restrict__ y,
                                                          int64_t ldy) {
  constexpr int kV = Vec16<E>::kCount;
  typedef typename Vec16<E>::type V;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x, size = static_cast<uint32_t>(T) * static_cast<uint32_t>(N);
  if (i >= size) return;
  const int t = static_cast<int>(i / static_cast<uint32_t>(N)), n = static_cast<int>(i % static_cast<uint32_t>(N));
  const int a = pair[t];
  float sum = 0.0f;
  for (int k = 0; k < shares; ++k) sum += part[static_cast<int64_t>(k) * size + i];
  if (bias) sum += bias[n];
  if (a >= 0) {
    const E* f = static_cast<const E*>(low.F) + (static_cast<int64_t>(a) * N + n) * low.ldf;
    const float* v = low.v + static_cast<int64_t>(t) * low.r;
    float dot = 0.0f;
#pragma unroll 2
    for (int rho = 0; rho < low.r; rho += kV) {
      const V b = load_some<E>(f + rho, low.r - rho, low.wide != 0);
#pragma unroll
      for (int e = 0; e < kV; ++e)
        dot = fmaf(rho + e < low.r ? v[rho + e] : 0.0f, static_cast<float>(b[e]), dot);
    }
    sum = fmaf(low.scale[a], dot, sum);
  }
  y[t * ldy + n] = static_cast<E>(sum);
}

// Rows of x that a workgroup of the projection takes.  float32 products are slow enough that two waves share them.
inline int few_tile_rows(int64_t T, size_t size) { return T <= 32 || size == 4 && T > kFewRows ? 32 : 64; }

// Shares of the contraction: about 256 workgroups, at least 512 bytes of a row each.
inline int few_shares(int64_t T, int K, int N, size_t size) {
  const int64_t tiles = ceil_div(N, 64) * ceil_div(T, few_tile_rows(T, size)), most = ceil_div(K * static_cast<int64_t>(size), 512);
  int64_t n = tiles > 0 ? 256 / tiles : 1;  // no rows: none
  if (n > most) n = most;
  return n < 1 ? 1 : n > 16 ? 16 : static_cast<int>(n);
}

template <class E>
lipcache_status ad_few(const AdRows<E>& x, int T, const AdRows<E>& W, int K, int N, const float* bias,
                       const AdRows<E>& A, const lipcache_adapters& ad, const AdLow& low, int32_t* pair, float* part,
                       float* v, E* y, int64_t ldy, hipStream_t s) {
  const int rows = few_tile_rows(T, sizeof(E)), row_tiles = static_cast<int>(ceil_div(T, rows));
  const int tiles = static_cast<int>(ceil_div(N, 64)) * row_tiles, wanted = few_shares(T, K, N, sizeof(E));
  const int each = static_cast<int>(round_up(ceil_div(K, wanted), 128 / sizeof(E)));
  const int shares = static_cast<int>(ceil_div(K, each));
  auto run = [&](auto shape, auto ranks) {
    typedef decltype(shape) S;
    constexpr int kRanks = decltype(ranks)::value;
    static_assert(S::kWaves == 4, "four rows and ranks a workgroup");
    const unsigned blocks = static_cast<unsigned>(tiles * shares + ceil_div(T * ceil_div(ad.r, kRanks), 4));
    ad_few_kernel<S, kRanks><<<blocks, S::kThreads, 0, s>>>(x.p, x.ld, T, W.p, W.ld, K, N, row_tiles, tiles,
                                                            tiles * shares, each, part, A.p, A.ld, ad, pair, v);
  };
  typedef TileShape<E, 32, 64, 1, 2, 2, 4, 1, false, false> Low;
  typedef TileShape<E, 64, 64, 2, 2, 1, 3, 1, false, false> High;
  // one rank a wave where the batch is a few rows (latency), four where its rows fill the chip
  if (T <= 32) run(Low{}, std::integral_constant<int, 1>{});
  else if (T <= kFewRows) run(High{}, std::integral_constant<int, 1>{});
  else if constexpr (sizeof(E) == 4) run(Low{}, std::integral_constant<int, 4>{});
  else run(High{}, std::integral_constant<int, 4>{});
  LC_LAUNCHED();
  ad_few_join_kernel<E><<<static_cast<unsigned>(ceil_div(static_cast<int64_t>(T) * N, 256)), 256, 0, s>>>(
      T, N, shares, part, bias, low, pair, y, ldy);
  LC_LAUNCHED();
  return LIPCACHE_OK;
}

// -------------------------------------------------------- gradients of pairs
// The factors u and v as the gradient kernel's operand: for each tile of the
// table a block of r rows of 128 bytes, row rho the tile's 32 values f[row][rho]
// as float32, or as 32 first and 32 second 16-bit parts; zeros past its rows.
// bfloat16's third parts follow as r rows of 64 bytes.
// float16: times 2^exponent[tile], a multiple of 4 (so that the sums, which
// follow it, seldom change) up to 40 (float16 gradients are zero from there).
constexpr int kNoExponent = -1000;  // a tile of zeros
template <class E>
inline constexpr int kFactorRow = kFactorParts<E> == 3 ? 192 : 128;  // bytes a rank and tile

template <class E>
__global__ __launch_bounds__(256) void ad_factor_kernel(const float* __restrict__ u, const float* __restrict__ v, int r,
                                                        int pairs, AdGroups g, E* __restrict__ to_u, E* __restrict__ to_v,
                                                        int32_t* __restrict__ exps_u, int32_t* __restrict__ exps_v,
                                                        int64_t first) {
  __shared__ float tile[32][kAdMaxRank + 1];
  __shared__ float wave_top[256 / kWave];
  const int t = static_cast<int>(first + blockIdx.x);
  const int last = g.tile_start[pairs], row0 = g.tile_row[t], rows = g.tile_rows[t];
  if (static_cast<uint32_t>(t) >= static_cast<uint32_t>(last)) return;
  const float* f = blockIdx.y ? v : u;
  E* to = (blockIdx.y ? to_v : to_u) + static_cast<int64_t>(t) * r * (kFactorRow<E> / sizeof(E));
  const int x = static_cast<int>(threadIdx.x) & 31, y = static_cast<int>(threadIdx.x) >> 5;
  float top = 0.0f;
#pragma unroll
  for (int i = y; i < 32; i += 8) {
    const float* from = f + static_cast<int64_t>(g.order[row0 + (i < rows ? i : 0)]) * r;
    for (int rho = x; rho < r; rho += 32) {
      const float w = i < rows ? from[rho] : 0.0f;
      tile[i][rho] = w;
      if constexpr (kScaledFactors<E>) top = fmaxf(top, finite_size(w));
    }
  }
  if constexpr (kScaledFactors<E>) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    if (lane_id() == 0) wave_top[threadIdx.x / kWave] = top;
  }
  __syncthreads();
  int up = 0;
  if constexpr (kScaledFactors<E>) {
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    if (top > 0.0f) up = factor_exponent(top) & ~3;
    if (up > 40) up = 40;
    if (threadIdx.x == 0) (blockIdx.y ? exps_v : exps_u)[t] = top > 0.0f ? up : kNoExponent;
  }
  for (int rho = y; rho < r; rho += 8) {
    const float w = two_to<E>(tile[x][rho], up);
    E* p = to + rho * (128 / sizeof(E)) + x;
    E part[kFactorParts<E>];
    if constexpr (std::is_same_v<E, float>) part[0] = w;
    else factor_parts(w, part);
    p[0] = part[0];
    if constexpr (kFactorParts<E> > 1) p[32] = part[1];
    if constexpr (kFactorParts<E> > 2) to[r * 64 + rho * 32 + x] = part[2];
  }
}

// D_a[rho][c] = scale_a sum over pair a's rows t of f[t][rho] z[t][c]: dA with
// f = u, z = x, and dB (transposed) with f = v, z = dy.  One workgroup takes
// 128 columns of one pair (and one of `splits` shares of its tiles); a tile's 32
// rows of z come gathered into LDS through a ring of buffers, two tiles a step,
// and are read across (the contraction runs over the rows); their row numbers
// come by scalar loads, which vmcnt does not count, so the ring's waits are
// exact.  Bound by reading x and dy once: 134 MB of bf16 in 35 us (3.8 TB/s; 30
// when the factors were two numbers, 42 with the row numbers loaded where they are used).
template <class E>
struct AdGradSide {
  const E* z;
  int64_t ldz;
  const E* f;      // ad_factor_kernel's
  E* out;          // dA: [S][r][width];  dB: [S][width][r]
  float* part;     // [splits][S][r][width] where splits > 1
  int width, blocks;
  bool across;     // dB's layout
};

template <class E, int NR>
__global__ __launch_bounds__(256) void ad_grad_kernel(AdGradSide<E> A, AdGradSide<E> B, int r, int S, int splits,
                                                      const float* __restrict__ scale, const int32_t* __restrict__ order,
                                                      const int32_t* __restrict__ start,
                                                      const int32_t* __restrict__ tile_start,
                                                      const int32_t* __restrict__ exps_a,
                                                      const int32_t* __restrict__ exps_b, const void* zeros, int64_t first) {
  constexpr bool kF32 = std::is_same_v<E, float>;
  constexpr int kV = Vec16<E>::kCount, kSize = static_cast<int>(sizeof(E));
  typedef typename Vec16<E>::type V;
  typedef TileOf<E, 128, true, 4> TileZ;                                       // rows of it, as many as there are
  typedef TileOf<std::conditional_t<kF32, float, Split>, 32 * NR, false, 4> TileF;
  // third parts: ranks rho and rho + 16 of 32 share a row of 128 bytes, swizzled as the others
  constexpr bool kThird = kFactorParts<E> == 3;
  constexpr int kZ = 32 * 128 * kSize, kF = NR * 4096, kT = kThird ? NR * 2048 : 0, kTile = kZ + kF + kT;  // LDS bytes of a tile
  // A third stage only where two workgroups share a CU all the same: with it bfloat16's (86 KB) took the
  // backward pass of 8192 x 4096 -> 4096, rank 32, from 350 to 364 us
  constexpr int kSub = 2, kStages = NR == 1 && !kThird ? 3 : 2;
  constexpr int kZCopies = kZ / 4096, kFCopies = NR, kTCopies = kThird ? (NR + 1) / 2 : 0;  // of a wave and tile
  constexpr int kTLanes = NR == 1 ? 32 : 64;                                   // of a copy of third parts
  constexpr int kRowsCopy = 64 / TileZ::kSlots;                                // rows of z a copy takes: 4 or 2
  constexpr int kGroups = kF32 ? 4 : 2, kParts = kF32 ? 1 : 2;
  __shared__ __align__(16) char lds[kStages * kSub * kTile];
  const int per = (A.blocks + B.blocks) * splits;
  const int number = static_cast<int>(first + blockIdx.x), a = number / per;
  int in = number % per;
  const int share = in % splits;
  in /= splits;
  const bool second = in >= A.blocks;
  const AdGradSide<E>& d = second ? B : A;
  const int c0 = (second ? in - A.blocks : in) * 128;
  const int end = start[a + 1], all = tile_start[a + 1] - tile_start[a];
  const int each = (all + splits - 1) / splits;
  const int tile0 = tile_start[a] + share * each;
  const int tiles = all - share * each < each ? all - share * each : each;
  const int lane = lane_id(), wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int li = lane & 31, half = lane >> 5;
  const uint32_t base = lds_address(lds);

  auto copy = [&](const void* p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(uniform(static_cast<int>(to)))
                 : "memory", "m0");
  };
  // a pair's tiles are neighbours, so the places of its rows are known; the rows there come a step ahead of the copies
  // (offsets that decrease may put a tile past the pair's end: it reads as empty)
  const int64_t place0 = uniform(start[a]) + static_cast<int64_t>(share) * each * kThinRows;
  auto place = [&](int n) {
    const int64_t at = place0 + static_cast<int64_t>(n) * kThinRows;
    return n < tiles && at < end ? static_cast<int>(at) : end;
  };
  typedef int32_t rows_t __attribute__((ext_vector_type(kRowsCopy), aligned(4)));
  rows_t ahead[kSub][kZCopies];
  auto rows_of_step = [&](int step) {
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      const int n = step * kSub + u;
#pragma unroll
      for (int c = 0; c < kZCopies; ++c)
        ahead[u][c] = *reinterpret_cast<const rows_t*>(order + uniform(place(n)) + (wave * kZCopies + c) * kRowsCopy);
    }
  };
  auto copy_tile = [&](int n, const rows_t (&row_of)[kZCopies], uint32_t to) {  // tile n of the share; zeros past the last
    const bool some = n < tiles;
    const int t = uniform(tile0 + (some ? n : 0));
    const int row0 = place(n);
#pragma unroll
    for (int c = 0; c < kZCopies; ++c) {
      const int first = (wave * kZCopies + c) * kRowsCopy;
      const rows_t rows = row_of[c];
      const int mine = lane / TileZ::kSlots;
      int row = rows[0];
#pragma unroll
      for (int e = 1; e < kRowsCopy; ++e) row = mine == e ? rows[e] : row;
      const int chunk = (lane % TileZ::kSlots) ^ TileZ::swz(first + mine);
      const int col = c0 + chunk * kV;
      const void* p = zeros;  // rows past the pair's and columns past the matrix
      if (first + mine < end - row0 && col < d.width) p = d.z + row * d.ldz + col;
      copy(p, to + (wave * kZCopies + c) * 1024);
    }
    const char* f = reinterpret_cast<const char*>(d.f) + static_cast<int64_t>(t) * r * kFactorRow<E>;
#pragma unroll
    for (int c = 0; c < kFCopies; ++c) {
      const int n8 = (wave * kFCopies + c) * 64 + lane, rho = n8 / 8, chunk = (n8 % 8) ^ TileF::swz(rho);
      copy(some && rho < r ? f + rho * 128 + chunk * 16 : static_cast<const char*>(zeros),
           to + kZ + (wave * kFCopies + c) * 1024);
    }
#pragma unroll
    for (int c = 0; c < kTCopies; ++c) {
      const int n8 = (wave * kTCopies + c) * kTLanes + lane, at = n8 / 8, chunk = (n8 % 8) ^ TileF::swz(at);
      const int rho = at / 16 * 32 + at % 16 + chunk / 4 * 16;
      if (lane < kTLanes)
        copy(some && rho < r ? f + r * 128 + rho * 64 + chunk % 4 * 16 : static_cast<const char*>(zeros),
             to + kZ + kF + (wave * kTCopies + c) * (kTLanes * 16));
    }
  };
  f32x16 acc[NR] = {};
  uint32_t rz[kGroups], rf[kGroups][kParts], rt[kGroups];
#pragma unroll
  for (int n = 0; n < kGroups; ++n) {
    rz[n] = TileZ::row_offset(TileZ::read_offset(n, 0), wave);
#pragma unroll
    for (int h = 0; h < kParts; ++h) rf[n][h] = kZ + TileF::read_offset(n, h);
    rt[n] = kZ + kF + (li & 15) * 128 + (((2 * n + half + (li >> 4) * 4) ^ TileF::swz(li & 15)) * 16);
  }
  const int steps = tiles > 0 ? (tiles + kSub - 1) / kSub : 0;
  constexpr int kCopies = kSub * (kZCopies + kFCopies + kTCopies);
  auto copy_step = [&](int step) {
#pragma unroll
    for (int u = 0; u < kSub; ++u)
      copy_tile(step * kSub + u, ahead[u], base + (step % kStages * kSub + u) * kTile);
    rows_of_step(step + 1);
  };
  rows_of_step(0);
  for (int step = 0; step < kStages - 1 && step < steps; ++step) copy_step(step);
  int up = 0;  // the sums are times 2^up
  for (int step = 0; step < steps; ++step) {
    int exps[kSub];
    if constexpr (kScaledFactors<E>) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const int n = step * kSub + u;
        exps[u] = n < tiles ? uniform((second ? exps_b : exps_a)[uniform(tile0 + n)]) : kNoExponent;
      }
    }
    if (kStages > 2 && step + 1 < steps) copies_left<(kStages - 2) * kCopies>();
    else copies_left<0>();
    __syncthreads();
    if (step + kStages - 1 < steps) copy_step(step + kStages - 1);
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      const char* at = lds + (step % kStages * kSub + u) * kTile;
      if constexpr (kScaledFactors<E>) {
        if (exps[u] != kNoExponent && exps[u] != up) {
#pragma unroll
          for (int m = 0; m < NR; ++m)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][e] = two_to<E>(acc[m][e], exps[u] - up);
          up = exps[u];
        }
      }
#pragma unroll
      for (int n = 0; n < kGroups; ++n) {
        const V z = __builtin_bit_cast(V, TileZ::read16(at + rz[n]));
#pragma unroll
        for (int m = 0; m < NR; ++m) {
          if constexpr (kThird)
            acc[m] = MfmaType<E>::mul(__builtin_bit_cast(V, TileF::read16(at + rt[n] + m * 2048)), z, acc[m]);
#pragma unroll
          for (int h = kParts - 1; h >= 0; --h)
            acc[m] = MfmaType<E>::mul(__builtin_bit_cast(V, TileF::read16(at + TileF::row_offset(rf[n][h], m))), z, acc[m]);
        }
      }
    }
  }
  const int col = c0 + wave * 32 + li;
  if (col >= d.width) return;
  const float sc = scale[a];
#pragma unroll
  for (int m = 0; m < NR; ++m)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int rho = 32 * m + acc_row(e) + 4 * half;
      if (rho >= r) continue;
      const float sum = two_to<E>(acc[m][e], -up);
      if (splits > 1) {
        d.part[((static_cast<int64_t>(share) * S + a) * r + rho) * d.width + col] = sum;
      } else {
        const int64_t to = d.across ? (static_cast<int64_t>(a) * d.width + col) * r + rho
                                    : (static_cast<int64_t>(a) * r + rho) * d.width + col;
        d.out[to] = static_cast<E>(all > 0 ? sc * sum : 0.0f);
      }
    }
}

// Adds the shares in order.
template <class E>
__global__ __launch_bounds__(256) void ad_join_kernel(AdGradSide<E> A, AdGradSide<E> B, int r, int S, int splits,
                                                      const float* __restrict__ scale, AdGroups g) {
  const AdGradSide<E>& d = blockIdx.y ? B : A;
  const int64_t size = static_cast<int64_t>(S) * r * d.width;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= size) return;
  float sum = 0.0f;
  for (int k = 0; k < splits; ++k) sum += d.part[k * size + i];
  const int col = static_cast<int>(i % d.width), rho = static_cast<int>(i / d.width % r);
  const int64_t a = i / d.width / r;
  const int64_t to = d.across ? (a * d.width + col) * r + rho : i;
  d.out[to] = static_cast<E>(g.tile_start[a] < g.tile_start[a + 1] ? scale[a] * sum : 0.0f);
}

// ------------------------------------------------------------------ the calls
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t ad_size(int32_t dtype) { return dtype == LIPCACHE_F32 ? 4 : 2; }

// The workspace, in order of use.  Sizes only: `at` NULL gives the sum.
struct AdSpace {
  char* at;
  size_t used = 0;
  template <class P>
  P* take(size_t count) {
    P* p = reinterpret_cast<P*>(at ? at + used : nullptr);
    used += align_up(count * sizeof(P), 256);
    return p;
  }
};

AdGroups ad_groups(AdSpace& ws, int64_t T, int S) {
  AdGroups g;
  g.order = ws.take<int32_t>(T + 64);  // scalar loads read whole vectors
  g.pair = ws.take<int32_t>(T);
  g.start = ws.take<int32_t>(S + 2);
  g.tile_pair = ws.take<int32_t>(ad_tiles(T, S) + 1);
  g.tile_row = ws.take<int32_t>(ad_tiles(T, S) + 1);
  g.tile_rows = ws.take<int32_t>(ad_tiles(T, S) + 1);
  g.tile_start = ws.take<int32_t>(S + 1);
  g.zeros = ws.take<uint32_t>(4);
  return g;
}

lipcache_status ad_group(int64_t t0, int64_t T, const lipcache_adapters& ad, const AdGroups& g, hipStream_t s) {
  ad_group_kernel<<<ad.S + 1, kGroupThreads, (ad.S + 1 + 2 * kGroupThreads + kGroupRound + kGroupThreads / kWave) * 4, s>>>(
      t0, static_cast<int>(T), ad.offsets, ad.adapter, ad.R, ad.S, g);
  LC_LAUNCHED();
  return LIPCACHE_OK;
}

// `rows` rows of a matrix as AdRows: itself, or its copy in `room`, which `copies` will make.
template <class E>
AdRows<E> ad_rows(const void* from, int64_t ld, int64_t rows, int width, E* room, AdCopyList& copies) {
  constexpr int kV = Vec16<E>::kCount;
  if (aligned16(from) && ld % kV == 0 && width % kV == 0 && ld * sizeof(E) <= (4u << 20))
    return {static_cast<const E*>(from), ld};
  const int64_t to = round_up(width, kV);
  const int n = static_cast<int>(rows);
  copies.add({from, room, ld, to, 0, 0, n, width, n, static_cast<int>(to), 1, 0});
  return {room, to};
}

// v (u) of every row; rows without a pair are written (zeros) where `all_rows`.
template <class E>
lipcache_status ad_thin(const AdRows<E>& x, int width, const E* F, int64_t ldf, int T, const lipcache_adapters& ad,
                        const AdGroups& g, float* out, float* peak, bool all_rows, hipStream_t s) {
  const int64_t table = ad_tiles(T, ad.S), more = all_rows ? ceil_div(T, 256) : 0;
  const unsigned blocks = static_cast<unsigned>(table + (more < 256 ? more : 256));
  if (blocks == 0) return LIPCACHE_OK;
  auto run = [&](auto shape) {
    typedef decltype(shape) S;
    ad_thin_kernel<S><<<blocks, S::kThreads, 0, s>>>(x.p, x.ld, width, F, ldf, ad.r, ad.S, T, g, out, peak);
    return hipGetLastError() == hipSuccess ? LIPCACHE_OK : LIPCACHE_EHIP;
  };
  if (ad.r <= 32) return run(TileShape<E, 32, 32, 1, 1, 4, 4, 2, false, false>{});
  if (ad.r <= 64) return run(TileShape<E, 32, 64, 1, 1, 4, 3, 2, false, false>{});
  return run(TileShape<E, 32, 128, 1, 1, 4, 3, 1, false, false>{});
}

struct AdArgs {
  const void *x, *W, *dy;
  int64_t ldx, ldw, lddy, T;
  int K, N;
  lipcache_adapters ad;
};

// Rows of one pass of the main product: their offsets stay below 2^31 bytes.
inline int64_t ad_chunk(int64_t ld, size_t size) {
  const int64_t rows = ((1ll << 31) - (8ll << 20)) / (ld * static_cast<int64_t>(size));
  return rows / 256 * 256 > 0 ? rows / 256 * 256 : 256;
}

template <class E>
struct AdForwardSpace {
  AdGroups g;
  float *v, *peak, *part;
  E *x, *W, *A;
  AdForwardSpace(AdSpace& ws, int64_t T, int K, int N, int r, int S) {
    constexpr int kV = Vec16<E>::kCount;
    g = ad_groups(ws, T, S);
    v = ws.take<float>(static_cast<size_t>(T) * r);
    peak = ws.take<float>(T);
    part = ws.take<float>(few_rows(T, K, N, r, sizeof(E)) ? static_cast<size_t>(T) * N * few_shares(T, K, N, sizeof(E)) : 0);
    x = ws.take<E>(static_cast<size_t>(T) * round_up(K, kV));
    W = ws.take<E>(static_cast<size_t>(N) * round_up(K, kV));
    A = ws.take<E>(static_cast<size_t>(S) * r * round_up(K, kV));
  }
};

template <class E>
lipcache_status ad_forward(const AdArgs& a, const float* bias, void* y, int64_t ldy, float* v, void* ws_, hipStream_t s) {
  constexpr int kV = Vec16<E>::kCount;
  AdSpace space{static_cast<char*>(ws_)};
  const AdForwardSpace<E> ws(space, a.T, a.K, a.N, a.ad.r, a.ad.S);
  AdCopyList copies;
  const AdRows<E> x = ad_rows<E>(a.x, a.ldx, a.T, a.K, ws.x, copies), W = ad_rows<E>(a.W, a.ldw, a.N, a.K, ws.W, copies),
                  A = ad_rows<E>(a.ad.A, a.K, static_cast<int64_t>(a.ad.S) * a.ad.r, a.K, ws.A, copies);
  lipcache_status st;
  if ((st = copies.launch<E>(s)) != LIPCACHE_OK) return st;
  const bool keep = v != nullptr;
  if (!keep) v = ws.v;
  const AdLow low{a.ad.B, a.ad.r, v, ws.peak, a.ad.scale, a.ad.r, a.ad.S, a.N, aligned16(a.ad.B) && a.ad.r % kV == 0,
                  aligned16(v) && a.ad.r % 4 == 0};
  if (few_rows(a.T, a.K, a.N, a.ad.r, sizeof(E)))
    return ad_few<E>(x, static_cast<int>(a.T), W, a.K, a.N, bias, A, a.ad, low, ws.g.pair, ws.part, v, static_cast<E*>(y), ldy, s);
  const int64_t chunk = ad_chunk(x.ld, sizeof(E));
  for (int64_t t0 = 0; t0 < a.T; t0 += chunk) {
    const int T = static_cast<int>(a.T - t0 < chunk ? a.T - t0 : chunk);
    const AdRows<E> xc{x.p + t0 * x.ld, x.ld};
    AdLow lc = low;
    lc.v = v + t0 * a.ad.r;
    if ((st = ad_group(t0, T, a.ad, ws.g, s)) != LIPCACHE_OK) return st;
    if ((st = ad_thin<E>(xc, a.K, A.p, A.ld, T, a.ad, ws.g, v + t0 * a.ad.r, ws.peak, keep, s)) != LIPCACHE_OK) return st;
    if ((st = ad_main<E, false>(xc.p, xc.ld, W.p, W.ld, T, a.N, a.K, bias, lc, ws.g, static_cast<E*>(y) + t0 * ldy, ldy, s)) !=
        LIPCACHE_OK)
      return st;
  }
  return LIPCACHE_OK;
}

// Shares of a pair's rows, so that few pairs still fill the chip: about 1024 workgroups, at least 128 rows each.
// 8192 rows of four pairs, 4096 wide, bfloat16 as two numbers: 70 us with 256 workgroups, 42 + 8 (the join) with 512, 30 + 9
// with 1024; 4096 rows of 16 pairs, 256 wide: 19 us with 64, 12 + 4 with 128.
inline int ad_splits(int64_t T, int K, int N, int S) {
  const int64_t blocks = (ceil_div(K, 128) + ceil_div(N, 128)) * (S > 0 ? S : 1);
  int64_t n = 1024 / blocks;
  const int64_t most = T / (S > 0 ? S : 1) / 128;
  if (n > most) n = most;
  return n < 1 ? 1 : n > 16 ? 16 : static_cast<int>(n);
}

template <class E>
struct AdBackwardSpace {
  AdGroups g;
  float *u, *v, *peak, *part_a, *part_b;
  int32_t *exps_u, *exps_v;
  E *x, *W, *dy, *A, *At, *Bt, *fu, *fv;
  AdBackwardSpace(AdSpace& ws, int64_t T, int K, int N, int r, int S) {
    constexpr int kV = Vec16<E>::kCount;
    const size_t K8 = round_up(K, kV), N8 = round_up(N, kV), n = S;
    g = ad_groups(ws, T, S);
    u = ws.take<float>(static_cast<size_t>(T) * r);
    v = ws.take<float>(static_cast<size_t>(T) * r);
    peak = ws.take<float>(T);
    exps_u = ws.take<int32_t>(ad_tiles(T, S));
    exps_v = ws.take<int32_t>(ad_tiles(T, S));
    At = ws.take<E>(n * K * round_up(r, kV));
    Bt = ws.take<E>(n * r * N8);
    const size_t factors = static_cast<size_t>(ad_tiles(T, S)) * r * (kFactorRow<E> / sizeof(E));
    fu = ws.take<E>(factors);
    fv = ws.take<E>(factors);
    const int splits = ad_splits(T, K, N, S);
    part_a = ws.take<float>(splits > 1 ? splits * n * r * K : 0);
    part_b = ws.take<float>(splits > 1 ? splits * n * r * N : 0);
    x = ws.take<E>(static_cast<size_t>(T) * K8);
    W = ws.take<E>(static_cast<size_t>(N) * K8);
    dy = ws.take<E>(static_cast<size_t>(T) * N8);
    A = ws.take<E>(n * r * K8);
  }
};

template <class E>
lipcache_status ad_backward(const AdArgs& a, const float* v_in, void* dx, int64_t lddx, void* dA, void* dB, void* ws_,
                            hipStream_t s) {
  constexpr int kV = Vec16<E>::kCount;
  AdSpace space{static_cast<char*>(ws_)};
  const AdBackwardSpace<E> ws(space, a.T, a.K, a.N, a.ad.r, a.ad.S);
  const int r = a.ad.r, S = a.ad.S, K = a.K, N = a.N;
  AdCopyList copies;
  AdRows<E> x{}, W{}, A{};
  const AdRows<E> dy = ad_rows<E>(a.dy, a.lddy, a.T, N, ws.dy, copies);
  if (dA) x = ad_rows<E>(a.x, a.ldx, a.T, K, ws.x, copies);
  const int64_t r8 = round_up(r, kV), N8 = round_up(N, kV);
  copies.add({a.ad.B, ws.Bt, r, N8, static_cast<int64_t>(N) * r, r * N8, N, r, r, static_cast<int>(N8), S, 1});
  if (dx) {
    copies.add({a.ad.A, ws.At, K, r8, static_cast<int64_t>(r) * K, K * r8, r, K, K, static_cast<int>(r8), S, 1});
    W = ad_rows<E>(a.W, a.ldw, N, K, ws.W, copies);
  }
  const bool need_v = dA && !v_in && S > 0;
  if (need_v) A = ad_rows<E>(a.ad.A, K, static_cast<int64_t>(S) * r, K, ws.A, copies);
  lipcache_status st;
  if ((st = copies.launch<E>(s)) != LIPCACHE_OK) return st;
  // u and, if it did not come, v of all rows; a pass for each chunk of rows whose offsets stay below 2^31 bytes
  const int64_t chunk_dy = ad_chunk(dy.ld, sizeof(E)), chunk_x = need_v ? ad_chunk(x.ld, sizeof(E)) : chunk_dy;
  const int64_t chunk = chunk_dy < chunk_x ? chunk_dy : chunk_x;
  for (int64_t t0 = 0; t0 < a.T; t0 += chunk) {
    const int T = static_cast<int>(a.T - t0 < chunk ? a.T - t0 : chunk);
    const AdRows<E> dyc{dy.p + t0 * dy.ld, dy.ld};
    if ((st = ad_group(t0, T, a.ad, ws.g, s)) != LIPCACHE_OK) return st;
    if ((st = ad_thin<E>(dyc, N, ws.Bt, N8, T, a.ad, ws.g, ws.u + t0 * r, ws.peak, false, s)) != LIPCACHE_OK) return st;
    if (need_v &&
        (st = ad_thin<E>({x.p + t0 * x.ld, x.ld}, K, A.p, A.ld, T, a.ad, ws.g, ws.v + t0 * r, nullptr, false, s)) != LIPCACHE_OK)
      return st;
    if (dx) {
      const AdLow low{ws.At, r8, ws.u + t0 * r, ws.peak, a.ad.scale, r, S, K, true, aligned16(ws.u + t0 * r) && r % 4 == 0};
      if ((st = ad_main<E, true>(dyc.p, dyc.ld, W.p, W.ld, T, K, N, nullptr, low, ws.g,
                                 static_cast<E*>(dx) + t0 * lddx, lddx, s)) != LIPCACHE_OK)
        return st;
    }
  }
  if (!dA || S == 0) return LIPCACHE_OK;
  if ((a.T == 0 || a.T > chunk) && (st = ad_group(0, a.T, a.ad, ws.g, s)) != LIPCACHE_OK) return st;
  if (const int64_t tiles = ad_tiles(a.T, S); tiles > 0) {
    st = in_passes(tiles, [&](int64_t first, unsigned n) {
      ad_factor_kernel<E><<<dim3(n, 2), 256, 0, s>>>(ws.u, need_v ? ws.v : v_in, r, S, ws.g, ws.fu, ws.fv, ws.exps_u, ws.exps_v, first);
    });
    if (st != LIPCACHE_OK) return st;
  }
  const int splits = ad_splits(a.T, K, N, S);
  const AdGradSide<E> ga{x.p, x.ld, ws.fu, static_cast<E*>(dA), ws.part_a, K, static_cast<int>(ceil_div(K, 128)), false};
  const AdGradSide<E> gb{dy.p, dy.ld, ws.fv, static_cast<E*>(dB), ws.part_b, N, static_cast<int>(ceil_div(N, 128)), true};
  auto grad = [&](auto ranks) {
    return in_passes(static_cast<int64_t>(ga.blocks + gb.blocks) * splits * S, [&](int64_t first, unsigned n) {
      ad_grad_kernel<E, decltype(ranks)::value><<<n, 256, 0, s>>>(ga, gb, r, S, splits, a.ad.scale, ws.g.order, ws.g.start,
                                                                 ws.g.tile_start, ws.exps_u, ws.exps_v, ws.g.zeros, first);
    });
  };
  if (r <= 32) st = grad(std::integral_constant<int, 1>{});
  else if (r <= 64) st = grad(std::integral_constant<int, 2>{});
  else st = grad(std::integral_constant<int, 4>{});
  if (st != LIPCACHE_OK) return st;
  if (splits > 1) {
    const int64_t most = static_cast<int64_t>(S) * r * (K > N ? K : N);
    ad_join_kernel<E><<<dim3(static_cast<unsigned>(ceil_div(most, 256)), 2), 256, 0, s>>>(ga, gb, r, S, splits, a.ad.scale, ws.g);
    LC_LAUNCHED();
  }
  return LIPCACHE_OK;
}

template <class E>
size_t ad_workspace(bool backward, int64_t T, int K, int N, int r, int S) {
  AdSpace space{nullptr};
  if (backward) AdBackwardSpace<E>(space, T, K, N, r, S);
  else AdForwardSpace<E>(space, T, K, N, r, S);
  return space.used;
}

size_t ad_workspace(bool backward, int64_t T, int K, int N, int r, int S, int32_t dtype) {
  if (dtype == LIPCACHE_F32) return ad_workspace<float>(backward, T, K, N, r, S);
  return dtype == LIPCACHE_BF16 ? ad_workspace<__bf16>(backward, T, K, N, r, S) : ad_workspace<_Float16>(backward, T, K, N, r, S);
}

// ------------------------------------------------------------- validation
bool ad_sizes_bad(int64_t T, int32_t K, int32_t N, int32_t dtype) {
  return T < 0 || K < 1 || N < 1 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16;
}

bool ad_unaligned(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == LIPCACHE_F32 ? 3u : 1u)) != 0;
}

lipcache_status ad_check(const lipcache_adapters* ad, int64_t T, int32_t K, int32_t N, int32_t dtype) {
  if (!ad || ad_sizes_bad(T, K, N, dtype)) return LIPCACHE_EINVAL;
  if (ad->S < 0 || ad->R < 0 || ad->r < 1) return LIPCACHE_EINVAL;
  if (ad->S > 0 && (!ad->A || !ad->B || !ad->scale || ad_unaligned(ad->A, dtype) || ad_unaligned(ad->B, dtype) ||
                    ad_unaligned(ad->scale, LIPCACHE_F32)))
    return LIPCACHE_EINVAL;
  if (ad->R > 0 && (!ad->offsets || !ad->adapter || ad_unaligned(ad->offsets, LIPCACHE_F32) ||
                    ad_unaligned(ad->adapter, LIPCACHE_F32)))
    return LIPCACHE_EINVAL;
  if (ad->r > kAdMaxRank || K > kAdMaxWidth || N > kAdMaxWidth || T > 0x7fffffff || ad->S > kAdMaxPairs || ad->R > kAdMaxRequests)
    return LIPCACHE_EUNSUPPORTED;
  return LIPCACHE_OK;
}

}  // namespace lc

using namespace lc;

extern "C" size_t lipcache_adapter_forward_workspace_bytes(int64_t T, int32_t K, int32_t N, int32_t r, int32_t S,
                                                           int32_t dtype) {
  if (ad_sizes_bad(T, K, N, dtype) || r < 1 || S < 0) return 0;
  return ad_workspace(false, T, K, N, r, S, dtype);
}

extern "C" lipcache_status lipcache_adapter_forward(const void* x, int64_t ldx, int64_t T, const void* W, int64_t ldw,
                                                    const float* bias, int32_t K, int32_t N,
                                                    const lipcache_adapters* ad, int32_t dtype, void* y, int64_t ldy,
                                                    float* v, void* ws, size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = ad_check(ad, T, K, N, dtype); st != LIPCACHE_OK) return st;
  if (ldx < K || ldw < K || ldy < N) return LIPCACHE_EINVAL;
  if (T > 0 && (!x || !W || !y)) return LIPCACHE_EINVAL;
  if (ad_unaligned(x, dtype) || ad_unaligned(W, dtype) || ad_unaligned(y, dtype) || ad_unaligned(bias, LIPCACHE_F32) ||
      ad_unaligned(v, LIPCACHE_F32))
    return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < lipcache_adapter_forward_workspace_bytes(T, K, N, ad->r, ad->S, dtype))
    return LIPCACHE_EWORKSPACE;
  if (T == 0) return LIPCACHE_OK;
  AdArgs g{x, W, nullptr, ldx, ldw, 0, T, K, N, *ad};
  switch (dtype) {
    case LIPCACHE_F32: return ad_forward<float>(g, bias, y, ldy, v, ws, stream);
    case LIPCACHE_BF16: return ad_forward<__bf16>(g, bias, y, ldy, v, ws, stream);
    default: return ad_forward<_Float16>(g, bias, y, ldy, v, ws, stream);
  }
}

extern "C" size_t lipcache_adapter_backward_workspace_bytes(int64_t T, int32_t K, int32_t N, int32_t r, int32_t S,
                                                            int32_t dtype) {
  if (ad_sizes_bad(T, K, N, dtype) || r < 1 || S < 0) return 0;
  return ad_workspace(true, T, K, N, r, S, dtype);
}

extern "C" lipcache_status lipcache_adapter_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t T,
                                                     const void* W, int64_t ldw, int32_t K, int32_t N,
                                                     const lipcache_adapters* ad, int32_t dtype, const float* v,
                                                     void* dx, int64_t lddx, void* dA, void* dB, void* ws,
                                                     size_t ws_bytes, lipcache_stream_t stream) {
  if (lipcache_status st = ad_check(ad, T, K, N, dtype); st != LIPCACHE_OK) return st;
  if (lddy < N || ldx < K || ldw < K || (dx && lddx < K) || !dA != !dB) return LIPCACHE_EINVAL;
  if (T > 0 && (!dy || !x || !W)) return LIPCACHE_EINVAL;
  if (ad_unaligned(dy, dtype) || ad_unaligned(x, dtype) || ad_unaligned(W, dtype) || ad_unaligned(dx, dtype) ||
      ad_unaligned(dA, dtype) || ad_unaligned(dB, dtype) || ad_unaligned(v, LIPCACHE_F32))
    return LIPCACHE_EINVAL;
  if (!ws || !aligned256(ws) || ws_bytes < lipcache_adapter_backward_workspace_bytes(T, K, N, ad->r, ad->S, dtype))
    return LIPCACHE_EWORKSPACE;
  AdArgs g{x, W, dy, ldx, ldw, lddy, T, K, N, *ad};
  switch (dtype) {
    case LIPCACHE_F32: return ad_backward<float>(g, v, dx, lddx, dA, dB, ws, stream);
    case LIPCACHE_BF16: return ad_backward<__bf16>(g, v, dx, lddx, dA, dB, ws, stream);
    default: return ad_backward<_Float16>(g, v, dx, lddx, dA, dB, ws, stream);
  }
}
