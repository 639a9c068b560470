// Rows of logits in registers: what the scoring and distillation kernels share.
//
// G threads take a row (several rows a wave, one a wave, or one a workgroup) and
// hold it as N chunks of 16 bytes each, chunk c in thread c % G, beside up to seven
// single elements past the last whole chunk, one in each of the first threads.  Chunks are read and
// written as vectors whatever the row's alignment (the hardware takes them from any element's address).
// What lies past the row is -inf, which adds nothing to any sum.
//
// A row is read from memory once.  A thread's sums follow its own largest value, block after block as the
// chunks arrive, and are scaled to the row's when the threads' are joined.  A
// workgroup goes on to another row where there are more rows than workgroups, and
// asks for each chunk of it as soon as the old one is not needed any more, so that memory has
// work while a row is finished.
#pragma once

#include <type_traits>

#include "lc_common.hpp"

namespace lc {

constexpr int kRowMostClasses = 1 << 20;
constexpr float kRowInf = __builtin_huge_valf();
constexpr float kRowLn2 = 0.6931471805599453f;
constexpr float kRowLog2e = 1.4426950408889634f;
constexpr float kRowLeast = -1000.0f;  // exponents below add nothing: 2^-1000 is zero, and -inf times zero is not

__device__ __forceinline__ float row_exp2(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float row_log2(float v) { return __builtin_amdgcn_logf(v); }

// ------------------------------------------------------------ element types
// Eight numbers rounded to nearest even, as vectors: the conversion takes two at a time.
template <class H>
__device__ __forceinline__ u32x4 row_pack(const float* v) {
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(u32x4, __builtin_convertvector(f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, H));
}

template <class E>
struct RowType;
template <>
struct RowType<float> {
  static constexpr int V = 4;
  static constexpr uint32_t kFill = 0xff800000u;
  typedef u32x4 __attribute__((aligned(4))) vec;
  static __device__ __forceinline__ float get(const u32x4& r, int e) { return __builtin_bit_cast(f32x4, r)[e]; }
  static __device__ __forceinline__ float part(uint32_t word, int) { return __builtin_bit_cast(float, word); }  // element of a word
  static __device__ __forceinline__ u32x4 pack(const float* v) {
    return __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
  }
};
template <>
struct RowType<__bf16> {
  static constexpr int V = 8;
  static constexpr uint32_t kFill = 0xff80ff80u;
  typedef u32x4 __attribute__((aligned(2))) vec;
  static __device__ __forceinline__ float get(const u32x4& r, int e) {
    const uint32_t both = r[e >> 1];
    return __builtin_bit_cast(float, e & 1 ? both & 0xffff0000u : both << 16);
  }
  static __device__ __forceinline__ float part(uint32_t word, int e) {
    return __builtin_bit_cast(float, (e & 1 ? word >> 16 : word) << 16);
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) { return row_pack<bf16x8>(v); }
};
template <>
struct RowType<_Float16> {
  static constexpr int V = 8;
  static constexpr uint32_t kFill = 0xfc00fc00u;
  typedef u32x4 __attribute__((aligned(2))) vec;
  static __device__ __forceinline__ float get(const u32x4& r, int e) {
    return static_cast<float>(__builtin_bit_cast(f16x8, r)[e]);
  }
  static __device__ __forceinline__ float part(uint32_t word, int e) {
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(e & 1 ? word >> 16 : word)));
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) { return row_pack<f16x8>(v); }
};

// ------------------------------------------------------ lanes of one wave
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
  const int b = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_f32(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

constexpr int kDppHalfMirror = 0x141;  // lane i of each 8 <- lane 7 - i
constexpr int kDppMirror = 0x140;      // lane i of each 16 <- lane 15 - i

// The join of a value over groups of L lanes (16: a row of the wave; 64: the wave).  Every step joins two halves that
// are alike throughout, so all lanes get the same bits (a product must not be fused into the first sum: it would be
// exact on one side of it and rounded on the other).
template <int L, class F>
__device__ __forceinline__ float lanes_join(float v, F join) {
  asm("" : "+v"(v));
  v = join(v, dpp_f32<kDppQuadXor1>(v));
  v = join(v, dpp_f32<kDppQuadXor2>(v));
  v = join(v, dpp_f32<kDppHalfMirror>(v));
  v = join(v, dpp_f32<kDppMirror>(v));
  if constexpr (L == 64) v = join(join(lane_f32(v, 0), lane_f32(v, 16)), join(lane_f32(v, 32), lane_f32(v, 48)));
  return v;
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  return lanes_join<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  return lanes_join<L>(v, [](float a, float b) { return fmaxf(a, b); });
}

struct RowNothing {
  template <class... A>
  __device__ __forceinline__ void operator()(A...) const {}
};

// LDS written by lanes of a wave, read by others of it.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ------------------------------------------------------------- a row's sums
// kMean: s and the sum of the exponents (to base 2) weighted by what they add to
// s; kTwo: s and the sum at a second temperature.
enum class RowWants { kSum, kMean, kTwo };

// About the value m: s = sum 2^(scale (x - m)), more as RowWants says.
struct RowSums {
  float m, s, more;
};
struct RowScale {
  float scale, second;  // log2(e) / temperature
};

// The same about another value, m or larger; from is finite unless m is +inf.
template <RowWants W>
__device__ __forceinline__ void row_move(RowSums& r, float from, const RowScale& k) {
  const float d = (r.m - from) * k.scale, f = row_exp2(d);
  if constexpr (W == RowWants::kMean) r.more = f * fmaf(fmaxf(d, kRowLeast), r.s, r.more);
  if constexpr (W == RowWants::kTwo) r.more *= row_exp2((r.m - from) * k.second);
  r.s *= f;
}
__device__ __forceinline__ float row_from(float m) { return m == -kRowInf ? 0.0f : m; }

template <int G_, int N_>
struct RowShape {
  static constexpr int G = G_, N = N_;
  static constexpr int kThreads = G > 256 ? G : 256;
  static constexpr int kRows = kThreads / G;             // of a workgroup
  static constexpr int kLanes = G < 64 ? G : 64;         // of a row in one wave
  static constexpr int kWaves = G <= 64 ? 1 : G / 64;    // of a row
};

// Where a thread stands in its row.
template <class S>
struct RowPlace {
  int g, row;  // thread of the row, row of the workgroup
  __device__ __forceinline__ RowPlace()
      : g(static_cast<int>(threadIdx.x) % S::G), row(static_cast<int>(threadIdx.x) / S::G) {
    if constexpr (S::G >= 64) row = uniform(row);
  }
  // Between the threads of a row.
  static __device__ __forceinline__ void sync() {
    if constexpr (S::G <= 64) wave_sync();
    else __syncthreads();
  }
};

// A segment of a row in registers: N chunks a thread from element `begin` (a multiple of a chunk) on, and the elements
// past the last whole chunk, which every segment holds.
template <class E, class S>
struct RowData {
  typedef RowType<E> Type;
  static constexpr int V = Type::V, N = S::N, G = S::G;
  u32x4 raw[N];
  float tail;
  const int wave;  // the first thread of the row in this wave
  __device__ __forceinline__ explicit RowData(int g) : wave(G > 64 ? uniform(g) / kWave * kWave : 0) {}

  // Chunk i as bits again: without it the compiler keeps the numbers that one pass made of them for the next, in two
  // to four times the registers.
  __device__ __forceinline__ void pin(int i) { asm volatile("" : "+v"(raw[i])); }
  static __device__ __forceinline__ u32x4 fill() { return u32x4{Type::kFill, Type::kFill, Type::kFill, Type::kFill}; }
  // Chunk first + G i + g of the row at x: a row's address (one for all lanes, where a row has whole waves), and a
  // lane's offset that is the same for all chunks.
  static __device__ __forceinline__ const char* chunk_at(const E* x, int first, int i, int g) {
    return reinterpret_cast<const char*>(x) + static_cast<int64_t>(first + G * i) * 16 + static_cast<uint32_t>(g * 16);
  }
  // The first chunk i of the wave's lanes (of the row's, where a wave holds several).
  __device__ __forceinline__ int chunk_of(int i, int first) const { return first + G * i + wave; }
  // Whether chunk i is past the row for all of them, in it for all of them.
  __device__ __forceinline__ bool past(int i, int first, int full) const { return chunk_of(i, first) >= full; }
  __device__ __forceinline__ bool inside(int i, int first, int full) const {
    return chunk_of(i, first) + (G < 64 ? G : 64) <= full;
  }
  __device__ __forceinline__ void load_chunk(int i, const E* x, int first, int full, int g) {
    if (inside(i, first, full)) {
      raw[i] = *reinterpret_cast<const typename Type::vec*>(chunk_at(x, first, i, g));
    } else {
      raw[i] = fill();
      if (g < full - (first + G * i)) raw[i] = *reinterpret_cast<const typename Type::vec*>(chunk_at(x, first, i, g));
    }
  }
  __device__ __forceinline__ void load_tail(const E* x, int C, int g) {
    const int full = C / V, j = full * V + g;
    tail = g < V && j < C ? static_cast<float>(x[j]) : -kRowInf;
  }
  __device__ __forceinline__ void load(const E* x, int first, int C, int g) {
    load_tail(x, C, g);
#pragma unroll
    for (int i = 0; i < N; ++i) load_chunk(i, x, first, C / V, g);
  }
  // Writes f of every element of chunk i (zeros unless `some`) to the row at out, where it has the chunk and is `live`.
  template <class F>
  __device__ __forceinline__ void store_chunk(int i, E* out, int first, int full, int g, bool live, bool some, F f) {
    if (past(i, first, full)) return;
    pin(i);
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = f(Type::get(raw[i], e));
    u32x4 bits = Type::pack(v);
#pragma unroll
    for (int w = 0; w < 4; ++w) bits[w] = some ? bits[w] : 0;
    if (live && g < full - (first + G * i))
      *reinterpret_cast<typename Type::vec*>(const_cast<char*>(chunk_at(out, first, i, g))) = bits;
    __builtin_amdgcn_sched_barrier(0);
  }
  template <class F>
  __device__ __forceinline__ void store_tail(E* out, int C, int g, bool live, bool some, F f) const {
    const int j = C / V * V + g;
    if (live && g < V && j < C) out[j] = static_cast<E>(some ? f(tail) : 0.0f);
  }
  // The sums of nothing but the thread's single element.
  template <RowWants W>
  __device__ __forceinline__ RowSums begin(const RowScale& k) const {
    RowSums r{fmaxf(tail, -kRowInf), 0.0f, 0.0f};  // (a NaN is no largest value; it goes into the sums)
    one<W>(tail, row_from(r.m), r, k);
    return r;
  }
  // The largest of the chunks' elements in P groups by their place in a chunk, and of the single element, which is of the
  // first (a NaN is none).
  template <int P>
  __device__ __forceinline__ void largest(int first, int full, int g, float (&m)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) m[p] = p == 0 ? fmaxf(tail, -kRowInf) : -kRowInf;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (past(i, first, full)) break;
      pin(i);
#pragma unroll
      for (int e = 0; e < V; ++e) m[e % P] = fmaxf(m[e % P], Type::get(raw[i], e));
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Adds the chunks to a thread's sums, a block of up to two at a time, each block by four sums of its own.
  // seen(m, each) is called with a block's largest value, each(hits, f) then calls f(any, value, index) for the elements
  // that hits(value), one of each lane at a time (`any`: the lane has one); used(i) when chunk i is not needed any more.
  template <RowWants W, class Seen, class Used>
  __device__ __forceinline__ void add(int first, int full, int g, RowSums& r, const RowScale& k, Seen seen, Used used) {
    constexpr int B = N == 1 || (N > 8 && V == 8) ? 1 : 2;  // chunks of a block
#pragma unroll
    for (int b = 0; b < N; b += B) {
      if (past(b, first, full)) {
#pragma unroll
        for (int i = b; i < b + B; ++i) used(i);
        continue;
      }
      float m = -kRowInf;
#pragma unroll
      for (int i = b; i < b + B; ++i) {
        pin(i);
#pragma unroll
        for (int e = 0; e < V; ++e) m = fmaxf(m, Type::get(raw[i], e));
      }
      seen(m, [&](auto hits, auto f) {
        // the lane's elements that hit, as bits; each round takes one of every lane that has some
        uint32_t mask = 0;
#pragma unroll
        for (int i = b + B - 1; i >= b; --i)
#pragma unroll
          for (int e = V - 1; e >= 0; --e) mask = 2 * mask + (hits(Type::get(raw[i], e)) ? 1u : 0u);
        while (__ballot(mask != 0) != 0) {
          const int at = __builtin_ctz(mask | 0x80000000u), word = at * 4 / V;
          uint32_t bits = raw[b][0];
#pragma unroll
          for (int w = 1; w < 4 * B; ++w) bits = word == w ? raw[b + w / 4][w % 4] : bits;
          f(mask != 0, Type::part(bits, at), (first + G * (b + at / V) + g) * V + at % V);
          mask &= mask - 1;
        }
      });
      m = fmaxf(m, r.m);
      const float from = row_from(m);
      row_move<W>(r, from, k);
      r.m = m;
      RowSums p[4] = {};
#pragma unroll
      for (int i = b; i < b + B; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) one<W>(Type::get(raw[i], e), from, p[e & 3], k);
      r.s += (p[0].s + p[1].s) + (p[2].s + p[3].s);
      if constexpr (W != RowWants::kSum) r.more += (p[0].more + p[1].more) + (p[2].more + p[3].more);
#pragma unroll
      for (int i = b; i < b + B; ++i) used(i);
      __builtin_amdgcn_sched_barrier(0);  // a block's numbers are not formed while the one before holds its own
    }
  }
  template <RowWants W>
  static __device__ __forceinline__ void one(float x, float from, RowSums& r, const RowScale& k) {
    const float d = x - from, a = d * k.scale, e = row_exp2(a);
    r.s += e;
    if constexpr (W == RowWants::kMean) r.more = fmaf(fmaxf(a, kRowLeast), e, r.more);
    if constexpr (W == RowWants::kTwo) r.more += row_exp2(d * k.second);
  }
};

// The sums of the row's threads, joined in one order: every thread gets them, about row_from(m).  Rows of more than a
// wave leave the waves' sums in `room` (kWaves of them) and meet at one barrier: what the row's threads wrote to LDS before is there after it.  The room
// may be written again after the next barrier.
template <class S, RowWants W>
__device__ __forceinline__ void row_join(RowSums& r, const RowScale& k, RowSums* room) {
  const float m = lanes_max<S::kLanes>(r.m);
  row_move<W>(r, row_from(m), k);
  r.m = m;
  r.s = lanes_sum<S::kLanes>(r.s);
  if constexpr (W != RowWants::kSum) r.more = lanes_sum<S::kLanes>(r.more);
  if constexpr (S::kWaves > 1) {
    static_assert(S::kWaves <= 16, "joined by 16 lanes");
    if (lane_id() == 0) room[threadIdx.x / kWave] = r;
    __syncthreads();
    const int w = lane_id() & 15;
    r = w < S::kWaves ? room[w] : RowSums{-kRowInf, 0.0f, 0.0f};
    const float all = lanes_max<16>(r.m);
    row_move<W>(r, row_from(all), k);
    r.m = all;
    r.s = lanes_sum<16>(r.s);
    if constexpr (W != RowWants::kSum) r.more = lanes_sum<16>(r.more);
  }
}

// --------------------------------------------------- classes named in a row
// Entries (class, value) of a row in LDS, at most `most` of them, kept by the
// row's first wave (or its lanes).  Those of one class are added up, in their
// order, by the first of them: a bit of `seen` for each class (or for several, where there are more
// than 8192) finds out in one pass which entries may be alone.
constexpr int kEntryBits = 8192;
inline int entry_bits(int C) {
  int bits = 256;
  while (bits < C && bits < kEntryBits) bits *= 2;
  return bits;
}
__host__ __device__ inline size_t entry_bytes(int most, int bits) {
  return most == 0 ? 0 : (static_cast<size_t>(most) * 12 + bits / 4 + 15) / 16 * 16;
}

struct RowEntry {
  int at;       // class, -1: none
  float value;
};

template <int LANES>
struct RowEntries {
  int* at;        // [n] class, -1: none
  float* value;   // [n]
  float* logit;   // [n] the row's own at the class
  uint32_t *seen, *twice;
  int n, bits;
  __device__ __forceinline__ RowEntries(char* lds, int n_, int bits_)
      : at(reinterpret_cast<int*>(lds + bits_ / 4)),
        value(reinterpret_cast<float*>(lds + bits_ / 4) + n_),
        logit(reinterpret_cast<float*>(lds + bits_ / 4) + 2 * n_),
        seen(reinterpret_cast<uint32_t*>(lds)),
        twice(reinterpret_cast<uint32_t*>(lds) + bits_ / 32),
        n(n_),
        bits(bits_) {}
  // By the lanes that keep the entries: entry `lane` is `mine` with its logit; entry_of and logit_of load the others, four at a
  // time so that their loads wait together.
  template <class Entry, class Logit>
  __device__ __forceinline__ void keep(int lane, RowEntry mine, float mine_logit, Entry entry_of, Logit logit_of) {  // logit_of(entry, class)
    if (lane < n) {
      at[lane] = mine.at;
      value[lane] = mine.value;
      logit[lane] = mine_logit;
    }
    for (int i = lane + LANES; i < n; i += 4 * LANES) {
      RowEntry e[4];
      float l[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) e[p] = entry_of(i + p * LANES);
#pragma unroll
      for (int p = 0; p < 4; ++p) l[p] = logit_of(i + p * LANES, e[p].at);
#pragma unroll
      for (int p = 0; p < 4; ++p)
        if (i + p * LANES < n) {
          at[i + p * LANES] = e[p].at;
          value[i + p * LANES] = e[p].value;
          logit[i + p * LANES] = l[p];
        }
    }
    wave_sync();
  }
  // Adds v to the first entry of class c; false where there is none.
  __device__ __forceinline__ bool add(int lane, int c, float v) {
    const int group = LANES == 64 ? 0 : lane_id() / LANES * LANES;  // first lane of the row
    for (int i = lane; i - lane < n; i += LANES) {
      const uint64_t all = __ballot(i < n && at[i] == c) >> group;
      const uint64_t hit = LANES == 64 ? all : all & ((1ull << (LANES & 63)) - 1);
      if (hit) {
        if (lane == __builtin_ctzll(hit)) value[i] += v;
        return true;
      }
    }
    return false;
  }
  // Which classes may be named twice.
  __device__ __forceinline__ void index(int lane) {
    if (n == 0) return;  // no room either
    for (int i = lane; i < bits / 16; i += LANES) seen[i] = 0;
    wave_sync();
    for (int i = lane; i < n; i += LANES) {
      const int c = at[i];
      if (c < 0) continue;
      const uint32_t b = static_cast<uint32_t>(c) & (bits - 1), bit = 1u << (b & 31);
      if (atomicOr(&seen[b >> 5], bit) & bit) atomicOr(&twice[b >> 5], bit);
    }
    wave_sync();
  }
  // After index(): put(i, sum) for the first entry i of every class, with the class's sum.  Only entries of a bit that was met
  // twice can share a class, so those alone are compared, each as the others' lanes hold it.
  template <class F>
  __device__ __forceinline__ void firsts(int lane, F put) const {
    auto marked = [&](int c) {
      const uint32_t b = static_cast<uint32_t>(c) & (bits - 1);
      return c >= 0 && (twice[b >> 5] >> (b & 31) & 1) != 0;
    };
    for (int i = lane; i - lane < n; i += LANES) {
      const int c = i < n ? at[i] : -1;
      float sum = i < n ? value[i] : 0.0f;
      const bool more = marked(c);
      bool mine = c >= 0;
      if (__ballot(more) != 0) {
        float all = 0.0f;
        auto meet = [&](int j, int other, float v) {
          const bool same = other == c;
          mine = mine && !(same && j < i);
          all = same ? all + v : all;
        };
        if constexpr (LANES == 64) {
          for (int base = 0; base < n; base += LANES) {
            const int own = base + lane < n ? at[base + lane] : -1;
            const float v = base + lane < n ? value[base + lane] : 0.0f;
            for (uint64_t left = __ballot(marked(own)); left != 0; left &= left - 1) {
              const int l = __builtin_ctzll(left);
              meet(base + l, __builtin_amdgcn_readlane(own, l), lane_f32(v, l));
            }
          }
        } else {
#pragma unroll 8
          for (int j = 0; j < n; ++j) meet(j, at[j], value[j]);
        }
        if (more) sum = all;
      }
      if (mine) put(i, sum);
    }
  }
};

// ----------------------------------------------------------------- host side
inline bool row_unaligned(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == LIPCACHE_F32 ? 3u : 1u)) != 0;
}
inline bool row_unaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

inline bool row_sizes_bad(int64_t T, int32_t C, int32_t k, int32_t dtype) {
  return T < 0 || C < 1 || k < 0 || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16;
}

inline lipcache_status row_check(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype, float temperature) {
  if (T < 0 || C < 1 || ldx < C || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16) return LIPCACHE_EINVAL;
  if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f)) return LIPCACHE_EINVAL;
  if ((T > 0 && !x) || row_unaligned(x, dtype)) return LIPCACHE_EINVAL;
  if (C > kRowMostClasses || T > 0x7fffffff) return LIPCACHE_EUNSUPPORTED;
  return LIPCACHE_OK;
}

template <class F>
lipcache_status row_typed(int32_t dtype, F f) {
  switch (dtype) {
    case LIPCACHE_F32: return f(float{});
    case LIPCACHE_BF16: return f(__bf16{});
    default: return f(_Float16{});
  }
}

// Calls f(shape) with a shape that holds a row of C, or one and false: the row goes in segments.  A wave takes rows of up to 512
// chunks, and of up to 1024, where there are enough for all waves: fewer threads join a row's sums, and none waits at a barrier
// for the wave that keeps the entries.  Distillation of 5003 bfloat16 with 16 entries, a wave and 256 threads a row:
// 1024 rows 13.4 and 11.6 us, 2048 rows 16.3 and 17.6, 3000 20.0 and 22.6, 8192 39 and 55.
template <class E, class F>
lipcache_status row_shaped(int64_t T, int C, F f) {
  const int chunks = C / RowType<E>::V;
  auto holds = [&](auto shape) { return chunks <= decltype(shape)::G * decltype(shape)::N; };
  if (holds(RowShape<16, 1>{})) return f(RowShape<16, 1>{}, std::true_type{});
  if (holds(RowShape<16, 2>{})) return f(RowShape<16, 2>{}, std::true_type{});
  if (holds(RowShape<16, 4>{})) return f(RowShape<16, 4>{}, std::true_type{});
  if (holds(RowShape<64, 4>{})) return f(RowShape<64, 4>{}, std::true_type{});
  if (T >= 2048 && holds(RowShape<64, 8>{})) return f(RowShape<64, 8>{}, std::true_type{});
  if (T >= 2560 && holds(RowShape<64, 16>{})) return f(RowShape<64, 16>{}, std::true_type{});
  if (holds(RowShape<256, 4>{})) return f(RowShape<256, 4>{}, std::true_type{});
  if (holds(RowShape<256, 8>{})) return f(RowShape<256, 8>{}, std::true_type{});
  if (holds(RowShape<512, 8>{})) return f(RowShape<512, 8>{}, std::true_type{});
  if (holds(RowShape<1024, 8>{})) return f(RowShape<1024, 8>{}, std::true_type{});
  if (holds(RowShape<1024, 16>{})) return f(RowShape<1024, 16>{}, std::true_type{});
  return f(RowShape<1024, 8>{}, std::false_type{});
}

// The same for kernels that keep n entries of each row in LDS: a wave for a row of 16 lanes where its entries take those many
// steps.  Distillation with two temperatures, 16 lanes and a wave a row: 32768 x 200 float16 with 20 entries 20 and 48 us, with
// 64 25 and 51, with 200 54 and 78; 32768 x 500 bfloat16 with 256 94 and 77; 4096 x 200 float32 with 64 14.4 and 13.5, with 200
// 20 and 14.
template <class E, class F>
lipcache_status row_shaped_entries(int64_t T, int C, int n, F f) {
  return row_shaped<E>(T, C, [&](auto shape, auto whole) {
    if constexpr (decltype(shape)::G < 64) {
      if (n > (T >= 16384 ? 224 : 64)) return f(RowShape<64, 4>{}, std::true_type{});
    }
    return f(shape, whole);
  });
}

// ------------------------------------------------- few rows, of many classes
// A row of a workgroup leaves the other CUs idle.  Up to 64 rows of more than 4096 chunks (a share is at least 1024, a chunk 16
// bytes) go in shares: one launch for the shares' sums, another that joins them and, for a gradient, writes it by
// shares.  What the second needs of the row beside its share (its logits at the classes that it names) the first
// puts by, as the gradient may be written over the row.
// One row of 131072 bfloat16: scores with 20 alternatives 21 us as one workgroup, gradient 20, with two temperatures 31.
constexpr int kRowFew = LIPCACHE_FEW_ROWS;
constexpr int kRowShares = 32;
struct RowShares {
  int count;  // 1: the rows are not split
  int each;   // chunks of a share
};
inline RowShares row_shares(int64_t T, int C, int32_t dtype) {
  const int chunks = C / (dtype == LIPCACHE_F32 ? 4 : 8);
  if (T < 1 || T > kRowFew || chunks <= 4096) return {1, chunks};
  const int each = ((chunks + kRowShares - 1) / kRowShares + 1023) / 1024 * 1024;
  return {(chunks + each - 1) / each, each};
}
// sums[t][share], and logits[t][k + 1] at the entries' classes and the label (0 where there is none).
lipcache_status row_share_sums(const void* x, int64_t ldx, int64_t T, int C, int32_t dtype, RowWants wants, RowScale scale,
                               RowShares shares, int k, const int32_t* index, const int32_t* label, RowSums* sums,
                               float* logits, hipStream_t s);
inline size_t row_share_bytes(int64_t T, int k, const RowShares& shares) {
  if (shares.count == 1) return 0;
  return align_up(static_cast<size_t>(T) * shares.count * sizeof(RowSums), 256) + align_up(static_cast<size_t>(T) * (k + 1) * 4, 256);
}
struct RowSplit {
  RowShares shares;
  const RowSums* sums;
  const float* logits;
};

// Workgroups: the rows, or 2048 threads a CU, the most that the chip can hold; kernels of more than 64 registers hold fewer
// (82 to 123 of them: half to five eighths, or a workgroup of 1024), and the rest start as others end.
template <class S>
unsigned row_blocks(int64_t T) {
  const int64_t need = (T + S::kRows - 1) / S::kRows, most = 256 * (2048 / S::kThreads);
  return static_cast<unsigned>(need < most ? need : most);
}

}  // namespace lc
