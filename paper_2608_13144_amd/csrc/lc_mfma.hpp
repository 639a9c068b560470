// Matrix-core products D = P Q^T of 16-bit or float32 operands with float32
// sums, one output tile a workgroup: the main loop that the adapter and
// orthogonalisation kernels share.
//
// An operand lies in memory with its contraction index contiguous ("row":
// element (i, k) at i ld + k) or with its tile index contiguous ("col":
// element (i, k) at k ld + i).  Both go from global memory straight into LDS
// with 16-byte copies (no registers), 128 bytes of the contraction a step,
// through a ring of kStages buffers, each of kSub such parts: the copy of step s + kStages - 1 is issued
// right after the barrier that publishes step s (whose products every wave's
// reads of the buffer it overwrites precede), so up to kStages - 1 steps are
// under way while one is multiplied.  The copies are buffer
// loads, so rows past the operand and the end of the contraction read as zero
// without a branch.
//
// LDS rows are not padded.  16-byte chunk c of a row goes to slot c ^ swz(row),
// a permutation of the copy's global addresses inside a row, so that the lanes
// of one read meet different banks: 16 rows of 128 bytes at one chunk for a
// "row" operand, 4 rows of k at two adjacent 16-column groups for a "col" one
// (read with the transposing LDS read, which hands lane i column i of four
// 16-element rows).
//
// The products are 32 x 32 tiles (v_mfma_f32_32x32x16 for 16-bit types, four
// v_mfma_f32_32x32x2 for float32): lane l holds row l % 32 of both operands
// and elements 8 (l / 32) .. + 8 of 16 (float32: 4 (l / 32) .. + 4 of 8, one a
// product: the order of the contraction is free as long as both agree), and
// ends with rows 8 (v / 4) + 4 (l / 32) + v % 4 of column l % 32.
#pragma once

#include "lc_common.hpp"

namespace lc {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr uint32_t kNoRow = 0x80000000u;  // a copy offset past every buffer (their sizes stay below 2^31): reads zero

// Buffer descriptor of `bytes` bytes at p (wave-uniform; raw 32-bit format, no stride).
__device__ __forceinline__ i32x4 buffer_of(const void* p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  i32x4 r;
  r[0] = uniform(static_cast<int32_t>(static_cast<uint32_t>(a)));
  r[1] = uniform(static_cast<int32_t>(static_cast<uint32_t>(a >> 32) & 0xffffu));
  r[2] = static_cast<int32_t>(bytes);
  r[3] = 0x00027000;
  return r;
}

// Lane i's 16 bytes at buf + voff land at LDS address lds + at + 16 i (buf and
// lds wave-uniform, `at` a constant).  Inline assembly, because the compiler's model of the
// intrinsic turns every wait for an ordinary LDS read into one for all of them
// while a copy is in flight.  vmcnt counts it; copies_done() waits.
__device__ __forceinline__ void copy16(i32x4 buf, uint32_t voff, uint32_t lds, int at) {
  asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(buf),
               "s"(lds), "i"(at)
               : "memory", "m0", "scc");
}

// Waits until at most N of this wave's copies are outstanding.
template <int N>
__device__ __forceinline__ void copies_left() {
  static_assert(N >= 0 && N < 64, "vmcnt holds 6 bits");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_char*)p));
}

// One operand of a product.  All offsets inside a tile (256 rows, or one step of
// the contraction, by ld) stay below 2^31.
struct Side {
  const void* p;         // element (0, 0) of the tile
  int64_t ld;            // bytes between rows
  int rows;              // rows (col: columns) of the tile that exist, >= 1
  const int32_t* pick;   // row only, or NULL: row i of the tile is pick[i] of p (the whole array below 2^31 bytes)
};

// Numbers held as a sum of two float16 (22 bits): a row of them is blocks of 32
// first parts followed by their 32 second parts, its length a multiple of 32.
// Their products are hi hi + hi lo + lo hi (the fourth is below the rounding of
// the float32 sums): three of the matrix cores' products on four fragments.
struct Split {
  uint32_t bits;
};
// v = first + second.  The empty assembly pins v's float32 value: without it the
// compiler may round `first` from an unrounded product in one place and from
// the float32 one in the other, an ulp of float16 apart near a tie.
__device__ __forceinline__ void split_f16(float v, _Float16& first, _Float16& second) {
  asm("" : "+v"(v));
  first = static_cast<_Float16>(v);
  second = static_cast<_Float16>(v - static_cast<float>(first));
}

template <class E>
struct MfmaType;
template <>
struct MfmaType<Split> {
  struct frag {
    f16x8 hi, lo;
  };
  static __device__ __forceinline__ f32x16 mul(const frag& a, const frag& b, f32x16 c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.hi, b.lo, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.lo, b.hi, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.hi, b.hi, c, 0, 0, 0);
  }
};
template <>
struct MfmaType<_Float16> {
  typedef f16x8 frag;
  static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct MfmaType<__bf16> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct MfmaType<float> {
  typedef f32x4 frag;
  static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c) {
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[0], b[0], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[1], b[1], c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[2], b[2], c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a[3], b[3], c, 0, 0, 0);
  }
};

// The tile of one operand in LDS: ROWS x 128 bytes (row) or kPart x ROWS elements
// (col), ROWS * 128 bytes either way.
template <class E, int ROWS, bool COL, int WAVES>
struct TileOf {
  static constexpr int kSize = static_cast<int>(sizeof(E));
  static constexpr bool kSplit = __is_same(E, Split);
  static constexpr int kPart = 128 / kSize;              // contraction elements of a part of a step
  static constexpr int kBytes = ROWS * 128;
  static constexpr int kCopies = kBytes / 1024 / WAVES;  // copies a wave and part
  static constexpr int kSlots = COL ? ROWS * kSize / 16 : 8;  // chunks of an LDS row
  static constexpr int kGroups = kSplit ? 2 : 4;         // fragments along a part
  static_assert(kCopies >= 1 && kBytes % (1024 * WAVES) == 0 && kSlots >= 8, "tile too small for the waves");
  static_assert(!COL || (ROWS & (ROWS - 1)) == 0, "the swizzle of a \"col\" tile permutes a power of two of chunks");

  static __device__ __forceinline__ int swz(int row) {
    if constexpr (!COL) return (row >> 1) & 7;
    if constexpr (__is_same(E, float)) return 0;
    if constexpr (kSlots >= 16) return (row & 3) << 2;
    return ((row >> 1) & 1) << 2;
  }

  const char* at;         // the operand at the next part (wave-uniform)
  int64_t advance;        // bytes to the one after
  uint32_t off[kCopies];  // byte offsets of this lane's chunks from `at`

  __device__ __forceinline__ void init(const Side& s, int wave) {
    const int lane = lane_id();
    at = static_cast<const char*>(s.p);
    advance = COL ? kPart * s.ld : 128;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int n = (wave * kCopies + c) * 64 + lane;  // slot of the tile
      const int row = n / kSlots, chunk = (n % kSlots) ^ swz(row);
      if constexpr (!COL) {
        off[c] = kNoRow;
        if (row < s.rows)
          off[c] = (s.pick ? static_cast<uint32_t>(s.pick[row]) : static_cast<uint32_t>(row)) * static_cast<uint32_t>(s.ld) +
                   chunk * 16;
      } else {
        off[c] = chunk * 16 < s.rows * kSize ? row * static_cast<uint32_t>(s.ld) + chunk * 16 : kNoRow;
      }
    }
  }

  // Copies the next part, whole (`lds`: this wave's share of the tile, AT: a constant on top).
  template <int AT>
  __device__ __forceinline__ void copy(uint32_t lds) {
    const i32x4 buf = buffer_of(at, 0x7fffffffu);
    copy_all<AT, 0>(buf, lds);
    at += advance;
  }
  template <int AT, int C>
  __device__ __forceinline__ void copy_all(i32x4 buf, uint32_t lds) const {
    copy16(buf, off[C], lds, AT + C * 1024);
    if constexpr (C + 1 < kCopies) copy_all<AT, C + 1>(buf, lds);
  }
  // The same for a part with only `left` elements of the contraction left (zeros past them; left <= 0: all).
  __device__ __forceinline__ void copy_some(int wave, int left, uint32_t lds) {
    const i32x4 buf = buffer_of(at, 0x7fffffffu);
    const int lane = lane_id();
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int n = (wave * kCopies + c) * 64 + lane;
      const int row = n / kSlots, chunk = (n % kSlots) ^ swz(row);
      copy16(buf, (COL ? row : chunk * (16 / kSize)) < left ? off[c] : kNoRow, lds + c * 1024, 0);
    }
    at += advance;
  }

  // Where this lane finds its fragment of 32 rows and group g of a part, from the tile's row 0 (col: column 0); the
  // rows' own offset is row_offset().
  static __device__ __forceinline__ uint32_t read_offset(int g, int second) {
    const int lane = lane_id();
    if constexpr (!COL) {
      const int r = lane & 31;
      return r * 128 + (((2 * g + (lane >> 5) + 4 * second) ^ swz(r)) * 16);
    } else if constexpr (__is_same(E, float)) {
      return (8 * g + 4 * (lane >> 5)) * (ROWS * 4) + (lane & 31) * 4;
    } else {
      const int i = lane & 15, k = 16 * g + 8 * (lane >> 5) + (i >> 2);
      const int j = (lane & 16) * 2 + 8 * (i & 3) + 64 * second;  // bytes
      return k * (ROWS * kSize) + (((j >> 4) ^ swz(k)) * 16) + (j & 8);
    }
  }
  // The offset 32 t rows (columns) on.  Rows keep their swizzle; columns, 64 or 128 bytes of an LDS row of a power of two
  // bytes, are an exclusive or, as the swizzle is (t may be added in parts that share no bits).
  static __device__ __forceinline__ uint32_t row_offset(uint32_t read, int t) {
    if constexpr (!COL) return read + t * 4096;
    else if constexpr (__is_same(E, float)) return read + t * 128;
    else return read ^ static_cast<uint32_t>(t * 32 * kSize);
  }
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  static __device__ __forceinline__ u32x4 read16(const char* p) {
    if constexpr (!COL) {
      return *reinterpret_cast<const u32x4*>(p);
    } else if constexpr (__is_same(E, float)) {
      const float* t = reinterpret_cast<const float*>(p);
      const f32x4 f = {t[0], t[ROWS], t[2 * ROWS], t[3 * ROWS]};
      return __builtin_bit_cast(u32x4, f);
    } else {
      // eight k of one column: two transposing reads of four rows each
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * ROWS * kSize));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// Shape of a workgroup's tile: BM x BN outputs, WM x WN x WK waves.  With WK > 1
// the waves of one output share the contraction's groups in turn and their sums
// are added in LDS at the end, in order: more waves to hide latency behind
// where a small tile leaves the matrix cores idle.
template <class E_, int BM_, int BN_, int WM_, int WN_, int WK_, int STAGES_, int SUB_, bool PCOL_, bool QCOL_>
struct TileShape {
  typedef E_ E;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WK = WK_, kStages = STAGES_, kSub = SUB_;
  static constexpr bool PCOL = PCOL_, QCOL = QCOL_;
  static constexpr int kWaves = WM * WN * WK, kThreads = 64 * kWaves;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // 32 x 32 tiles of a wave
  static constexpr int kPart = 128 / static_cast<int>(sizeof(E));  // contraction elements of a part of a step
  static constexpr int kBuffer = (BM + BN) * 128;             // one part in LDS
  static constexpr int kRing = kStages * kSub * kBuffer;
  static constexpr int kJoin = (WK - 1) * WM * WN * TM * TN * 4096;  // sums of the other waves of an output
  static constexpr int kLds = kRing > kJoin ? kRing : kJoin;
  typedef TileOf<E, BM, PCOL, kWaves> TileP;
  typedef TileOf<E, BN, QCOL, kWaves> TileQ;
  static constexpr int kCopies = kSub * (TileP::kCopies + TileQ::kCopies);  // of a wave and step
  static constexpr int kMine = kSub * TileP::kGroups / WK;                  // groups of a wave and step
  static_assert(kMine >= 1 && kMine * WK == kSub * TileP::kGroups, "the groups of a step must divide among the waves");
};

// Waits until the oldest step under way has arrived, with `newer` steps issued after it.
template <class S, int N = S::kStages - 2>
__device__ __forceinline__ void step_arrived(int newer) {
  if constexpr (N == 0) {
    copies_left<0>();
  } else {
    if (newer >= N) copies_left<N * S::kCopies>();
    else step_arrived<S, N - 1>(newer);
  }
}

// The main loop's state of one wave.
template <class S>
struct TileLoop {
  typedef typename S::E E;
  typedef typename S::TileP TileP;
  typedef typename S::TileQ TileQ;
  static constexpr int kStepBytes = S::kSub * S::kBuffer, kStepK = S::kSub * S::kPart;
  static constexpr int kParts = __is_same(E, Split) ? 2 : 1;  // 16-byte reads of a fragment

  TileP tp;
  TileQ tq;
  uint32_t lp, lq;                      // this wave's share of part 0 in LDS
  uint32_t rp[S::kMine][kParts], rq[S::kMine][kParts];
  int wave, wm, wn;

  __device__ __forceinline__ void init(const Side& P, const Side& Q, uint32_t base) {
    wave = uniform(static_cast<int>(threadIdx.x) / kWave);
    const int wk = S::WK == 1 ? 0 : wave / (S::WM * S::WN), wo = S::WK == 1 ? wave : wave % (S::WM * S::WN);
    wm = wo / S::WN;
    wn = wo % S::WN;
    tp.init(P, wave);
    tq.init(Q, wave);
    lp = base + wave * (TileP::kCopies * 1024);
    lq = base + S::BM * 128 + wave * (TileQ::kCopies * 1024);
#pragma unroll
    for (int n = 0; n < S::kMine; ++n) {
      const int g = n * S::WK + wk, part = g / TileP::kGroups * S::kBuffer;
#pragma unroll
      for (int h = 0; h < kParts; ++h) {
        // the wave's own rows (columns) come in here, the 32 x 32 tiles of the wave on top
        rp[n][h] = TileP::row_offset(TileP::read_offset(g % TileP::kGroups, h), wm * S::TM) + part;
        rq[n][h] = TileQ::row_offset(TileQ::read_offset(g % TileP::kGroups, h), wn * S::TN) + part + S::BM * 128;
      }
    }
  }

  template <int POS, int U = 0>
  __device__ __forceinline__ void copy_step() {
    tp.template copy<POS * kStepBytes + U * S::kBuffer>(lp);
    tq.template copy<POS * kStepBytes + U * S::kBuffer>(lq);
    if constexpr (U + 1 < S::kSub) copy_step<POS, U + 1>();
  }
  // The step that starts at element k of K, into ring position pos: any of it may be past the end.
  __device__ __forceinline__ void copy_edge(int pos, int k, int K) {
#pragma unroll
    for (int u = 0; u < S::kSub; ++u) {
      const uint32_t at = pos * kStepBytes + u * S::kBuffer;
      tp.copy_some(wave, K - k - u * S::kPart, lp + at);
      tq.copy_some(wave, K - k - u * S::kPart, lq + at);
    }
  }

  template <class T>
  static __device__ __forceinline__ typename MfmaType<E>::frag fragment(const char* lds, const uint32_t (&r)[kParts], int t) {
    if constexpr (kParts == 2)
      return {__builtin_bit_cast(f16x8, T::read16(lds + T::row_offset(r[0], t))),
              __builtin_bit_cast(f16x8, T::read16(lds + T::row_offset(r[1], t)))};
    else
      return __builtin_bit_cast(typename MfmaType<E>::frag, T::read16(lds + T::row_offset(r[0], t)));
  }

  // Multiplies the step in LDS at `lds`: the fragments of group n + 1 are read while group n is multiplied.
  __device__ __forceinline__ void multiply(const char* lds, f32x16 (&acc)[S::TM][S::TN]) const {
    typename MfmaType<E>::frag fp[2][S::TM], fq[2][S::TN];
    auto read_group = [&](int n) {
#pragma unroll
      for (int a = 0; a < S::TM; ++a) fp[n & 1][a] = fragment<TileP>(lds, rp[n], a);
#pragma unroll
      for (int b = 0; b < S::TN; ++b) fq[n & 1][b] = fragment<TileQ>(lds, rq[n], b);
    };
    read_group(0);
#pragma unroll
    for (int n = 0; n < S::kMine; ++n) {
      if (n + 1 < S::kMine) read_group(n + 1);
      __builtin_amdgcn_sched_barrier(0);  // keeps the reads ahead of the products they overlap
#pragma unroll
      for (int a = 0; a < S::TM; ++a)
#pragma unroll
        for (int b = 0; b < S::TN; ++b) acc[a][b] = MfmaType<E>::mul(fp[n & 1][a], fq[n & 1][b], acc[a][b]);
    }
  }

  // One step in the middle of the contraction, at ring position POS: all constants known.
  template <int POS>
  __device__ __forceinline__ void middle(const char* lds, f32x16 (&acc)[S::TM][S::TN]) {
    copies_left<(S::kStages - 2) * S::kCopies>();
    __syncthreads();
    copy_step<(POS + S::kStages - 1) % S::kStages>();
    multiply(lds + POS * kStepBytes, acc);
    if constexpr (POS + 1 < S::kStages) middle<POS + 1>(lds, acc);
  }
};

// acc[a][b] += the wave's 32 x 32 tiles of P Q^T over a contraction of length K.
// Every thread of the workgroup calls it.  With WK > 1 the sums are whole in the
// waves of the first WM x WN only (tile_store knows).
template <class S>
__device__ __forceinline__ void tile_products(const Side& P, const Side& Q, int K, char* lds,
                                              f32x16 (&acc)[S::TM][S::TN]) {
  typedef TileLoop<S> Loop;
  Loop loop;
  loop.init(P, Q, lds_address(lds));
  const int steps = (K + Loop::kStepK - 1) / Loop::kStepK, whole = K / Loop::kStepK;
  int copied = 0, from = 0;
  for (; copied < S::kStages - 1 && copied < steps; ++copied) loop.copy_edge(copied, copied * Loop::kStepK, K);
  int left = steps;
  // rounds of the ring whose copies are all whole steps
  for (; copied + S::kStages <= whole; copied += S::kStages, left -= S::kStages) loop.template middle<0>(lds, acc);
  for (; left > 0; --left) {
    step_arrived<S>(left - 1);
    __syncthreads();
    if (copied < steps) {
      loop.copy_edge(copied % S::kStages, copied * Loop::kStepK, K);
      ++copied;
    }
    loop.multiply(lds + from * Loop::kStepBytes, acc);
    from = from + 1 == S::kStages ? 0 : from + 1;
  }
  const int wave = loop.wave;
  const int wk = S::WK == 1 ? 0 : wave / (S::WM * S::WN), wo = S::WK == 1 ? wave : wave % (S::WM * S::WN);
  __syncthreads();
  if constexpr (S::WK > 1) {
    f32x4* part = reinterpret_cast<f32x4*>(lds);
    const int lane = lane_id();
    auto slot = [&](int k, int t, int q) { return (((k * S::WM * S::WN + wo) * S::TM * S::TN + t) * 4 + q) * 64 + lane; };
#pragma unroll
    for (int t = 0; t < S::TM * S::TN; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& v = acc[t / S::TN][t % S::TN];
        if (wk > 0) part[slot(wk - 1, t, q)] = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      }
    __syncthreads();
    if (wk == 0) {
#pragma unroll
      for (int t = 0; t < S::TM * S::TN; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < S::WK - 1; ++k) {
            const f32x4 v = part[slot(k, t, q)];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t / S::TN][t % S::TN][4 * q + e] += v[e];
          }
    }
  }
}

// Calls f(i, j, v) for every accumulator of the wave: element 4 q + e of v is
// row i + 8 q + e, column j (both inside the workgroup's tile).
template <class S, class F>
__device__ __forceinline__ void tile_store(const f32x16 (&acc)[S::TM][S::TN], F f) {
  const int lane = lane_id();
  const int wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  if (S::WK > 1 && wave >= S::WM * S::WN) return;
  const int wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
  for (int a = 0; a < S::TM; ++a)
#pragma unroll
    for (int b = 0; b < S::TN; ++b)
      f((wm * S::TM + a) * 32 + 4 * (lane >> 5), (wn * S::TN + b) * 32 + (lane & 31), acc[a][b]);
}
__device__ __forceinline__ constexpr int acc_row(int v) { return 8 * (v >> 2) + (v & 3); }

// Workgroup b of `count` -> the tile it takes: workgroups go round the 8 XCDs
// in turn, so each XCD gets a contiguous share of the tiles (whose operands its
// L2 then holds), the first `count % 8` of them one more.
__device__ __forceinline__ int xcd_order(int b, int count) {
  const int x = b & 7, n = count >> 3, more = count & 7;
  return x * n + (x < more ? x : more) + (b >> 3);
}

// The output tile (bi, bj) of this workgroup on a grid of rows x cols tiles for
// each matrix of a stack; returns the matrix.  Tiles go in panels of four
// columns, so that an XCD's share is a block, not a strip: fewer rows of both operands.
__device__ __forceinline__ int tile_of(int rows, int cols, int& bi, int& bj) {
  const int all = xcd_order(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
  const int z = all / (rows * cols), t = all % (rows * cols);
  const int panel = t / (4 * rows), in = t % (4 * rows);
  const int width = cols - 4 * panel < 4 ? cols - 4 * panel : 4;
  bi = in / width;
  bj = 4 * panel + in % width;
  return z;
}

}  // namespace lc
