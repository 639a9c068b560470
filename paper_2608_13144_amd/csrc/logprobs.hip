// Log probabilities of rows of logits, their gradient, and distillation from a
// teacher's top logits (see lipcache.h for the formulas).
//
// One workgroup a row.  A row's largest value comes first, then its sums of
// exp((x - max) / temperature), so no sum is ever scaled again; differences to
// the largest value are formed before they are divided, so that logits of the
// type's lowest value stay apart from -inf.
#include "lc_common.hpp"

namespace lc {

constexpr int kLpMostClasses = 1 << 20;
constexpr int kLpMostTop = 64;
constexpr int kLpMostEntries = 1024;
constexpr int kLpThreads = 256;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ float lp_exp2(float v) { return __builtin_amdgcn_exp2f(v); }

// Sum (largest) of a value over the workgroup; every thread gets it.
template <class F>
__device__ __forceinline__ float lp_reduce(float v, float* room, F join) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = join(v, __shfl_xor(v, o, kWave));
  const int wave = static_cast<int>(threadIdx.x) / kWave;
  __syncthreads();
  if (lane_id() == 0) room[wave] = v;
  __syncthreads();
  v = room[0];
#pragma unroll
  for (int w = 1; w < kLpThreads / kWave; ++w) v = join(v, room[w]);
  return v;
}
__device__ __forceinline__ float lp_sum(float v, float* room) {
  return lp_reduce(v, room, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float lp_max(float v, float* room) {
  return lp_reduce(v, room, [](float a, float b) { return fmaxf(a, b); });
}

// What a row's logits come to at one temperature.
struct LpRow {
  float m;       // the largest value, 0 for a row that is -inf throughout
  float scale;   // log2(e) / temperature
  float s;       // sum of exp2(scale (x - m))
  float mean;    // sum of the exponents, weighted by that
};

template <class E>
__device__ __forceinline__ LpRow lp_row(const E* __restrict__ x, int C, float temperature, float* room) {
  LpRow r;
  float m = -kInf;
  for (int j = threadIdx.x; j < C; j += kLpThreads) m = fmaxf(m, static_cast<float>(x[j]));
  m = lp_max(m, room);
  r.m = m == -kInf ? 0.0f : m;
  r.scale = kLog2e / temperature;
  float s = 0.0f, mean = 0.0f;
  for (int j = threadIdx.x; j < C; j += kLpThreads) {
    const float a = (static_cast<float>(x[j]) - r.m) * r.scale, e = lp_exp2(a);
    s += e;
    mean = fmaf(fmaxf(a, -1000.0f), e, mean);
  }
  r.s = lp_sum(s, room);
  r.mean = lp_sum(mean, room);
  return r;
}

struct LpScore {
  float temperature;
  const int32_t* label;
  int k;
  float *logp, *lse, *entropy;
  int32_t* top_index;
  float* top_logp;
};

template <class E>
__global__ __launch_bounds__(kLpThreads) void lp_score_kernel(const E* __restrict__ logits, int64_t ldx, int C, LpScore a) {
  __shared__ float room[kLpThreads / kWave];
  __shared__ int room_i[kLpThreads / kWave];
  const int64_t t = blockIdx.x;
  const E* x = logits + t * ldx;
  const LpRow r = lp_row(x, C, a.temperature, room);
  const float log_s = __log2f(r.s);  // -inf for a row that is -inf throughout
  auto logp = [&](float v) { return r.s == 0.0f ? -kInf : (v - r.m) / a.temperature - log_s * kLn2; };
  if (threadIdx.x == 0) {
    if (a.logp) {
      const int y = a.label ? a.label[t] : -1;
      a.logp[t] = y >= 0 && y < C ? logp(static_cast<float>(x[y])) : 0.0f;
    }
    if (a.lse) a.lse[t] = r.m / a.temperature + log_s * kLn2;
    if (a.entropy) a.entropy[t] = r.s == 0.0f ? 0.0f : (log_s - r.mean / r.s) * kLn2;
  }
  // one alternative after another: the largest below the one before, ties by index
  float last = kInf;
  int last_at = -1;
  for (int i = 0; i < a.k; ++i) {
    float best = -kInf;
    int at = C;
    for (int j = threadIdx.x; j < C; j += kLpThreads) {
      const float v = static_cast<float>(x[j]);
      if ((v < last || (v == last && j > last_at)) && v > best) best = v, at = j;
    }
    const float top = lp_max(best, room);
    if (best != top) at = C;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) at = min(at, __shfl_xor(at, o, kWave));
    __syncthreads();
    if (lane_id() == 0) room_i[threadIdx.x / kWave] = at;
    __syncthreads();
    at = room_i[0];
#pragma unroll
    for (int w = 1; w < kLpThreads / kWave; ++w) at = min(at, room_i[w]);
    if (threadIdx.x == 0) {
      a.top_index[t * a.k + i] = top == -kInf ? -1 : at;
      a.top_logp[t * a.k + i] = top == -kInf ? -kInf : logp(top);
    }
    last = top;
    last_at = at;
  }
}

struct LpBackward {
  float temperature;
  const int32_t* label;
  const float *g_logp, *g_lse, *g_entropy;
  int k;
  const int32_t* top_index;
  const float* g_top;
};

// The entries of a row that name classes, those of one class added up in their order by the first of them.
template <class F>
__device__ __forceinline__ void lp_entries(int k, int C, const int* at, const float* value, F f) {
  for (int i = threadIdx.x; i < k; i += kLpThreads) {
    const int c = at[i];
    if (c < 0) continue;
    bool first = true;
    float sum = 0.0f;
    for (int j = 0; j < k; ++j)
      if (at[j] == c) {
        first = first && j >= i;
        sum += value[j];
      }
    if (first) f(c, sum);
  }
}

template <class E>
__global__ __launch_bounds__(kLpThreads) void lp_backward_kernel(const E* logits, int64_t ldx, int C, LpBackward a,
                                                                 E* out, int64_t ldd) {
  __shared__ float room[kLpThreads / kWave];
  __shared__ int at[kLpMostEntries + 1];
  __shared__ float value[kLpMostEntries + 1];
  const int64_t t = blockIdx.x;
  const E* x = logits + t * ldx;
  E* dx = out + t * ldd;
  const LpRow r = lp_row(x, C, a.temperature, room);
  // the label and the alternatives alike: entries of the row
  float mass = 0.0f;
  int y = a.label && a.g_logp ? a.label[t] : -1;
  if (y >= C) y = -1;
  for (int i = threadIdx.x; i < a.k + 1; i += kLpThreads) {
    int c = i == a.k ? y : a.top_index[t * a.k + i];
    if (c < 0 || c >= C) c = -1;
    const float g = c < 0 ? 0.0f : i == a.k ? a.g_logp[t] : a.g_top[t * a.k + i];
    at[i] = g == 0.0f ? -1 : c;
    value[i] = g;
    mass += g;
  }
  mass = lp_sum(mass, room);
  const float gl = a.g_lse ? a.g_lse[t] : 0.0f, ge = a.g_entropy ? a.g_entropy[t] : 0.0f;
  bool some = mass != 0.0f || gl != 0.0f || ge != 0.0f;
  for (int i = 0; i < a.k + 1; ++i) some = some || at[i] >= 0;
  some = some && r.s != 0.0f;  // (true for NaN)
  const float inv_t = 1.0f / a.temperature, inv_s = 1.0f / r.s, offset = r.mean * inv_s;
  auto smooth = [&](float v) {
    const float e = (v - r.m) * r.scale;
    return lp_exp2(e) * inv_s * (gl - mass - ge * kLn2 * (fmaxf(e, -1000.0f) - offset));
  };
  // entries' values before any is written: out may be x
  float kept[(kLpMostEntries + 1 + kLpThreads - 1) / kLpThreads];
  int n = 0;
  lp_entries(a.k + 1, C, at, value, [&](int c, float g) { kept[n++] = (smooth(static_cast<float>(x[c])) + g) * inv_t; });
  __syncthreads();
  for (int j = threadIdx.x; j < C; j += kLpThreads)
    dx[j] = static_cast<E>(some ? smooth(static_cast<float>(x[j])) * inv_t : 0.0f);
  __syncthreads();
  n = 0;
  if (some) lp_entries(a.k + 1, C, at, value, [&](int c, float) { dx[c] = static_cast<E>(kept[n++]); });
}

struct LpDistill {
  float temperature, hard, soft;
  const int32_t* label;
  const float* weight;
  int k;
  const float* teacher;
  const int32_t* index;
  float *ce, *kl;
};

template <class E>
__global__ __launch_bounds__(kLpThreads) void lp_distill_kernel(const E* logits, int64_t ldx, int C, LpDistill a,
                                                                E* out, int64_t ldd) {
  __shared__ float room[kLpThreads / kWave];
  __shared__ int at[kLpMostEntries + 1];
  __shared__ float value[kLpMostEntries + 1];
  const int64_t t = blockIdx.x;
  const E* x = logits + t * ldx;
  const LpRow hot = lp_row(x, C, a.temperature, room), cold = lp_row(x, C, 1.0f, room);
  int y = a.label ? a.label[t] : -1;
  if (y >= C) y = -1;
  float top = -kInf;
  bool some = false;
  for (int i = threadIdx.x; i < a.k; i += kLpThreads) {
    int c = a.index[t * a.k + i];
    if (c < 0 || c >= C) c = -1;
    at[i] = c;
    value[i] = a.teacher[t * a.k + i];
    if (c >= 0) top = fmaxf(top, value[i]);
    some = some || (c >= 0 && !(value[i] == -kInf));
  }
  top = lp_max(top, room);
  some = lp_max(some ? 1.0f : 0.0f, room) > 0.0f;
  if (top == -kInf) top = 0.0f;
  float sum = 0.0f;
  for (int i = threadIdx.x; i < a.k; i += kLpThreads)
    if (at[i] >= 0) sum += lp_exp2((value[i] - top) * hot.scale);
  sum = lp_sum(sum, room);
  float kl = 0.0f;
  for (int i = threadIdx.x; i < a.k; i += kLpThreads) {
    if (at[i] < 0) continue;
    const float b = value[i] - top, q = some ? lp_exp2(b * hot.scale) / sum : 0.0f;
    if (!(q == 0.0f)) kl += q * ((b - (static_cast<float>(x[at[i]]) - hot.m)) * hot.scale);
    value[i] = q;
  }
  kl = lp_sum(kl, room);
  const float w = a.weight ? a.weight[t] : 1.0f;
  if (threadIdx.x == 0) {
    if (a.ce) {
      const float v = y >= 0 ? static_cast<float>(x[y]) : 0.0f;
      a.ce[t] = y < 0 ? 0.0f : cold.s == 0.0f ? kInf : __log2f(cold.s) * kLn2 - (v - cold.m);
    }
    if (a.kl) a.kl[t] = !some ? 0.0f : hot.s == 0.0f ? kInf : (kl + __log2f(hot.s) - __log2f(sum)) * kLn2;
    at[a.k] = y;
    value[a.k] = 0.0f;
  }
  if (!out) return;
  const float hard = y >= 0 ? w * a.hard : 0.0f, soft = some ? w * a.soft / a.temperature : 0.0f;
  const bool any = (hard != 0.0f || soft != 0.0f) && cold.s != 0.0f;
  __syncthreads();
  for (int i = threadIdx.x; i <= a.k; i += kLpThreads) {
    if (i == a.k) value[i] = hard;
    else if (at[i] >= 0) value[i] *= soft;
    if (value[i] == 0.0f) at[i] = -1;
  }
  __syncthreads();
  const float hot_s = soft / hot.s, cold_s = hard / cold.s;
  auto smooth = [&](float v) {
    float g = 0.0f;
    if (soft != 0.0f) g += lp_exp2((v - hot.m) * hot.scale) * hot_s;
    if (hard != 0.0f) g += lp_exp2((v - cold.m) * cold.scale) * cold_s;
    return g;
  };
  E* dx = out + t * ldd;
  float kept[(kLpMostEntries + 1 + kLpThreads - 1) / kLpThreads];
  int n = 0;
  lp_entries(a.k + 1, C, at, value, [&](int c, float q) { kept[n++] = smooth(static_cast<float>(x[c])) - q; });
  __syncthreads();
  for (int j = threadIdx.x; j < C; j += kLpThreads) dx[j] = static_cast<E>(any ? smooth(static_cast<float>(x[j])) : 0.0f);
  __syncthreads();
  n = 0;
  if (any) lp_entries(a.k + 1, C, at, value, [&](int c, float) { dx[c] = static_cast<E>(kept[n++]); });
}

// ------------------------------------------------------------- validation
bool lp_unaligned(const void* p, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & (dtype == LIPCACHE_F32 ? 3u : 1u)) != 0;
}
bool lp_unaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

lipcache_status lp_check(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype, float temperature) {
  if (T < 0 || C < 1 || ldx < C || dtype < LIPCACHE_F32 || dtype > LIPCACHE_F16) return LIPCACHE_EINVAL;
  if (!(temperature >= 0x1p-20f && temperature <= 0x1p20f)) return LIPCACHE_EINVAL;
  if ((T > 0 && !x) || lp_unaligned(x, dtype)) return LIPCACHE_EINVAL;
  if (C > kLpMostClasses || T > 0x7fffffff) return LIPCACHE_EUNSUPPORTED;
  return LIPCACHE_OK;
}

// Rows of a launch: fewer than 2^32 threads.
constexpr int64_t kLpPass = 1 << 23;
template <class F>
lipcache_status lp_passes(int64_t T, F launch) {
  for (int64_t t = 0; t < T; t += kLpPass) {
    launch(t, static_cast<unsigned>(T - t < kLpPass ? T - t : kLpPass));
    LC_LAUNCHED();
  }
  return LIPCACHE_OK;
}

template <class F>
lipcache_status lp_typed(int32_t dtype, F f) {
  switch (dtype) {
    case LIPCACHE_F32: return f(float{});
    case LIPCACHE_BF16: return f(__bf16{});
    default: return f(_Float16{});
  }
}

template <class T>
T* lp_at(T* p, int64_t i) {
  return p ? p + i : nullptr;
}

}  // namespace lc

using namespace lc;

extern "C" lipcache_status lipcache_logprobs(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                             float temperature, const int32_t* label, int32_t k, float* logp,
                                             float* lse, float* entropy, int32_t* top_index, float* top_logp,
                                             lipcache_stream_t stream) {
  if (lipcache_status st = lp_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || (T > 0 && k > 0 && (!top_index || !top_logp))) return LIPCACHE_EINVAL;
  if (lp_unaligned4(label) || lp_unaligned4(logp) || lp_unaligned4(lse) || lp_unaligned4(entropy) ||
      lp_unaligned4(top_index) || lp_unaligned4(top_logp))
    return LIPCACHE_EINVAL;
  if (k > kLpMostTop) return LIPCACHE_EUNSUPPORTED;
  return lp_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    return lp_passes(T, [&](int64_t t, unsigned n) {
      const LpScore a{temperature, lp_at(label, t), k, lp_at(logp, t), lp_at(lse, t), lp_at(entropy, t),
                      lp_at(top_index, t * k), lp_at(top_logp, t * k)};
      lp_score_kernel<E><<<n, kLpThreads, 0, stream>>>(static_cast<const E*>(x) + t * ldx, ldx, C, a);
    });
  });
}

extern "C" lipcache_status lipcache_logprobs_backward(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                                      float temperature, const int32_t* label, const float* g_logp,
                                                      const float* g_lse, const float* g_entropy, int32_t k,
                                                      const int32_t* top_index, const float* g_top, void* dx,
                                                      int64_t lddx, lipcache_stream_t stream) {
  if (lipcache_status st = lp_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || lddx < C || (T > 0 && !dx) || (T > 0 && k > 0 && (!top_index || !g_top)) || (g_logp && !label))
    return LIPCACHE_EINVAL;
  if (lp_unaligned(dx, dtype) || lp_unaligned4(label) || lp_unaligned4(g_logp) || lp_unaligned4(g_lse) ||
      lp_unaligned4(g_entropy) || lp_unaligned4(top_index) || lp_unaligned4(g_top))
    return LIPCACHE_EINVAL;
  if (k > kLpMostEntries) return LIPCACHE_EUNSUPPORTED;
  return lp_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    return lp_passes(T, [&](int64_t t, unsigned n) {
      const LpBackward a{temperature, lp_at(label, t), lp_at(g_logp, t), lp_at(g_lse, t), lp_at(g_entropy, t), k,
                         lp_at(top_index, t * k), lp_at(g_top, t * k)};
      lp_backward_kernel<E><<<n, kLpThreads, 0, stream>>>(static_cast<const E*>(x) + t * ldx, ldx, C, a,
                                                         static_cast<E*>(dx) + t * lddx, lddx);
    });
  });
}

extern "C" lipcache_status lipcache_distill(const void* x, int64_t ldx, int64_t T, int32_t C, int32_t dtype,
                                            float temperature, float hard, float soft, int32_t k,
                                            const float* teacher, const int32_t* index, const int32_t* label,
                                            const float* weight, float* ce, float* kl, void* dx, int64_t lddx,
                                            lipcache_stream_t stream) {
  if (lipcache_status st = lp_check(x, ldx, T, C, dtype, temperature); st != LIPCACHE_OK) return st;
  if (k < 0 || (dx && lddx < C) || (T > 0 && k > 0 && (!teacher || !index))) return LIPCACHE_EINVAL;
  if (!(__builtin_fabsf(hard) < kInf) || !(__builtin_fabsf(soft) < kInf)) return LIPCACHE_EINVAL;
  if (lp_unaligned(dx, dtype) || lp_unaligned4(teacher) || lp_unaligned4(index) || lp_unaligned4(label) ||
      lp_unaligned4(weight) || lp_unaligned4(ce) || lp_unaligned4(kl))
    return LIPCACHE_EINVAL;
  if (k > kLpMostEntries) return LIPCACHE_EUNSUPPORTED;
  return lp_typed(dtype, [&](auto type) {
    typedef decltype(type) E;
    return lp_passes(T, [&](int64_t t, unsigned n) {
      const LpDistill a{temperature, hard, soft, lp_at(label, t), lp_at(weight, t), k,
                        lp_at(teacher, t * k), lp_at(index, t * k), lp_at(ce, t), lp_at(kl, t)};
      lp_distill_kernel<E><<<n, kLpThreads, 0, stream>>>(static_cast<const E*>(x) + t * ldx, ldx, C, a,
                                                        dx ? static_cast<E*>(dx) + t * lddx : nullptr, lddx);
    });
  });
}
