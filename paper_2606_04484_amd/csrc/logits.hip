// Rows of logits: their k largest as log-probs (what a teacher hands over), and the
// loss of a student's rows against such lists, with its gradient.
//
// Every row is one pass of 16-byte loads over [vocab] values; nothing is reused, so
// the floor is the bytes of the logits (and of d logits).  A row need not start at a
// 16-byte boundary: its values are numbered from the boundary before it (u = v + shift),
// so that every thread's run of 16 bytes is aligned and only the row's first and last runs
// are guarded value by value.
#include <algorithm>
#include "ops.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLog2eD = 1.4426950408889634074, kLn2D = 0.69314718055994530942;
constexpr int kMaxK = 256;

// 2^x on the hardware unit for x <= 0 or -inf (values under 2^-126 come out 0)
AJ_DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T> constexpr int kRun = 16 / sizeof(T);   // values of a 16-byte run

template <typename V> AJ_DEV V wave_max(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
  return v;
}
template <typename V> AJ_DEV V wave_sum(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// A row's values by u = v + shift; runs start at multiples of kRun.
template <typename T>
struct Row {
  const T *aligned;   // the run boundary at or before the row's first value
  int shift, end;     // values are at u in [shift, end)
  AJ_DEV Row(const void *base, int64_t row, int64_t ld, int vocab) {
    const T *p = (const T *)base + row * ld;
    shift = (int)(((uintptr_t)p & 15) / sizeof(T));
    aligned = p - shift;
    end = vocab + shift;
  }
  // the run at u as loaded; values outside the row are -inf
  struct Bits { uint4 w; };
  AJ_DEV Bits load(int u) const {
    Bits b;
    if (u >= shift && u + kRun<T> <= end) {
      b.w = *reinterpret_cast<const uint4 *>(aligned + u);
    } else {
      uint32_t w[4] = {};
#pragma unroll
      for (int j = 0; j < kRun<T>; ++j) {
        const bool in = u + j >= shift && u + j < end;
        if constexpr (sizeof(T) == 4)
          w[j] = in ? ((const uint32_t *)aligned)[u + j] : 0xff800000u;
        else
          w[j / 2] |= (in ? (uint32_t)aligned[u + j] : 0xff80u) << (16 * (j & 1));
      }
      b.w = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return b;
  }
  AJ_DEV static void values(const Bits &b, float (&z)[kRun<T>]) {
    const uint32_t w[4] = {b.w.x, b.w.y, b.w.z, b.w.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] = __uint_as_float(w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        z[2 * j] = __uint_as_float(w[j] << 16);
        z[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
};

// ------------------------------------------------------------------ top k
// Order of values: larger first, equal ones (-0 and 0 among them) by the lower index, NaN
// before all.  A value's place is one 64-bit number, its order-keeping bits above the
// complement of its index, so that no two are equal.
AJ_DEV uint32_t order_bits(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return z != z ? 0xffffffffu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
AJ_DEV uint64_t place(float z, int v) { return (uint64_t)order_bits(z) << 32 | (uint32_t)~v; }
AJ_DEV float order_value(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

constexpr int kTopNT = 512, kTopWaves = kTopNT / 64;
constexpr int kTopCap = 2048;    // candidates kept in LDS

// The sum of v over the workgroup, in every thread.
AJ_DEV int block_sum(int v, int *red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  int s = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += red[w];
  return s;
}

// The kk-th largest of the places that `count(t)`, the number at or above t in this
// thread, tells of.
template <typename F>
AJ_DEV uint64_t kth_place(int kk, int *red, F count) {
  uint64_t t = 0;
  for (int b = 63; b >= 0; --b) {
    const uint64_t c = t | (uint64_t)1 << b;
    if (block_sum(count(c), red) >= kk) t = c;
  }
  return t;
}

// Largest to smallest: out[r] = the place with r larger ones among the n of c (LDS), r < kk
AJ_DEV void write_ranked(const uint64_t *c, int n, int kk, uint64_t *out) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const uint64_t mine = c[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += c[j] > mine;
    if (r < kk) out[r] = mine;
  }
}

// One workgroup per part of a row: kTopNT * E values held in registers.  Gives
// the part's k largest places in order (0 after the last), its maximum and its sum of
// exp2((z - max) c).
//
// A threshold that at least k values reach comes from the threads' maxima: in every
// wave the ceil(k / 8)-th largest of its 64 (a bisection over the bits with one ballot
// a step, to 20 bits: a lower threshold is as right), and of these the smallest.  The
// values at or above it, about k of them, are ranked by counting.  Where equal values
// or a NaN break that, a bisection over the places finds the k-th itself.
template <typename T, int E>
__global__ __launch_bounds__(kTopNT) void topk_part_kernel(const void *logits, int64_t ld, int vocab,
                                                           int parts, int k, float c,
                                                           uint64_t *cand, float2 *ms) {
  constexpr int R = kRun<T>, Q = E / R;
  __shared__ uint64_t list[kTopCap];
  __shared__ float red_m[kTopWaves], red_s[kTopWaves];
  __shared__ uint32_t red_t[kTopWaves];
  __shared__ int red_i[kTopWaves], n_list;
  const int64_t row = blockIdx.x / parts;
  const int part = blockIdx.x % parts;
  const Row<T> x(logits, row, ld, vocab);
  const int u0 = part * kTopNT * E + threadIdx.x * R;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  typename Row<T>::Bits b[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) b[q] = x.load(u0 + q * kTopNT * R);
  float z[E];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    float t[R];
    Row<T>::values(b[q], t);
#pragma unroll
    for (int j = 0; j < R; ++j) z[q * R + j] = t[j];
  }
  auto index = [&](int e) { return u0 + (e / R) * kTopNT * R + e % R - x.shift; };
  auto inside = [&](int e) { return (unsigned)index(e) < (unsigned)vocab; };
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) m = fmaxf(m, z[e]);
  // the wave's threshold
  const uint32_t mo = order_bits(m);
  const int j = (k + kTopWaves - 1) / kTopWaves;
  uint32_t t = 0;
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t try_t = t | 1u << bit;
    if (__popcll(__builtin_amdgcn_ballot_w64(mo >= try_t)) >= j) t = try_t;
  }
  const float wm = wave_max(m);
  if (threadIdx.x == 0) n_list = 0;
  if (lane == 0) {
    red_m[wave] = wm;
    red_t[wave] = t;
  }
  __syncthreads();
  float M = red_m[0];
  t = red_t[0];
#pragma unroll
  for (int w = 1; w < kTopWaves; ++w) {
    M = fmaxf(M, red_m[w]);
    t = min(t, red_t[w]);
  }
  // the partial log-sum-exp, and the candidates
  const float base = M == -INFINITY ? 0.f : M;
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) s += fast_exp2((z[e] - base) * c);
  const float tau = t <= order_bits(-INFINITY) ? -INFINITY : order_value(t);
  int mine = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) mine += inside(e) & (z[e] >= tau);
  int at = mine;      // inclusive prefix over the wave, then the wave's place in the list
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(at, o, 64);
    if (lane >= o) at += v;
  }
  int first = 0;
  if (lane == 63) first = atomicAdd(&n_list, at);
  at += __shfl(first, 63, 64) - mine;
  s = wave_sum(s);
  if (lane == 0) red_s[wave] = s;
  __syncthreads();
  float S = 0.f;
#pragma unroll
  for (int w = 0; w < kTopWaves; ++w) S += red_s[w];
  if (threadIdx.x == 0) ms[blockIdx.x] = make_float2(M, S);
  uint64_t *out = cand + (int64_t)blockIdx.x * k;
  const int lo = part * kTopNT * E, kk =
      max(0, min(k, min(x.end, lo + kTopNT * E) - max(x.shift, lo)));
  int n = n_list;
  uint64_t least = 0;
  // S is NaN where a NaN (or +inf, whose own difference is one) is among the values
  const bool listed = n >= kk && n <= kTopCap && S == S;
  if (!listed) {
    least = kth_place(kk, red_i, [&](uint64_t p) {
      int cnt = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) cnt += inside(e) & (place(z[e], index(e)) >= p);
      return cnt;
    });
    __syncthreads();
    if (threadIdx.x == 0) n_list = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (inside(e) & (place(z[e], index(e)) >= least)) list[atomicAdd(&n_list, 1)] = place(z[e], index(e));
    n = kk;
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (inside(e) & (z[e] >= tau)) list[at++] = place(z[e], index(e));
  }
  __syncthreads();
  write_ranked(list, n, kk, out);
  for (int i = kk + threadIdx.x; i < k; i += kTopNT) out[i] = 0;
}

// One workgroup per row joins its parts' lists and log-sum-exps.  A threshold that k
// candidates reach: the ceil(k / parts)-th of every part, the smallest of them, or the
// k-th of any one part.
constexpr int kMergeNT = 256;
template <typename T>
__global__ __launch_bounds__(kMergeNT) void topk_merge_kernel(const void *logits, int64_t ld,
                                                              int vocab, int parts, int k,
                                                              double c, const uint64_t *cand,
                                                              const float2 *ms, int32_t *idx,
                                                              float *logprob, float *lse) {
  __shared__ uint64_t list[kTopCap], least[kMergeNT / 64], most[kMergeNT / 64], ranked[kMaxK];
  __shared__ double red[kMergeNT / 64];
  __shared__ float red_m[kMergeNT / 64];
  __shared__ int red_i[kMergeNT / 64], n_list;
  const int64_t row = blockIdx.x;
  const uint64_t *in = cand + row * parts * k;
  const float2 *p = ms + row * parts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_in = parts * k;
  const int j = (k + parts - 1) / parts;
  uint64_t lo = ~(uint64_t)0, hi = 0;
  float M = -INFINITY;
  for (int q = threadIdx.x; q < parts; q += kMergeNT) {
    lo = min(lo, in[(int64_t)q * k + j - 1]);
    hi = max(hi, in[(int64_t)q * k + k - 1]);
    M = fmaxf(M, p[q].x);
  }
  lo = ~wave_max(~lo);
  hi = wave_max(hi);
  M = wave_max(M);
  if (threadIdx.x == 0) n_list = 0;
  if (lane == 0) least[wave] = lo, most[wave] = hi, red_m[wave] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kMergeNT / 64; ++w) {
    lo = min(lo, least[w]);
    hi = max(hi, most[w]);
    M = fmaxf(M, red_m[w]);
  }
  uint64_t t = max(lo, hi);
  // the row's log-sum-exp in 64 bits from the parts' sums
  double s = 0.0;
  for (int q = threadIdx.x; q < parts; q += kMergeNT)
    s += p[q].x == -INFINITY && p[q].y == 0.f ? 0.0 : (double)p[q].y * exp2(((double)p[q].x - M) * c);
  s = wave_sum(s);
  if (lane == 0) red[wave] = s;
  int cnt = 0;
  for (int i = threadIdx.x; i < n_in; i += kMergeNT) cnt += in[i] >= t && in[i] != 0;
  cnt = block_sum(cnt, red_i);
  s = 0.0;
#pragma unroll
  for (int w = 0; w < kMergeNT / 64; ++w) s += red[w];
  const double l = M == -INFINITY && s == 0.0 ? -INFINITY : (M * c + log2(s)) * kLn2D;
  if (cnt > kTopCap)
    t = kth_place(k, red_i, [&](uint64_t v) {
      int n = 0;
      for (int i = threadIdx.x; i < n_in; i += kMergeNT) n += in[i] >= v;
      return n;
    });
  for (int i = threadIdx.x; i < n_in; i += kMergeNT)
    if (in[i] >= t && in[i] != 0) list[atomicAdd(&n_list, 1)] = in[i];
  __syncthreads();
  write_ranked(list, n_list, k, ranked);
  __syncthreads();
  for (int i = threadIdx.x; i < k; i += kMergeNT) {
    const int v = (int)~(uint32_t)ranked[i];
    const double z = ldf((const T *)logits + row * ld + v);
    idx[row * k + i] = v;
    // a row of nothing but -inf has no probabilities: -inf for each
    logprob[row * k + i] = l == -INFINITY ? -INFINITY : (float)(z * (c * kLn2D) - l);
  }
  if (threadIdx.x == 0) lse[row] = (float)l;
}

// ------------------------------------------------------------------ distillation
constexpr int kNT = 256, kWaves = kNT / 64;
constexpr int kQ = 4;                // 16-byte runs a thread has in flight
constexpr int kSplit = 65536;        // values of a row per workgroup at most: 8 KB of bits

struct Teacher {
  int k, tail;
  const int32_t *idx;
  const float *logprob, *weight;
  float coef;
};

// A row's list in LDS, one entry per thread (k <= kNT): entries that are unused
// (negative), outside the vocabulary or repeated count for nothing.
struct Listed {
  int v;          // -1: nothing
  double p;       // the teacher's probability (tail 0: renormalised over the list)
  double logp;
  double mass, rest;   // of the whole row: sum of p and what is left of 1 (tail 1)
};

AJ_DEV double block_sum(double v, double *red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += red[w];
  return s;
}

AJ_DEV Listed listed(const Teacher &t, int64_t row, int vocab, int32_t *err, int *ids, double *red) {
  const int i = threadIdx.x;
  Listed e;
  e.v = -1;
  double lp = -INFINITY;
  int raw = -1;
  if (i < t.k) {
    raw = t.idx[row * t.k + i];
    lp = t.logprob[row * t.k + i];
  }
  ids[i] = raw;
  __syncthreads();
  if (raw >= vocab) {
    if (err) atomicOr(err, AJ_DEVERR_TOKEN_RANGE);
  } else if (raw >= 0) {
    bool again = false;
    for (int j = 0; j < i; ++j) again |= ids[j] == raw;
    if (!again) e.v = raw;
    else if (err) atomicOr(err, AJ_DEVERR_TOKEN_TWICE);
  }
  if (e.v < 0) lp = -INFINITY;
  if (t.tail) {
    e.logp = lp;
    e.p = exp(lp);
    e.mass = block_sum(e.p, red);
    // (a NaN stays one)
    e.rest = e.mass > 1.0 ? 0.0 : 1.0 - e.mass;
    e.mass += e.rest;
  } else {
    double m = wave_max(lp);
    __syncthreads();
    if ((i & 63) == 0) red[i >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = max(m, red[w]);
    const double ex = lp == -INFINITY ? 0.0 : exp(lp - m);
    const double s = block_sum(ex, red);
    e.p = s == 0.0 ? 0.0 : ex / s;
    e.logp = lp - m - log(s);
    e.mass = s == 0.0 ? 0.0 : 1.0;
    e.rest = 0.0;
  }
  return e;
}

// One bit per value of u in [u0, u0 + kSplit): whether the list names it.
AJ_DEV void mark(uint32_t *bits, int v, int shift, int vocab, int u0, int u1) {
  if (v < 0 || v >= vocab) return;
  const int u = v + shift;
  if (u >= u0 && u < u1) atomicOr(&bits[(u - u0) >> 5], 1u << ((u - u0) & 31));
}

// One workgroup per part [u0, u1) of a row: maximum and sum of exp2((z - max) c) of the
// values that the list does not name.
template <typename T>
__global__ __launch_bounds__(kNT) void distill_part_kernel(const void *logits, int64_t ld, int vocab,
                                                           int parts, int width, Teacher t, float c,
                                                           float2 *ms) {
  constexpr int R = kRun<T>, kStep = kNT * R * kQ;
  __shared__ uint32_t bits[kSplit / 32];
  __shared__ float red_m[kWaves], red_s[kWaves];
  const int64_t row = blockIdx.x / parts;
  const Row<T> x(logits, row, ld, vocab);
  const int u0 = blockIdx.x % parts * width, u1 = min(u0 + width, x.end);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  typename Row<T>::Bits b[kQ];
  auto fetch = [&](int u) {
#pragma unroll
    for (int q = 0; q < kQ; ++q) b[q] = x.load(u + (q * kNT + threadIdx.x) * R);
  };
  fetch(u0);
  for (int i = threadIdx.x; i < width / 32; i += kNT) bits[i] = 0;
  __syncthreads();
  if ((int)threadIdx.x < t.k) mark(bits, t.idx[row * t.k + threadIdx.x], x.shift, vocab, u0, u1);
  __syncthreads();
  float m = -INFINITY, s = 0.f;
  for (int u = u0; u < u1; u += kStep) {
    float z[kQ * R];
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      float v[R];
      Row<T>::values(b[q], v);
      const int at = u - u0 + (q * kNT + threadIdx.x) * R;
      uint32_t w = 0;
      if (u0 + at < u1) w = bits[at >> 5] >> (at & 31);
      const bool in = u0 + at < u1;
#pragma unroll
      for (int j = 0; j < R; ++j) z[q * R + j] = (w >> j & 1) | !in ? -INFINITY : v[j];
    }
    if (u + kStep < u1) fetch(u + kStep);
    float n = m;
#pragma unroll
    for (int e = 0; e < kQ * R; ++e) n = fmaxf(n, z[e]);
    const float base = n == -INFINITY ? 0.f : n;
    s *= m == -INFINITY ? 0.f : fast_exp2((m - base) * c);
    m = n;
#pragma unroll
    for (int e = 0; e < kQ * R; ++e) s += fast_exp2((z[e] - base) * c);
  }
  float M = wave_max(m);
  if (lane == 0) red_m[wave] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, red_m[w]);
  // (0 times an infinity, of a thread that has met +inf, is the NaN it should be)
  s = wave_sum(m == -INFINITY ? s : s * fast_exp2((m - M) * c));
  if (lane == 0) red_s[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) ms[blockIdx.x] = make_float2(M, red_s[0] + red_s[1] + red_s[2] + red_s[3]);
}

// One workgroup per row: joins the parts, adds the list's own values, and forms the loss.
template <typename T>
__global__ __launch_bounds__(kNT) void distill_row_kernel(const void *logits, int64_t ld, int vocab,
                                                          int rows, int parts, Teacher t, double inv_temp,
                                                          const float2 *ms, float *loss, float *lse,
                                                          int32_t *err) {
  __shared__ int ids[kNT];
  __shared__ double red[kWaves];
  const int64_t row = blockIdx.x;
  const Listed e = listed(t, row, vocab, err, ids, red);
  const double c = inv_temp * kLog2eD;
  const double z = e.v >= 0 ? (double)ldf((const T *)logits + row * ld + e.v) : -INFINITY;
  const float2 *p = ms + row * parts;
  double M = -INFINITY;
  for (int q = threadIdx.x; q < parts; q += kNT) M = max(M, (double)p[q].x);
  auto block_max = [&](double v) {
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v = max(v, red[w]);
    return v;
  };
  M = block_max(M);
  double s = 0.0;
  for (int q = threadIdx.x; q < parts; q += kNT)
    s += p[q].x == -INFINITY && p[q].y == 0.f ? 0.0 : (double)p[q].y * exp2(((double)p[q].x - M) * c);
  s = block_sum(s, red);
  const double rest = s == 0.0 ? -INFINITY : (M * c + log2(s)) * kLn2D;   // of the others
  const double mz = block_max(z);
  const double sz = block_sum(z == -INFINITY ? 0.0 : exp2((z - mz) * c), red);
  const double list = sz == 0.0 ? -INFINITY : (mz * c + log2(sz)) * kLn2D;
  const double hi = max(rest, list);
  double all = rest + list;     // NaN where one is
  if (all == all || hi == -INFINITY)
    all = hi == -INFINITY ? -INFINITY : hi + log(exp(rest - hi) + exp(list - hi));
  double term = 0.0;
  if (e.p > 0.0 || e.p != e.p) term = e.p * (e.logp - (z * inv_temp - all));
  term = block_sum(term, red);
  if (t.tail && e.rest > 0.0) term += e.rest * (log(e.rest) - (rest - all));
  if (threadIdx.x == 0) {
    loss[row] = (float)term;
    lse[row] = (float)all;
    lse[rows + row] = (float)rest;
  }
}

// stats[0] += sum of coef * weight * loss, stats[1] += rows, in one fixed order
__global__ __launch_bounds__(1024) void distill_stats_kernel(const float *loss, const float *weight,
                                                             int rows, float coef, float *stats) {
  __shared__ double red[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < rows; i += 1024) s += (double)coef * (weight ? weight[i] : 1.f) * loss[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 16; ++w) s += red[w];
    stats[0] += (float)s;
    stats[1] += (float)rows;
  }
}

// d logits of one part of a row.  A value that the list does not name gets
// exp(z' - lse_rest) F with F = w (mass q_rest - rest), q_rest = exp(lse_rest - lse) (tail
// 1), or exp(z' - lse) w mass (tail 0); a named one w (mass q - p).
template <typename T, typename G>
__global__ __launch_bounds__(kNT) void distill_bwd_kernel(const void *logits, int64_t ld, int vocab,
                                                          int rows, int parts, int width, Teacher t,
                                                          double inv_temp, const float *lse, G *dz,
                                                          int64_t ldd) {
  constexpr int R = kRun<T>, kStep = kNT * R * kQ;
  __shared__ int ids[kNT];
  __shared__ double red[kWaves];
  const int64_t row = blockIdx.x / parts;
  const Row<T> x(logits, row, ld, vocab);
  const int u0 = blockIdx.x % parts * width, u1 = min(u0 + width, x.end);
  typename Row<T>::Bits b[kQ];
  auto fetch = [&](int u) {
#pragma unroll
    for (int q = 0; q < kQ; ++q) b[q] = x.load(u + (q * kNT + threadIdx.x) * R);
  };
  fetch(u0);
  const Listed e = listed(t, row, vocab, nullptr, ids, red);
  const double all = lse[row], others = lse[rows + row];
  const double w = (double)t.coef * inv_temp * (t.weight ? t.weight[row] : 1.f);
  // this part's named values, read before any is written (d logits may be the logits)
  const bool mine = e.v >= 0 && e.v + x.shift >= u0 && e.v + x.shift < u1;
  float named = 0.f;
  if (mine) {
    const double z = ldf((const T *)logits + row * ld + e.v);
    named = e.mass == 0.0 ? 0.f : (float)(w * (e.mass * exp(z * inv_temp - all) - e.p));
  }
  __syncthreads();
  const double L = t.tail ? others : all;
  const float L2 = L == -INFINITY ? 0.f : (float)(L * kLog2eD), c = (float)(inv_temp * kLog2eD);
  const float F = (float)(t.tail ? w * (e.mass * exp(others - all) - e.rest) : w * e.mass);
  const bool none = e.mass == 0.0;     // nothing listed: no loss, no gradient
  G *out = dz + row * ldd - x.shift;
  // runs are stored whole where d logits is aligned as the runs are
  const bool vec = ((uintptr_t)out & (R * sizeof(G) - 1)) == 0 || ((uintptr_t)out & 15) == 0;
  for (int u = u0; u < u1; u += kStep) {
    float g[kQ][R];
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      Row<T>::values(b[q], g[q]);
#pragma unroll
      for (int j = 0; j < R; ++j) g[q][j] = none ? 0.f : fast_exp2(fmaf(g[q][j], c, -L2)) * F;
    }
    if (u + kStep < u1) fetch(u + kStep);
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      const int at = u + (q * kNT + threadIdx.x) * R;
      if (at >= u1) continue;
      if (vec && at >= x.shift && at + R <= x.end) {
        if constexpr (sizeof(G) == 4) {
#pragma unroll
          for (int j = 0; j < R; j += 4)
            *reinterpret_cast<float4 *>(out + at + j) = make_float4(g[q][j], g[q][j + 1], g[q][j + 2], g[q][j + 3]);
        } else if constexpr (R == 4) {
          *reinterpret_cast<uint2 *>(out + at) = make_uint2(f2bf2(g[q][0], g[q][1]), f2bf2(g[q][2], g[q][3]));
        } else {
          *reinterpret_cast<uint4 *>(out + at) =
              make_uint4(f2bf2(g[q][0], g[q][1]), f2bf2(g[q][2], g[q][3]), f2bf2(g[q][4], g[q][5]),
                         f2bf2(g[q][6], g[q][7]));
        }
      } else {
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (at + j >= x.shift && at + j < x.end) stf(out + at + j, g[q][j]);
      }
    }
  }
  __syncthreads();    // the named ones over what the runs left there
  if (mine) stf(out + e.v + x.shift, named);
}

// ------------------------------------------------------------------ host
// Room for the parts' results is asked for so that a workspace sized for some rows serves
// fewer: `full` parts a row, or, where small numbers of rows are cut finer (`fine` parts a
// row at most), the `most` of them that this ever gives.
size_t part_room(int64_t rows, int64_t full, int64_t fine, int64_t most) {
  return (size_t)std::max(rows * full, std::min(rows * fine, most));
}

struct TopWs {
  uint64_t *cand;
  float2 *ms;
  int parts, per_thread;
  size_t bytes;
};

// Values per thread of the part kernel: 32 (16384 a part); fewer where the rows are
// too few to give every CU a part.
int top_per_thread(int rows, int vocab) {
  int e = 32;
  while (e > 8 && (int64_t)rows * ((vocab + kTopNT * e - 1) / (kTopNT * e)) < 256) e /= 2;
  return e;
}

TopWs carve_top(int rows, int vocab, int k, void *base) {
  aj::Carver cv(base);
  TopWs w;
  w.per_thread = top_per_thread(rows, vocab);
  // a row that starts past a run boundary reaches at most 7 values further
  auto parts = [&](int e) { return (vocab + 7 + kTopNT * e - 1) / (kTopNT * e); };
  w.parts = parts(w.per_thread);
  // finer parts are taken from under 256 in all, and at most double them and one a row
  const size_t room = part_room(rows, parts(32), parts(8), 768);
  w.cand = cv.take<uint64_t>(room * k);
  w.ms = cv.take<float2>(room);
  w.bytes = cv.bytes();
  return w;
}

struct Split { int parts, width; };
// Parts of a row: kSplit values at most, fewer until 2048 workgroups run, 2048 at least.
Split row_split(int rows, int vocab) {
  int width = kSplit;
  while (width > 2048 && (int64_t)rows * ((vocab + width - 1) / width) < 2048) width /= 2;
  return {(vocab + 7 + width - 1) / width, width};
}

int check_logits(const aj_logits *lg, const char *name) {
  AJ_REQUIRE(lg, AJ_ERR_NULL, "%s: null logits", name);
  AJ_REQUIRE(lg->dtype == AJ_F32 || lg->dtype == AJ_BF16, AJ_ERR_UNSUPPORTED, "%s: dtype %d", name,
             lg->dtype);
  AJ_REQUIRE(lg->rows >= 0 && lg->vocab > 0 && lg->vocab <= 1 << 24 && lg->ld >= lg->vocab, AJ_ERR_SHAPE,
             "%s: rows %d vocab %d (at most 2^24) ld %lld", name, lg->rows, lg->vocab, (long long)lg->ld);
  AJ_REQUIRE(lg->inv_temp > 0.f && lg->inv_temp <= 1e30f, AJ_ERR_SHAPE, "%s: inv_temp %g", name,
             (double)lg->inv_temp);
  AJ_REQUIRE((int64_t)lg->rows * (lg->vocab / 2048 + 2) < (int64_t)1 << 31, AJ_ERR_SHAPE,
             "%s: rows %d of vocab %d", name, lg->rows, lg->vocab);
  AJ_REQUIRE(lg->rows == 0 || lg->logits, AJ_ERR_NULL, "%s: null logits", name);
  AJ_REQUIRE(((uintptr_t)lg->logits & (lg->dtype == AJ_BF16 ? 1 : 3)) == 0, AJ_ERR_SHAPE,
             "%s: logits between elements", name);
  return AJ_OK;
}

int check_teacher(const aj_logits *lg, const aj_teacher *t, const char *name) {
  AJ_REQUIRE(t, AJ_ERR_NULL, "%s: null teacher", name);
  AJ_REQUIRE(t->k >= 1 && t->k <= kMaxK, AJ_ERR_SHAPE, "%s: k %d (1..%d)", name, t->k, kMaxK);
  AJ_REQUIRE(lg->rows == 0 || (t->idx && t->logprob), AJ_ERR_NULL, "%s: null list", name);
  return AJ_OK;
}

Teacher teacher_of(const aj_teacher &t) {
  return {t.k, t.tail != 0, t.idx, t.logprob, t.weight, t.coef};
}

template <typename T>
void launch_topk(const aj_logits &lg, int k, int32_t *idx, float *logprob, float *lse, const TopWs &w,
                 hipStream_t st) {
  const float c = lg.inv_temp * kLog2e;
  const unsigned grid = (unsigned)lg.rows * w.parts;
  if (w.per_thread == 32)
    topk_part_kernel<T, 32><<<grid, kTopNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, w.parts, k, c, w.cand, w.ms);
  else if (w.per_thread == 16)
    topk_part_kernel<T, 16><<<grid, kTopNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, w.parts, k, c, w.cand, w.ms);
  else
    topk_part_kernel<T, 8><<<grid, kTopNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, w.parts, k, c, w.cand, w.ms);
  topk_merge_kernel<T><<<lg.rows, kMergeNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, w.parts, k,
                                                     lg.inv_temp * kLog2eD, w.cand, w.ms, idx, logprob, lse);
}

template <typename T>
void launch_loss(const aj_logits &lg, const aj_teacher &t, float *loss, float *lse, float *stats,
                 int32_t *err, float2 *ms, hipStream_t st) {
  const Split s = row_split(lg.rows, lg.vocab);
  distill_part_kernel<T><<<(unsigned)lg.rows * s.parts, kNT, 0, st>>>(
      lg.logits, lg.ld, lg.vocab, s.parts, s.width, teacher_of(t), lg.inv_temp * kLog2e, ms);
  distill_row_kernel<T><<<lg.rows, kNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, lg.rows, s.parts, teacher_of(t),
                                                 lg.inv_temp, ms, loss, lse, err);
  if (stats) distill_stats_kernel<<<1, 1024, 0, st>>>(loss, t.weight, lg.rows, t.coef, stats);
}

template <typename T>
void launch_grad(const aj_logits &lg, const aj_teacher &t, const float *lse, void *dz, int64_t ldd,
                 int d_dtype, hipStream_t st) {
  const Split s = row_split(lg.rows, lg.vocab);
  const unsigned grid = (unsigned)lg.rows * s.parts;
  if (d_dtype == AJ_BF16)
    distill_bwd_kernel<T, bf16_t><<<grid, kNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, lg.rows, s.parts, s.width,
                                                        teacher_of(t), lg.inv_temp, lse, (bf16_t *)dz, ldd);
  else
    distill_bwd_kernel<T, float><<<grid, kNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, lg.rows, s.parts, s.width,
                                                       teacher_of(t), lg.inv_temp, lse, (float *)dz, ldd);
}

size_t distill_ws(int rows, int vocab) {
  auto parts = [&](int width) { return (vocab + 7 + width - 1) / width; };
  aj::Carver cv(nullptr);
  // (as above: halved from under 2048)
  cv.take<float2>(part_room(rows, parts(kSplit), parts(2048), 3 * 2048));
  return cv.bytes();
}

int check_grad(const aj_logits *lg, const void *dz, int64_t ldd, int d_dtype, const char *name) {
  AJ_REQUIRE(d_dtype == AJ_F32 || d_dtype == AJ_BF16, AJ_ERR_UNSUPPORTED, "%s: d logits dtype %d", name, d_dtype);
  AJ_REQUIRE(ldd >= lg->vocab, AJ_ERR_SHAPE, "%s: d logits ld %lld", name, (long long)ldd);
  AJ_REQUIRE(dz || lg->rows == 0, AJ_ERR_NULL, "%s: null d logits", name);
  AJ_REQUIRE(((uintptr_t)dz & (d_dtype == AJ_BF16 ? 1 : 3)) == 0, AJ_ERR_SHAPE, "%s: d logits between elements", name);
  AJ_REQUIRE(dz != lg->logits || (d_dtype == lg->dtype && ldd == lg->ld), AJ_ERR_SHAPE,
             "%s: d logits in the logits' place need their type and ld", name);
  return AJ_OK;
}

}  // namespace

extern "C" size_t aj_topk_workspace_bytes(int32_t rows, int32_t vocab, int32_t k) {
  if (rows < 0 || vocab <= 0 || k <= 0) return 0;
  return carve_top(rows, vocab, k, nullptr).bytes;
}

extern "C" int aj_topk_logprob(const aj_logits *lg, int32_t k, int32_t *idx, float *logprob, float *lse,
                               void *ws, size_t ws_bytes, void *stream) {
  const char *name = "aj_topk_logprob";
  if (int r = check_logits(lg, name)) return r;
  AJ_REQUIRE(k >= 1 && k <= kMaxK && k <= lg->vocab, AJ_ERR_SHAPE, "%s: k %d (1..%d, at most vocab)", name, k, kMaxK);
  if (lg->rows == 0) return AJ_OK;
  AJ_REQUIRE(idx && logprob && lse && ws, AJ_ERR_NULL, "%s: null pointer", name);
  const TopWs w = carve_top(lg->rows, lg->vocab, k, ws);
  AJ_REQUIRE(ws_bytes >= w.bytes, AJ_ERR_WORKSPACE, "%s: workspace %zu < %zu", name, ws_bytes, w.bytes);
  hipStream_t st = (hipStream_t)stream;
  if (lg->dtype == AJ_BF16) launch_topk<bf16_t>(*lg, k, idx, logprob, lse, w, st);
  else launch_topk<float>(*lg, k, idx, logprob, lse, w, st);
  return aj::check_launch(name);
}

extern "C" size_t aj_distill_workspace_bytes(int32_t rows, int32_t vocab, int32_t k) {
  if (rows < 0 || vocab <= 0 || k <= 0) return 0;
  return distill_ws(rows, vocab);
}

extern "C" int aj_distill_loss_fwd(const aj_logits *lg, const aj_teacher *t, float *loss, float *lse,
                                   float *stats, int32_t *err, void *ws, size_t ws_bytes, void *stream) {
  const char *name = "aj_distill_loss_fwd";
  int r;
  if ((r = check_logits(lg, name)) || (r = check_teacher(lg, t, name))) return r;
  if (lg->rows == 0) return AJ_OK;
  AJ_REQUIRE(loss && lse && ws, AJ_ERR_NULL, "%s: null pointer", name);
  const size_t need = distill_ws(lg->rows, lg->vocab);
  AJ_REQUIRE(ws_bytes >= need, AJ_ERR_WORKSPACE, "%s: workspace %zu < %zu", name, ws_bytes, need);
  hipStream_t st = (hipStream_t)stream;
  float2 *ms = aj::Carver(ws).take<float2>(1);
  if (lg->dtype == AJ_BF16) launch_loss<bf16_t>(*lg, *t, loss, lse, stats, err, ms, st);
  else launch_loss<float>(*lg, *t, loss, lse, stats, err, ms, st);
  return aj::check_launch(name);
}

extern "C" int aj_distill_loss_bwd(const aj_logits *lg, const aj_teacher *t, const float *lse, void *dlogits,
                                   int64_t ldd, int32_t d_dtype, void *stream) {
  const char *name = "aj_distill_loss_bwd";
  int r;
  if ((r = check_logits(lg, name)) || (r = check_teacher(lg, t, name)) ||
      (r = check_grad(lg, dlogits, ldd, d_dtype, name)))
    return r;
  if (lg->rows == 0) return AJ_OK;
  AJ_REQUIRE(lse, AJ_ERR_NULL, "%s: null lse", name);
  hipStream_t st = (hipStream_t)stream;
  if (lg->dtype == AJ_BF16) launch_grad<bf16_t>(*lg, *t, lse, dlogits, ldd, d_dtype, st);
  else launch_grad<float>(*lg, *t, lse, dlogits, ldd, d_dtype, st);
  return aj::check_launch(name);
}

extern "C" int aj_distill_loss_fwd_bwd(const aj_logits *lg, const aj_teacher *t, float *loss, float *lse,
                                       float *stats, int32_t *err, void *dlogits, int64_t ldd,
                                       int32_t d_dtype, void *ws, size_t ws_bytes, void *stream) {
  const char *name = "aj_distill_loss_fwd_bwd";
  int r;
  if ((r = check_logits(lg, name)) || (r = check_teacher(lg, t, name)) ||
      (r = check_grad(lg, dlogits, ldd, d_dtype, name)))
    return r;
  if ((r = aj_distill_loss_fwd(lg, t, loss, lse, stats, err, ws, ws_bytes, stream))) return r;
  return aj_distill_loss_bwd(lg, t, lse, dlogits, ldd, d_dtype, stream);
}
