// Rows of logits: their k largest as log-probs (what a teacher hands over), and the
// loss of a student's rows against such lists, with its gradient.
//
// Every row is one pass of 16-byte loads over [vocab] values; nothing is reused, so
// the floor is the bytes of the logits (and of d logits).  A row need not start at a
// 16-byte boundary: its values are numbered from the boundary before it (u = v + shift),
// so that every thread's run of 16 bytes is aligned and only the row's first and last runs
// are guarded value by value.
#include <cfloat>
#include <algorithm>
#include <type_traits>
#include "ops.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLog2eD = 1.4426950408889634074;
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

// Sums of 2^((z - m) c) over values z, m the largest of them.  The unit is a value and not
// its product with c, which finite values may take out of float32's range (a vocabulary masked
// with the lowest value, a low temperature); and the difference is formed of halves, as that
// of two finite values may be.  c2 = 2 c, c = inv_temp log2(e).
AJ_DEV float half_unit(float m) { return m == -INFINITY ? 0.f : 0.5f * m; }
AJ_DEV float below(float z, float half, float c2) { return fmaf(z, 0.5f, -half) * c2; }
// s of unit m in the unit `half` (of a value not below m); a NaN stays one
AJ_DEV float in_unit(float m, float s, float half, float c2) {
  return m == -INFINITY ? (s == s ? 0.f : s) : s * fast_exp2(below(m, half, c2));
}
struct RunSum {
  float m = -INFINITY, s = 0.f;
  // the values z, the largest of which is `top`
  template <int N> AJ_DEV void add(const float (&z)[N], float top, float c2) {
    const float up = fmaxf(m, top), half = half_unit(up);
    s = in_unit(m, s, half, c2);
    m = up;
#pragma unroll
    for (int e = 0; e < N; ++e) s += fast_exp2(below(z[e], half, c2));
  }
  template <int N> AJ_DEV void add(const float (&z)[N], float c2) {
    float top = z[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
    add(z, top, c2);
  }
};
// Parts' sums (m, s) in 64 bits, one wave's or one thread's share of them: in the unit M.
AJ_DEV double part_in_unit(float2 p, double M, double c) {
  return p.x == -INFINITY && p.y == 0.f ? 0.0 : (double)p.y * exp2(((double)p.x - M) * c);
}

// A natural log of a sum as unit + log, apart: the unit may be so large that their sum leaves
// nothing of log.  log -inf: the sum of nothing.
struct LogSum {
  double unit, log;
  AJ_DEV bool none() const { return log == -INFINITY; }
};
AJ_DEV LogSum log_of(double m, double s, double inv_temp) { return {m == -INFINITY ? 0.0 : m * inv_temp, log(s)}; }
AJ_DEV LogSum join(const LogSum &a, const LogSum &b) {
  if (a.none()) return b;
  if (b.none()) return a;
  const double hi = max(a.unit, b.unit);
  return {hi, log(exp(a.unit - hi + a.log) + exp(b.unit - hi + b.log))};
}
// log of a's sum over b's
AJ_DEV double log_ratio(const LogSum &a, const LogSum &b) { return (a.unit - b.unit) + (a.log - b.log); }
// as a result: -inf of nothing only
AJ_DEV float as_float(const LogSum &a) {
  const double v = a.unit + a.log;
  return a.none() ? -INFINITY : v != v ? (float)v : (float)min(max(v, -(double)FLT_MAX), (double)FLT_MAX);
}

// LDS writes (or reads) complete, then a barrier.  __syncthreads would wait for the loads
// of the next values too, which are to be on their way meanwhile (top k of 4096 rows of 152064
// float32: 702 us with it).
AJ_DEV void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
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
  // the run at u if it lies in the row as a whole, else all -inf: what that leaves out
  // are the values before the row's first and behind its last boundary, `rim` by number
  AJ_DEV Bits whole(int u) const {
    Bits b;
    if (u >= shift && u + kRun<T> <= end) b.w = *reinterpret_cast<const uint4 *>(aligned + (uint32_t)u);
    else b.w.x = b.w.y = b.w.z = b.w.w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return b;
  }
  // u of rim value i in [0, 2 kRun), or -1
  AJ_DEV int rim(int i) const {
    const int last = max(end & -kRun<T>, shift > 0 ? kRun<T> : 0);   // (one run may hold both ends)
    const int u = i < kRun<T> ? i : last + i - kRun<T>;
    return (i < kRun<T> ? shift > 0 && u >= shift : i < 2 * kRun<T>) && u < end ? u : -1;
  }
  // N runs of a thread, `stride` values apart from u + at on; [u, u + span) holds all threads'
  template <int N> AJ_DEV void load(Bits (&b)[N], int u, int at, int stride, int span) const {
    if (u >= shift && u + span <= end) {
      const T *p = aligned + u;
#pragma unroll
      for (int q = 0; q < N; ++q) b[q].w = *reinterpret_cast<const uint4 *>(p + (uint32_t)(q * stride + at));
    } else {
#pragma unroll
      for (int q = 0; q < N; ++q) b[q] = load(u + q * stride + at);
    }
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
// before all.  A value's place is one number, its order-keeping bits above the
// complement of its index, so that no two are equal.
constexpr uint32_t kNaNOrder = 0xff800001u;      // +inf's and one
constexpr int kIndexBits = 24;                      // vocab <= 2^24
constexpr uint64_t kAbove = (uint64_t)(kNaNOrder + 1) << kIndexBits;     // above every place
AJ_DEV uint32_t order_bits(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return z != z ? kNaNOrder : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
AJ_DEV uint64_t place(float z, int v) {
  return (uint64_t)order_bits(z) << kIndexBits | (~(uint32_t)v & ((1u << kIndexBits) - 1));
}
AJ_DEV int place_index(uint64_t p) { return (int)(~(uint32_t)p & ((1u << kIndexBits) - 1)); }
// the value of such bits (-inf for bits below its own)
AJ_DEV float order_value(uint32_t o) {
  return o <= 0x007fffffu ? -INFINITY : __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

constexpr int kTopNT = 256, kTopWaves = kTopNT / 64;
// Values a thread holds at a time.  32 would be 1.5 % faster on 4096 rows of 152064 float32 (448
// against 456 us) but slower on 3000 of 151936 bfloat16 (264 against 224), whose rate is that
// of the instructions: more of these waves fit a SIMD.
constexpr int kTopValues = 16, kTopChunk = kTopNT * kTopValues;
constexpr int kWaveHold = 5, kWaveCap = 64 * kWaveHold;    // candidates a wave keeps in LDS
constexpr int kRankPad = 16;
constexpr int kSlack = 64;       // over k that a last cut may leave to the ranking

// A threshold in [lo, hi) that kk places reach and no more than `most`, where kk and more
// reach lo and fewer hi; `count(t)` tells how many of its wave do.  (A bisection: places
// are spread, so where `most` leaves some room a dozen steps find one; that equal values
// are told apart by their indices alone takes 24 more.)
template <typename F>
AJ_DEV uint64_t kth_place(int kk, int most, uint64_t lo, uint64_t hi, int (*red)[kTopWaves], F count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int slot = 0;      // (three in turn: one barrier a step)
  lds_barrier();
  for (uint64_t t = lo;; t = lo + (hi - lo) / 2) {
    const int mine = count(t);
    if (lane == 0) red[slot][wave] = mine;
    lds_barrier();
    const int n = __builtin_amdgcn_readfirstlane(red[slot][0] + red[slot][1] + red[slot][2] + red[slot][3]);
    slot = slot == 2 ? 0 : slot + 1;
    if (n >= kk) lo = t;
    else hi = t;
    if ((n >= kk && n <= most) || hi - lo <= 1) break;
  }
  return lo;
}

// Candidates met by a workgroup: a list in LDS per wave, which it alone appends to and cuts,
// so that no atomic is waited for; n is its own wave's length.
struct WaveList {
  uint64_t *at;
  int n;
  // those lanes' places that reach `least`; nothing is lost but what is past kWaveCap,
  // which n tells of
  AJ_DEV void add(uint64_t p, uint64_t least) {
    const bool hit = p >= least;
    const uint64_t b = __builtin_amdgcn_ballot_w64(hit);
    const int i = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0));
    if (hit && i < kWaveCap) at[i] = p;
    n += __popcll(b);
  }
  AJ_DEV uint64_t get(int h) const {
    const int i = h * 64 + (threadIdx.x & 63);
    return i < n ? at[i] : 0;
  }
  AJ_DEV void keep(uint64_t least) {
    uint64_t v[kWaveHold];
#pragma unroll
    for (int h = 0; h < kWaveHold; ++h) v[h] = get(h);
    n = 0;
#pragma unroll
    for (int h = 0; h < kWaveHold; ++h) add(v[h], least);
  }
};

// The sum over the waves of what each gives (the barrier also ends what they did in LDS).
AJ_DEV int waves_sum(int v, int *red) {
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  lds_barrier();
  return __builtin_amdgcn_readfirstlane(red[0] + red[1] + red[2] + red[3]);
}

// Cuts the lists to the kk largest of their places, of which all reach lo, and some next
// ones, `most` in all; the return value is a threshold that these reach and no other.
AJ_DEV uint64_t cut(WaveList &l, int kk, int most, uint64_t lo, int (*red)[kTopWaves]) {
  uint64_t v[kWaveHold];
  uint32_t largest = 0;
#pragma unroll
  for (int h = 0; h < kWaveHold; ++h) {
    v[h] = l.get(h);
    largest = max(largest, (uint32_t)(v[h] >> kIndexBits));
  }
  largest = wave_max(largest);
  lds_barrier();
  if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = (int)largest;
  lds_barrier();
  uint32_t hi = 0;
#pragma unroll
  for (int w = 0; w < kTopWaves; ++w) hi = max(hi, (uint32_t)red[0][w]);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const uint64_t t = kth_place(kk, most, max(lo, (uint64_t)1), (uint64_t)(hi + 1) << kIndexBits, red,
                               [&](uint64_t p) {
    int c = 0;
#pragma unroll
    for (int h = 0; h < kWaveHold; ++h) c += __popcll(__builtin_amdgcn_ballot_w64(v[h] >= p));
    return c;
  });
  l.n = 0;
#pragma unroll
  for (int h = 0; h < kWaveHold; ++h) l.add(v[h], t);
  return t;
}

// Largest to smallest: out[r] (LDS) = the place with r larger ones in the waves' lists, r < kk.
// Every thread counts for candidates of its own, 16 of the others at a time: as many LDS
// reads in flight cover each other's latency.  The time goes with the square of the
// number, so longer lists are cut first.
AJ_DEV void write_ranked(const WaveList &l, uint64_t (*lists)[kWaveCap + kRankPad], int kk, uint64_t *out,
                         int *red) {
  const int lane = threadIdx.x & 63;
  if (lane < kRankPad) l.at[l.n + lane] = 0;
  lds_barrier();
  waves_sum(l.n, red);
  int r[kWaveHold] = {};
  uint64_t mine[kWaveHold];
#pragma unroll
  for (int h = 0; h < kWaveHold; ++h) mine[h] = l.get(h);
  for (int w = 0; w < kTopWaves; ++w) {
    const int n = __builtin_amdgcn_readfirstlane(red[w]);
    for (int j = 0; j < n; j += kRankPad) {
      ulonglong2 v[kRankPad / 2];
#pragma unroll
      for (int q = 0; q < kRankPad / 2; ++q) v[q] = *reinterpret_cast<const ulonglong2 *>(lists[w] + j + 2 * q);
#pragma unroll
      for (int h = 0; h < kWaveHold; ++h) {
        if (h * 64 >= l.n) break;
#pragma unroll
        for (int q = 0; q < kRankPad / 2; ++q) r[h] += (int)(v[q].x > mine[h]) + (int)(v[q].y > mine[h]);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < kWaveHold; ++h)
    if (h * 64 + lane < l.n && r[h] < kk) out[r[h]] = mine[h];
}

// A row's results from its k largest places and its log-sum-exp.
template <typename T>
AJ_DEV void write_row(const void *logits, int64_t ld, int64_t row, int k, double inv_temp, const uint64_t *ranked,
                      const LogSum &l, int32_t *idx, float *logprob, float *lse) {
  const int i = threadIdx.x;
  if (i < k) {
    const int id = place_index(ranked[i]);
    const double z = ldf((const T *)logits + row * ld + id);
    idx[row * k + i] = id;
    // a row of nothing but -inf has no probabilities: -inf for each
    logprob[row * k + i] = l.none() ? -INFINITY : (float)((z * inv_temp - l.unit) - l.log);
  }
  if (i == 0) lse[row] = as_float(l);
}

// One workgroup per part [u0, u0 + width) of a row, kTopChunk values at a time, the next
// ones on their way meanwhile.  Gives the part's k largest places in order (0 after the
// last), and its sum of 2^((z - m) c) with m.
//
// Values not below a threshold that k of those met so far reach go to a list in LDS.
// The first threshold comes from the threads' maxima (two each): in every wave the
// ceil(k / 4)-th largest of its 128 (a bisection over the bits with ballots, to 20 bits:
// a lower threshold is as right), and of these the smallest.  Later ones are the k-th
// of the list (or one a little lower), which is cut whenever twice k and more are in it, so
// that of a long row few values pass.  Where too many pass all the same (equal values, NaN,
// which is never below), a bisection over the places finds the k-th itself.
template <typename T>
__global__ __launch_bounds__(kTopNT, 5) void topk_part_kernel(
    const void *logits, int64_t ld, int vocab, int parts, int width, int k, float inv_temp, uint64_t *cand,
    float2 *ms, int32_t *idx, float *logprob, float *lse) {
  constexpr int E = kTopValues, R = kRun<T>, Q = E / R, C = kTopNT * E;
  __shared__ __attribute__((aligned(16))) uint64_t lists[kTopWaves][kWaveCap + kRankPad];
  __shared__ uint64_t ranked[kMaxK];
  __shared__ float red_m[kTopWaves], red_s[kTopWaves];
  __shared__ uint32_t red_t[kTopWaves];
  __shared__ int red_i[3][kTopWaves], red_n[3][kTopWaves];
  const float c2 = 2.f * inv_temp * kLog2e;
  const int64_t row = blockIdx.x / parts;
  const int part = blockIdx.x % parts;
  const Row<T> x(logits, row, ld, vocab);
  const int u0 = part * width, u1 = min(u0 + width, x.end);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  typename Row<T>::Bits b[Q];
  auto fetch = [&](int u) __attribute__((always_inline)) {
    if (u >= x.shift && u + C <= x.end) {
      const T *p = x.aligned + u;
#pragma unroll
      for (int q = 0; q < Q; ++q) b[q].w = *reinterpret_cast<const uint4 *>(p + (q * kTopNT + threadIdx.x) * R);
    } else {
#pragma unroll
      for (int q = 0; q < Q; ++q) b[q] = x.whole(u + (q * kTopNT + threadIdx.x) * R);
    }
  };
  fetch(u0);
  // the row's rim goes with its first part, a value for each of some threads
  const int rim = part == 0 && threadIdx.x < 2 * R ? x.rim(threadIdx.x) : -1;
  const float zr = rim >= 0 ? ldf(x.aligned + rim) : -INFINITY;
  WaveList list{lists[wave], 0};
  uint64_t least = 0;         // the least place that goes to a list
  float tau = -INFINITY;      // ... and its value
  RunSum sum;
  int turn = 0;
  for (int u = u0; u < u1; u += C) {
    float z[E];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      float t[R];
      Row<T>::values(b[q], t);
#pragma unroll
      for (int j = 0; j < R; ++j) z[q * R + j] = t[j];
    }
    if (u + C < u1) fetch(u + C);
    const bool first = u == u0;
    float top[Q], m0 = first ? zr : -INFINITY, m1 = -INFINITY;       // top: of each run
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      top[q] = z[q * R];
#pragma unroll
      for (int j = 1; j < R; ++j) top[q] = fmaxf(top[q], z[q * R + j]);
      if (q & 1) m1 = fmaxf(m1, top[q]);
      else m0 = fmaxf(m0, top[q]);
    }
    sum.add(z, fmaxf(m0, m1), c2);
    if (first) {
      sum.s += fast_exp2(below(zr, half_unit(sum.m), c2));
      const uint32_t o0 = order_bits(m0), o1 = order_bits(m1);
      const int j = (k + kTopWaves - 1) / kTopWaves;
      uint32_t t = 0;
      for (int bit = 31; bit >= 12; --bit) {
        const uint32_t v = t | 1u << bit;
        if (__popcll(__builtin_amdgcn_ballot_w64(o0 >= v)) + __popcll(__builtin_amdgcn_ballot_w64(o1 >= v)) >= j)
          t = v;
      }
      if (lane == 0) red_t[wave] = t;
      lds_barrier();
      t = min(min(red_t[0], red_t[1]), min(red_t[2], red_t[3]));
      t = __builtin_amdgcn_readfirstlane(t);
      tau = order_value(t);
      least = (uint64_t)t << kIndexBits;
    }
    // the place of value e, 0 outside the row
    const int at0 = u + (int)threadIdx.x * R - x.shift;
    auto place_of = [&](int e) {
      // through copies that the compiler does not see into, or it forms every place ahead
      // of the loops that want them, for which there are no registers
      float ze = z[e];
      int a = at0;
      asm volatile("" : "+v"(ze), "+v"(a));
      const int v = a + (e / R) * kTopNT * R + e % R;
      const int ur = v - e % R + x.shift;      // its run; the rim is not among them
      return ur >= x.shift && ur + R <= x.end ? place(ze, v) : 0;
    };
    const uint64_t pr = first && rim >= 0 ? place(zr, rim - x.shift) : 0;
    // a thread whose sum is NaN has met a NaN (which no maximum shows) or +inf: it
    // looks at all it holds
    float bar = sum.s == sum.s ? tau : -INFINITY;
    int had = list.n, n;
    for (;;) {
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (__builtin_amdgcn_ballot_w64(!(top[q] < bar))) {
#pragma unroll
          for (int j = 0; j < R; ++j)
            if (__builtin_amdgcn_ballot_w64(!(z[q * R + j] < bar))) list.add(place_of(q * R + j), max(least, (uint64_t)1));
        }
      if (first) list.add(pr, max(least, (uint64_t)1));
      // (a list that is too long counts for more than all may hold)
      n = waves_sum(list.n > kWaveCap ? kTopWaves * kWaveCap + 1 : list.n, red_n[turn]);
      turn = turn == 2 ? 0 : turn + 1;
      if (n <= kTopWaves * kWaveCap) break;
      // too many: again with the k-th place of the lists as they were and these values
      list.n = had;
      least = kth_place(k, k, 1, kAbove, red_i, [&](uint64_t p) {
        int cnt = __popcll(__builtin_amdgcn_ballot_w64(pr >= p));
#pragma unroll
        for (int h = 0; h < kWaveHold; ++h) cnt += __popcll(__builtin_amdgcn_ballot_w64(list.get(h) >= p));
#pragma unroll
        for (int e = 0; e < E; ++e) cnt += __popcll(__builtin_amdgcn_ballot_w64(place_of(e) >= p));
        return cnt;
      });
      list.keep(least);
      had = list.n;
      tau = order_value((uint32_t)(least >> kIndexBits));
      bar = -INFINITY;
    }
    if (n >= 2 * k + 64 && u + C < u1) {
      least = cut(list, k, k + k / 4 + 32, least, red_i);
      tau = order_value((uint32_t)(least >> kIndexBits));
    }
  }
  // (the barrier ends the reads of this turn's sum)
  lds_barrier();
  const int n = waves_sum(list.n, red_n[0]);
  if (n > k + 128) cut(list, k, k + kSlack, least, red_i);
  const float wm = wave_max(sum.m);
  if (lane == 0) red_m[wave] = wm;
  __syncthreads();
  const float M = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
  const float s = wave_sum(in_unit(sum.m, sum.s, half_unit(M), c2));
  if (lane == 0) red_s[wave] = s;
  if ((int)threadIdx.x < k) ranked[threadIdx.x] = 0;
  write_ranked(list, lists, k, ranked, red_i[0]);
  __syncthreads();
  const float S = red_s[0] + red_s[1] + red_s[2] + red_s[3];
  if (parts == 1) {
    write_row<T>(logits, ld, row, k, inv_temp, ranked, log_of(M, S, inv_temp), idx, logprob, lse);
    return;
  }
  if ((int)threadIdx.x < k) cand[(int64_t)blockIdx.x * k + threadIdx.x] = ranked[threadIdx.x];
  if (threadIdx.x == 0) ms[blockIdx.x] = make_float2(M, S);
}

// One workgroup per row joins its parts' lists and log-sum-exps.  A threshold that k
// candidates reach: the ceil(k / parts)-th of every part, the smallest of them, or the
// k-th of any one part.
// The candidates are read once, into registers (kMergeHold a thread hold all there
// can be).
constexpr int kMergeNT = 256, kMergeWaves = kMergeNT / 64, kMergeHold = 16;
constexpr int kMaxCand = kMergeNT * kMergeHold;
template <typename T>
__global__ __launch_bounds__(kMergeNT) void topk_merge_kernel(const void *logits, int64_t ld,
                                                              int vocab, int parts, int k,
                                                              double inv_temp, const uint64_t *cand,
                                                              const float2 *ms, int32_t *idx,
                                                              float *logprob, float *lse) {
  __shared__ __attribute__((aligned(16))) uint64_t lists[kTopWaves][kWaveCap + kRankPad];
  __shared__ uint64_t least[kMergeWaves], most[kMergeWaves], first[kMergeWaves], ranked[kMaxK];
  __shared__ double red[kMergeWaves];
  __shared__ float red_m[kMergeWaves];
  __shared__ int red_i[3][kMergeWaves];
  static_assert(kMergeWaves == kTopWaves && kMaxK + kSlack <= kWaveCap, "the waves' lists");
  const int64_t row = blockIdx.x;
  const uint64_t *in = cand + row * parts * k;
  const float2 *p = ms + row * parts;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_in = parts * k;
  uint64_t v[kMergeHold];
#pragma unroll
  for (int h = 0; h < kMergeHold; ++h) {
    const int i = h * kMergeNT + threadIdx.x;
    v[h] = i < n_in ? in[i] : 0;
  }
  const int j = (k + parts - 1) / parts;
  uint64_t lo = ~(uint64_t)0, hi = 0, top = 0;
  float M = -INFINITY;
  for (int q = threadIdx.x; q < parts; q += kMergeNT) {
    lo = min(lo, in[(int64_t)q * k + j - 1]);
    hi = max(hi, in[(int64_t)q * k + k - 1]);
    top = max(top, in[(int64_t)q * k]);
    M = fmaxf(M, p[q].x);
  }
  lo = ~wave_max(~lo);
  hi = wave_max(hi);
  top = wave_max(top);
  M = wave_max(M);
  if (lane == 0) least[wave] = lo, most[wave] = hi, first[wave] = top, red_m[wave] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kMergeWaves; ++w) {
    lo = min(lo, least[w]);
    hi = max(hi, most[w]);
    top = max(top, first[w]);
    M = fmaxf(M, red_m[w]);
  }
  uint64_t t = max(max(lo, hi), (uint64_t)1);   // (0 is no place)
  // the row's log-sum-exp in 64 bits from the parts' sums
  double s = 0.0;
  for (int q = threadIdx.x; q < parts; q += kMergeNT) s += part_in_unit(p[q], M, inv_temp * kLog2eD);
  s = wave_sum(s);
  if (lane == 0) red[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < kMergeWaves; ++w) s += red[w];
  t = kth_place(k, k + kSlack, t, top + 1, red_i, [&](uint64_t p) {
    int n = 0;
#pragma unroll
    for (int h = 0; h < kMergeHold; ++h) n += __popcll(__builtin_amdgcn_ballot_w64(v[h] >= p));
    return n;
  });
  WaveList list{lists[wave], 0};
#pragma unroll
  for (int h = 0; h < kMergeHold; ++h) list.add(v[h], t);
  lds_barrier();
  write_ranked(list, lists, k, ranked, red_i[0]);
  __syncthreads();
  write_row<T>(logits, ld, row, k, inv_temp, ranked, log_of(M, s, inv_temp), idx, logprob, lse);
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
  double mass, rest;   // of the whole row: sum of p, and of that what is left of 1 (tail 1)
};

template <int WAVES> AJ_DEV double block_sum(double v, double *red) {
  v = wave_sum(v);
  lds_barrier();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  lds_barrier();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) s += red[w];
  return s;
}
template <int WAVES> AJ_DEV double block_max(double v, double *red) {
  v = wave_max(v);
  lds_barrier();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  lds_barrier();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) v = max(v, red[w]);
  return v;
}

// (threads past the k-th hold nothing; the entries sit in the first kMaxK threads)
template <int WAVES>
AJ_DEV Listed listed(const Teacher &t, int64_t row, int vocab, int32_t *err, int *ids, double *red) {
  const int i = threadIdx.x;
  Listed e;
  e.v = -1;
  double lp = -INFINITY;
  int raw = -1;
  if (i < t.k) {
    raw = t.idx[row * t.k + i];
    lp = t.logprob[row * t.k + i];
    ids[i] = raw;
  }
  lds_barrier();
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
    e.p = lp == -INFINITY ? 0.0 : exp(lp);
    e.mass = block_sum<WAVES>(e.p, red);
    // (a NaN stays one)
    e.rest = e.mass > 1.0 ? 0.0 : 1.0 - e.mass;
    e.mass += e.rest;
  } else {
    const double m = block_max<WAVES>(lp, red);
    const double ex = lp == -INFINITY ? 0.0 : exp(lp - m);
    const double s = block_sum<WAVES>(ex, red);
    e.p = s == 0.0 ? 0.0 : ex / s;
    e.logp = e.p == 0.0 ? -INFINITY : lp - m - log(s);   // (most waves hold no entry)
    e.mass = s == 0.0 ? 0.0 : 1.0;
    e.rest = 0.0;
  }
  return e;
}

// Of a row's named values: their log-sum-exp and sum p (log p - (z inv_temp - its unit)).
// (Known before the others' sum is: what comes after that is on every row's critical path.)
struct NamedSums { LogSum list; double term; };
template <int WAVES>
AJ_DEV NamedSums named_sums(const Listed &e, double z, double inv_temp, double *red) {
  const double top = block_max<WAVES>(z, red), m = top == -INFINITY ? 0.0 : top;
  const double sz = block_sum<WAVES>(z == -INFINITY ? 0.0 : exp2((z - m) * (inv_temp * kLog2eD)), red);
  double term = 0.0;
  if (e.p > 0.0 || e.p != e.p) term = e.p * (e.logp - (z - m) * inv_temp);
  return {log_of(m, sz, inv_temp), block_sum<WAVES>(term, red)};
}

// What a teacher's float32 log-probs leave of 1 by their rounding, at most: half a step each, and
// the error of the log-sum-exp they share (some 600 of 2^-24).
constexpr double kListRounding = 1.0 / 16384;
// Where the student has nothing outside the list, that much there is no class of the teacher's:
// its divergence would be infinite or not as the roundings fall.
AJ_DEV void settle(Listed &e, const LogSum &rest) {
  if (rest.none() && e.rest <= kListRounding) {
    e.mass -= e.rest;
    e.rest = 0.0;
  }
}

// A row's log-sum-exps, of all values and of those not named, and its loss; in one wave.
// ms: the sums of the values not named, with their units.
struct RowSums { LogSum all, rest; double loss; };
AJ_DEV RowSums row_sums(Listed e, const NamedSums &n, const float2 *ms, int parts, double inv_temp) {
  const int lane = threadIdx.x & 63;
  RowSums r;
  float M = -INFINITY;
  for (int q = lane; q < parts; q += 64) M = fmaxf(M, ms[q].x);
  M = wave_max(M);
  double s = 0.0;
  for (int q = lane; q < parts; q += 64) s += part_in_unit(ms[q], M, inv_temp * kLog2eD);
  r.rest = log_of(M, wave_sum(s), inv_temp);
  r.all = join(r.rest, n.list);
  settle(e, r.rest);
  r.loss = n.term;
  const double p = e.mass - e.rest;
  if (p != 0.0) r.loss += p * ((r.all.unit - n.list.unit) + r.all.log);
  if (e.rest > 0.0) r.loss += e.rest * (log(e.rest) - log_ratio(r.rest, r.all));
  return r;
}

// The gradient of the values not named, 2^((z - 2 half) c - more) f, and of a named one.
struct RowGrad {
  float c2, half, more, f;
  int none;       // nothing listed, or a weight of 0: no gradient, whatever the logits
  double w, mass;
  LogSum all;
  AJ_DEV void init(const Teacher &t, Listed e, double inv_temp, double weight, const LogSum &all_,
                   const LogSum &rest) {
    settle(e, rest);
    all = all_;
    mass = e.mass;
    w = (double)t.coef * inv_temp * weight;
    const LogSum &l = t.tail ? rest : all;
    // (a log-sum-exp over a tiny inv_temp may leave float32; `more` makes up for the bound)
    half = l.none() ? 0.f : (float)min(max(0.5 * l.unit / inv_temp, -0.5 * FLT_MAX), 0.5 * FLT_MAX);
    more = l.none() ? 0.f : (float)((l.unit - 2.0 * half * inv_temp + l.log) * kLog2eD);
    c2 = (float)(2.0 * inv_temp * kLog2eD);
    f = (float)(t.tail ? w * (e.mass * exp(log_ratio(rest, all)) - e.rest) : w * e.mass);
    none = e.mass == 0.0 || weight == 0.0;
  }
  AJ_DEV float other(float z) const {
    return none ? 0.f : fast_exp2(fmaf(fmaf(z, 0.5f, -half), c2, -more)) * f;
  }
  AJ_DEV float named(double p, double z, double inv_temp) const {
    return none ? 0.f : (float)(w * (mass * exp((z * inv_temp - all.unit) - all.log) - p));
  }
};

// Stores a run's gradients at out + u (whole: the run lies in the row and out is aligned as
// it is).
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <typename G, int R> AJ_DEV void store_run(G *out, const float (&g)[R]) {
  if constexpr (sizeof(G) == 4) {
#pragma unroll
    for (int j = 0; j < R; j += 4)
      __builtin_nontemporal_store(f32x4_t{g[j], g[j + 1], g[j + 2], g[j + 3]}, reinterpret_cast<f32x4_t *>(out + j));
  } else if constexpr (R == 4) {
    __builtin_nontemporal_store(u32x2_t{f2bf2(g[0], g[1]), f2bf2(g[2], g[3])}, reinterpret_cast<u32x2_t *>(out));
  } else {
    __builtin_nontemporal_store(
        u32x4_t{f2bf2(g[0], g[1]), f2bf2(g[2], g[3]), f2bf2(g[4], g[5]), f2bf2(g[6], g[7])},
        reinterpret_cast<u32x4_t *>(out));
  }
}
template <typename G, int R> AJ_DEV bool runs_aligned(const G *out) {
  return ((uintptr_t)out & (R * sizeof(G) - 1)) == 0 || ((uintptr_t)out & 15) == 0;
}

// One bit per value of u in [u0, u0 + kSplit): whether the list names it.
AJ_DEV void mark(uint32_t *bits, int v, int shift, int vocab, int u0, int u1) {
  if (v < 0 || v >= vocab) return;
  const int u = v + shift;
  if (u >= u0 && u < u1) atomicOr(&bits[(u - u0) >> 5], 1u << ((u - u0) & 31));
}

// One workgroup per part [u0, u1) of a row: the sum of 2^((z - m) c) over the values that the
// list does not name, with m.
template <typename T>
__global__ __launch_bounds__(kNT) void distill_part_kernel(const void *logits, int64_t ld, int vocab,
                                                           int parts, int width, Teacher t, float c2,
                                                           float2 *ms) {
  constexpr int R = kRun<T>, kStep = kNT * R * kQ;
  __shared__ uint32_t bits[kSplit / 32];
  __shared__ float red_m[kWaves], red_s[kWaves];
  const int64_t row = blockIdx.x / parts;
  const Row<T> x(logits, row, ld, vocab);
  const int u0 = blockIdx.x % parts * width, u1 = min(u0 + width, x.end);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  typename Row<T>::Bits b[kQ];
  auto fetch = [&](int u) __attribute__((always_inline)) { x.load(b, u, threadIdx.x * R, kNT * R, kStep); };
  fetch(u0);
  for (int i = threadIdx.x; i < width / 32; i += kNT) bits[i] = 0;
  __syncthreads();
  if ((int)threadIdx.x < t.k) mark(bits, t.idx[row * t.k + threadIdx.x], x.shift, vocab, u0, u1);
  __syncthreads();
  RunSum sum;
  for (int u = u0; u < u1; u += kStep) {
    float z[kQ * R];
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      float v[R];
      Row<T>::values(b[q], v);
      const int at = u - u0 + (q * kNT + threadIdx.x) * R;
      // few runs hold a named value, or lie in the next part: the rest skip this whole
      uint32_t w = at < width ? bits[at >> 5] >> (at & 31) & ((1u << R) - 1) : (1u << R) - 1;
#pragma unroll
      for (int j = 0; j < R; ++j) z[q * R + j] = v[j];
      if (__builtin_amdgcn_ballot_w64(w != 0)) {
#pragma unroll
        for (int j = 0; j < R; ++j) z[q * R + j] = w >> j & 1 ? -INFINITY : v[j];
      }
    }
    if (u + kStep < u1) fetch(u + kStep);
    sum.add(z, c2);
  }
  const float wm = wave_max(sum.m);
  if (lane == 0) red_m[wave] = wm;
  __syncthreads();
  float M = red_m[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, red_m[w]);
  const float s = wave_sum(in_unit(sum.m, sum.s, half_unit(M), c2));
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
  __shared__ int ids[kMaxK];
  __shared__ double red[kWaves];
  const int64_t row = blockIdx.x;
  const Listed e = listed<kWaves>(t, row, vocab, err, ids, red);
  const double z = e.v >= 0 ? (double)ldf((const T *)logits + row * ld + e.v) : -INFINITY;
  const NamedSums n = named_sums<kWaves>(e, z, inv_temp, red);
  if (threadIdx.x >= 64) return;
  const RowSums r = row_sums(e, n, ms + row * parts, parts, inv_temp);
  if (threadIdx.x == 0) {
    loss[row] = (float)r.loss;
    lse[row] = as_float(r.all);
    lse[rows + row] = as_float(r.rest);
  }
}

// stats[0] += sum of coef * weight * loss, stats[1] += rows, in one fixed order
__global__ __launch_bounds__(1024) void distill_stats_kernel(const float *loss, const float *weight,
                                                             int rows, float coef, float *stats) {
  __shared__ double red[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < rows; i += 1024) {
    const float w = weight ? weight[i] : 1.f;
    if (w != 0.f) s += (double)coef * w * loss[i];
  }
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
// A log-sum-exp l in float32 is off by 2^-24 |l|, and q by that much relatively.  From kFarLse
// on (2^-10) the row is summed again, by the workgroup of its first part alone, which then
// writes all of it (d logits may be the logits).
constexpr float kFarLse = 16384.f;
AJ_DEV bool far_lse(float l) { return fabsf(l) >= kFarLse && fabsf(l) <= FLT_MAX; }
AJ_DEV LogSum near_lse(float l) { return l == -INFINITY ? LogSum{0.0, -INFINITY} : LogSum{l, 0.0}; }

template <typename T, typename G>
AJ_DEV void far_row_grad(const Row<T> &x, int vocab, const Teacher &t, int64_t row, const Listed &e, double zn,
                         double inv_temp, G *out, uint32_t *bits, double *red, float2 *sums, RowGrad *shared) {
  constexpr int R = kRun<T>;
  const float c2 = (float)(2.0 * inv_temp * kLog2eD);
  RunSum sum;
  for (int u0 = 0; u0 < x.end; u0 += kSplit) {
    const int u1 = min(u0 + kSplit, x.end);
    __syncthreads();
    for (int i = threadIdx.x; i < kSplit / 32; i += kNT) bits[i] = 0;
    __syncthreads();
    mark(bits, e.v, x.shift, vocab, u0, u1);
    __syncthreads();
#pragma unroll 1
    for (int u = u0 + threadIdx.x * R; u < u1; u += kNT * R) {
      float z[R];
      Row<T>::values(x.load(u), z);
      const uint32_t w = bits[(u - u0) >> 5] >> ((u - u0) & 31);
#pragma unroll
      for (int j = 0; j < R; ++j) z[j] = w >> j & 1 ? -INFINITY : z[j];
      sum.add(z, c2);
    }
  }
  const float wm = wave_max(sum.m);
  const float s = wave_sum(in_unit(sum.m, sum.s, half_unit(wm), c2));
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = make_float2(wm, s);
  const NamedSums n = named_sums<kWaves>(e, zn, inv_temp, red);
  __syncthreads();
  if (threadIdx.x < 64) {
    const RowSums r = row_sums(e, n, sums, kWaves, inv_temp);
    if (threadIdx.x == 0) shared->init(t, e, inv_temp, t.weight ? t.weight[row] : 1.f, r.all, r.rest);
  }
  __syncthreads();
  const RowGrad grad = *shared;
#pragma unroll 1
  for (int u = threadIdx.x * R; u < x.end; u += kNT * R) {
    float z[R];
    Row<T>::values(x.load(u), z);
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (u + j >= x.shift && u + j < x.end) stf(out + u + j, grad.other(z[j]));
  }
  __syncthreads();
  if (e.v >= 0) stf(out + e.v + x.shift, grad.named(e.p, zn, inv_temp));
}
template <typename T, typename G>
__global__ __launch_bounds__(kNT) void distill_bwd_kernel(const void *logits, int64_t ld, int vocab,
                                                          int rows, int parts, int width, Teacher t,
                                                          double inv_temp, const float *lse, G *dz,
                                                          int64_t ldd) {
  constexpr int R = kRun<T>, kStep = kNT * R * kQ;
  __shared__ int ids[kMaxK];
  __shared__ double red[kWaves];
  const int64_t row = blockIdx.x / parts;
  const Row<T> x(logits, row, ld, vocab);
  const int u0 = blockIdx.x % parts * width, u1 = min(u0 + width, x.end);
  typename Row<T>::Bits b[kQ];
  auto fetch = [&](int u) __attribute__((always_inline)) { x.load(b, u, threadIdx.x * R, kNT * R, kStep); };
  fetch(u0);
  const Listed e = listed<kWaves>(t, row, vocab, nullptr, ids, red);
  const float all = lse[row], others = lse[rows + row];
  __shared__ RowGrad shared_grad;
  G *out = dz + row * ldd - x.shift;
  if (far_lse(all) || (t.tail && far_lse(others))) {
    __shared__ uint32_t bits[kSplit / 32];
    __shared__ float2 sums[kWaves];
    if (u0 == 0)
      far_row_grad<T, G>(x, vocab, t, row, e, e.v >= 0 ? (double)ldf((const T *)logits + row * ld + e.v) : -INFINITY,
                         inv_temp, out, bits, red, sums, &shared_grad);
    return;
  }
  if (threadIdx.x == 0)
    shared_grad.init(t, e, inv_temp, t.weight ? t.weight[row] : 1.f, near_lse(all), near_lse(others));
  __syncthreads();
  const RowGrad grad = shared_grad;
  // this part's named values, read before any is written (d logits may be the logits)
  const bool mine = e.v >= 0 && e.v + x.shift >= u0 && e.v + x.shift < u1;
  const float named = mine ? grad.named(e.p, ldf((const T *)logits + row * ld + e.v), inv_temp) : 0.f;
  __syncthreads();
  // runs are stored whole where d logits is aligned as the runs are
  const bool vec = runs_aligned<G, R>(out);
  for (int u = u0; u < u1; u += kStep) {
    float g[kQ][R];
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      Row<T>::values(b[q], g[q]);
#pragma unroll
      for (int j = 0; j < R; ++j) g[q][j] = grad.other(g[q][j]);
    }
    if (u + kStep < u1) fetch(u + kStep);
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      const int at = u + (q * kNT + threadIdx.x) * R;
      if (at >= u1) continue;
      if (vec && at >= x.shift && at + R <= x.end) {
        store_run<G, R>(out + at, g[q]);
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

// Loss and gradient of a row in one go: one workgroup of 16 waves per row keeps what it
// reads for the loss on the chip, in registers (REG runs a thread) and LDS (LDS runs), and
// forms the gradient from there; of a row of 152064 values that is 81920 in float32 (54 %) and
// 131072 in bfloat16 (86 %), the rest is read again, newest first, while the caches still have it.
// Rows of up to kSmallVocab values take four waves each, which hold all of a row in registers.
struct LongRows {
  static constexpr int NT = 1024, REG = 12, REG16 = 8, LDS = 8, WORDS = 6144;    // 128 KB of runs, 24 KB of bits
};
// of more than kLongVocab values, whose bits take a run's place in LDS
struct VeryLongRows {
  static constexpr int NT = 1024, REG = 12, REG16 = 8, LDS = 7, WORDS = 8448;
};
struct ShortRows {
  static constexpr int NT = 256, REG = 12, REG16 = 8, LDS = 0, WORDS = 512;
};
constexpr int kLongVocab = LongRows::WORDS * 32 - 16, kStepVocab = VeryLongRows::WORDS * 32 - 16;
constexpr int kSmallVocab = ShortRows::NT * ShortRows::REG * 4 - 8;
static_assert(kSmallVocab <= ShortRows::WORDS * 32 - 16 && kSmallVocab <= ShortRows::NT * ShortRows::REG16 * 8 - 8,
              "short rows fit");
template <typename T, typename G, typename S>
__global__ __launch_bounds__(S::NT) void distill_step_kernel(const void *logits, int64_t ld, int vocab, int rows,
                                                             Teacher t, double inv_temp, float *loss, float *lse,
                                                             int32_t *err, G *dz, int64_t ldd) {
  constexpr int kStepNT = S::NT, kStepWaves = kStepNT / 64, kHoldLds = S::LDS;
  constexpr int R = kRun<T>, C = kStepNT * R, NR = sizeof(T) == 4 ? S::REG : S::REG16;
  __shared__ __attribute__((aligned(16))) uint4 held[kHoldLds ? kHoldLds : 1][kStepNT];
  __shared__ uint32_t bits[S::WORDS];
  __shared__ int ids[kMaxK];
  __shared__ double red[kStepWaves];
  __shared__ float2 sums[kStepWaves];
  __shared__ RowGrad shared_grad;
  // what a thread knows of the list waits here: its registers hold the row
  __shared__ double list_p[kMaxK];
  __shared__ Listed shared_list;
  __shared__ NamedSums shared_named;
  const int64_t row = blockIdx.x;
  const Row<T> x(logits, row, ld, vocab);
  const int me = threadIdx.x * R;
  const int stripes = (x.end + C - 1) / C;
  typedef typename Row<T>::Bits Bits;
  auto fetch = [&](int k) __attribute__((always_inline)) { return x.whole(k * C + me); };
  Bits b[NR];
  // (of a long row the last two wait until the list's sums in 64 bits have left registers)
  constexpr int kEarly = kHoldLds ? NR - 2 : NR;
#pragma unroll
  for (int k = 0; k < kEarly; ++k) b[k] = fetch(k);
  for (int i = threadIdx.x; i <= x.end / 32; i += kStepNT) bits[i] = 0;
  int my_v;
  float my_z;
  {
    const Listed e = listed<kStepWaves>(t, row, vocab, err, ids, red);
    my_v = e.v;
    my_z = e.v >= 0 ? ldf((const T *)logits + row * ld + e.v) : -INFINITY;
    mark(bits, e.v, x.shift, vocab, 0, x.end);
    const NamedSums n = named_sums<kStepWaves>(e, my_z, inv_temp, red);
    if ((int)threadIdx.x < t.k) list_p[threadIdx.x] = e.p;
    if (threadIdx.x == 0) {
      shared_list = e;
      shared_named = n;
    }
  }
  const int rim = threadIdx.x < 2 * R ? x.rim(threadIdx.x) : -1;
  const float zr = rim >= 0 ? ldf(x.aligned + rim) : -INFINITY;
  RunSum sum;
  // copies of `me` that the compiler does not see into, or it keeps every run's place from the
  // loads for the sums and the stores, for which there are no registers
  int mine = me;
  asm volatile("" : "+v"(mine));
  // adds the values of N runs, at stripes k0, k0 + 1 and so on, that are not named
  auto absorb = [&](auto N, const Bits *v, int k0) __attribute__((always_inline)) {
    constexpr int n = decltype(N)::value;
    float z[n * R];
#pragma unroll
    for (int q = 0; q < n; ++q) {
      float f[R];
      Row<T>::values(v[q], f);
      const int u = min((k0 + q) * C + mine, x.end);
      const uint32_t w = bits[u >> 5] >> (u & 31) & ((1u << R) - 1);
#pragma unroll
      for (int j = 0; j < R; ++j) z[q * R + j] = f[j];
      if (__builtin_amdgcn_ballot_w64(w != 0)) {
#pragma unroll
        for (int j = 0; j < R; ++j) z[q * R + j] = w >> j & 1 ? -INFINITY : f[j];
      }
    }
    sum.add(z, (float)(2.0 * inv_temp * kLog2eD));
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  auto absorb_two = [&](const Bits *v, int k) __attribute__((always_inline)) {
    if constexpr (R == 4) {
      absorb(Two{}, v, k);
    } else {      // (16 values at a time want more registers than there are)
      absorb(One{}, v, k);
      absorb(One{}, v + 1, k + 1);
    }
  };
#pragma unroll
  for (int k = kEarly; k < NR; ++k) b[k] = fetch(k);
  // LDS's share by way of registers, two stripes ahead
#pragma unroll
  for (int k = 0; k < kHoldLds; ++k) {
    const Bits v = fetch(NR + k);
    held[k][threadIdx.x] = v.w;
  }
#pragma unroll
  for (int k = 0; k < NR; k += 2) absorb_two(b + k, k);
  Bits v[2] = {fetch(NR + kHoldLds), fetch(NR + kHoldLds + 1)};
#pragma unroll 1
  for (int k = 0; k < kHoldLds; ++k) {
    Bits h;
    h.w = held[k][threadIdx.x];     // (its own writes)
    absorb(One{}, &h, NR + k);
  }
  for (int k = NR + kHoldLds; k < stripes; k += 2) {
    const Bits now[2] = {v[0], v[1]};
    v[0] = fetch(k + 2);
    v[1] = fetch(k + 3);
    absorb_two(now, k);
  }
  const bool rim_named = rim >= 0 && (bits[rim >> 5] >> (rim & 31) & 1);
  if (rim >= 0 && !rim_named) {
    const float z[1] = {zr};
    sum.add(z, (float)(2.0 * inv_temp * kLog2eD));
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float wm = wave_max(sum.m);
  const float s = wave_sum(in_unit(sum.m, sum.s, half_unit(wm), (float)(2.0 * inv_temp * kLog2eD)));
  if (lane == 0) sums[wave] = make_float2(wm, s);
  lds_barrier();
  if (wave == 0) {
    const Listed e = shared_list;     // (of the first thread, whose mass and rest are the row's)
    const RowSums r = row_sums(e, shared_named, sums, kStepWaves, inv_temp);
    if (lane == 0) {
      shared_grad.init(t, e, inv_temp, t.weight ? t.weight[row] : 1.f, r.all, r.rest);
      loss[row] = (float)r.loss;
      lse[row] = as_float(r.all);
      lse[rows + row] = as_float(r.rest);
    }
  }
  lds_barrier();
  const RowGrad grad = shared_grad;
  G *out = dz + row * ldd - x.shift;
  const bool vec = runs_aligned<G, R>(out);
  asm volatile("" : "+v"(mine));
  auto put = [&](const Bits &v, int k) __attribute__((always_inline)) {
    const int u = k * C + mine;
    if (u < x.shift || u + R > x.end) return;
    float g[R];
    Row<T>::values(v, g);
#pragma unroll
    for (int j = 0; j < R; ++j) g[j] = grad.other(g[j]);
    if (vec) {
      store_run<G, R>(out + u, g);
    } else {
#pragma unroll
      for (int j = 0; j < R; ++j) stf(out + u + j, g[j]);
    }
  };
  int k = stripes - 1;
  if (k >= NR + kHoldLds) {
    Bits a = fetch(k), c2 = fetch(k - 1);
    for (; k >= NR + kHoldLds; --k) {
      const Bits now = a;
      a = c2;
      if (k - 2 >= NR + kHoldLds) c2 = fetch(k - 2);
      put(now, k);
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) put(b[k], k);
#pragma unroll 1
  for (int k = 0; k < kHoldLds; ++k) {
    Bits h;
    h.w = held[k][threadIdx.x];
    put(h, NR + k);
  }
  if (rim >= 0) stf(out + rim, grad.other(zr));
  __syncthreads();    // the named ones over what the runs left there
  if (my_v >= 0) stf(out + my_v + x.shift, shared_grad.named(list_p[threadIdx.x], my_z, inv_temp));
}

// ------------------------------------------------------------------ host
struct TopWs {
  uint64_t *cand;
  float2 *ms;
  int parts, width;
  size_t bytes;
};

// Parts of a row: one where there are kTopRows rows and more, else about 4096 in all (three
// rounds of what the card holds), but never more a row than the join holds: candidates of
// all a row's parts, kMaxCand.
constexpr int kTopRows = 1024;
TopWs carve_top(int rows, int vocab, int k, void *base) {
  aj::Carver cv(base);
  TopWs w;
  const int64_t span = (int64_t)vocab + 7;   // a row may start 7 values past a run boundary
  const int64_t n = (span + kTopChunk - 1) / kTopChunk;
  const int64_t parts = rows >= kTopRows ? 1 : std::min({n, (int64_t)4096 / std::max(rows, 1), (int64_t)kMaxCand / k});
  w.width = (int)((n + parts - 1) / parts) * kTopChunk;
  w.parts = (int)((span + w.width - 1) / w.width);
  // at least what fewer rows, cut finer, ask for
  const size_t room = (size_t)std::max((int64_t)rows * w.parts, std::min<int64_t>(rows * n, 4096));
  w.cand = cv.take<uint64_t>(room * k);
  w.ms = cv.take<float2>(room);
  w.bytes = cv.bytes();
  return w;
}

struct Split { int parts, width; };
int whole_parts(int vocab) { return (vocab + 7 + kSplit - 1) / kSplit; }    // the fewest a row is cut into
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
  // workgroups of 256 threads, of which a launch takes fewer than 2^32
  AJ_REQUIRE((int64_t)lg->rows * whole_parts(lg->vocab) < 1 << 24, AJ_ERR_SHAPE,
             "%s: rows %d of %d parts each (below 2^24 in all)", name, lg->rows, whole_parts(lg->vocab));
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
  const unsigned grid = (unsigned)lg.rows * w.parts;
  topk_part_kernel<T><<<grid, kTopNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, w.parts, w.width, k, lg.inv_temp, w.cand,
                                               w.ms, idx, logprob, lse);
  if (w.parts > 1)
    topk_merge_kernel<T><<<lg.rows, kMergeNT, 0, st>>>(lg.logits, lg.ld, lg.vocab, w.parts, k, lg.inv_temp,
                                                     w.cand, w.ms, idx, logprob, lse);
}

template <typename T>
void launch_loss(const aj_logits &lg, const aj_teacher &t, float *loss, float *lse, float *stats,
                 int32_t *err, float2 *ms, hipStream_t st) {
  const Split s = row_split(lg.rows, lg.vocab);
  distill_part_kernel<T><<<(unsigned)lg.rows * s.parts, kNT, 0, st>>>(
      lg.logits, lg.ld, lg.vocab, s.parts, s.width, teacher_of(t), 2.f * lg.inv_temp * kLog2e, ms);
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

// Long rows take a workgroup each from two rounds of the CUs on, and from so many values that
// what they keep is worth the list's sums at the start of every row; others go by the loss's and
// the gradient's kernels, cut into parts.  Those two / the one, us, k 64, bfloat16 d logits:
//   rows of 152064   256 rows   384       512       1024      4096
//     float32         68 / 52    94 / 89  139 / 107 317 / 226 1177 / 866
//     bfloat16        49 / 42    66 / 72   85 / 78  182 / 159  738 / 628
//   4096 rows of    32768       40000     50257     65536     80000     100000
//     float32       286 / 327  344 / 358 465 / 400 594 / 443 680 / 503 824 / 583
//     bfloat16      166 / 338  215 / 350 299 / 375 397 / 400 446 / 433 543 / 481
// (At 256 rows, one full round, the one kernel is the faster too; at 128, 42 / 40, they are
// alike, and at 64, 28 / 37, it is the slower.)
constexpr int kStepRows = 512, kStepLeastF32 = 45056, kStepLeastBf16 = 73728;
bool one_step(const aj_logits &lg) {
  const int least = lg.dtype == AJ_BF16 ? kStepLeastBf16 : kStepLeastF32;
  return lg.vocab <= kSmallVocab || (lg.rows >= kStepRows && lg.rows < 1 << 22 && lg.vocab >= least &&
                                     lg.vocab <= kStepVocab);     // (2^22 workgroups of 1024 threads: too many)
}
template <typename T, typename G>
void launch_step(const aj_logits &lg, const aj_teacher &t, float *loss, float *lse, int32_t *err, void *dz,
                 int64_t ldd, hipStream_t st) {
  if (lg.vocab <= kSmallVocab)
    distill_step_kernel<T, G, ShortRows><<<lg.rows, ShortRows::NT, 0, st>>>(
        lg.logits, lg.ld, lg.vocab, lg.rows, teacher_of(t), lg.inv_temp, loss, lse, err, (G *)dz, ldd);
  else if (lg.vocab > kLongVocab)
    distill_step_kernel<T, G, VeryLongRows><<<lg.rows, VeryLongRows::NT, 0, st>>>(
        lg.logits, lg.ld, lg.vocab, lg.rows, teacher_of(t), lg.inv_temp, loss, lse, err, (G *)dz, ldd);
  else
    distill_step_kernel<T, G, LongRows><<<lg.rows, LongRows::NT, 0, st>>>(
        lg.logits, lg.ld, lg.vocab, lg.rows, teacher_of(t), lg.inv_temp, loss, lse, err, (G *)dz, ldd);
}

size_t distill_ws(int rows, int vocab) {
  auto parts = [&](int width) { return (vocab + 7 + width - 1) / width; };
  aj::Carver cv(nullptr);
  // at least what fewer rows, cut finer (halved from under 2048 parts), ask for
  cv.take<float2>(std::max((int64_t)rows * parts(kSplit), std::min<int64_t>((int64_t)rows * parts(2048), 3 * 2048)));
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
  if (rows < 0 || vocab <= 0 || k <= 0 || k > kMaxK) return 0;
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
  if (rows < 0 || vocab <= 0 || k <= 0 || k > kMaxK) return 0;
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
  if (lg->rows > 0 && one_step(*lg)) {
    AJ_REQUIRE(loss && lse && ws, AJ_ERR_NULL, "%s: null pointer", name);
    const size_t need = distill_ws(lg->rows, lg->vocab);
    AJ_REQUIRE(ws_bytes >= need, AJ_ERR_WORKSPACE, "%s: workspace %zu < %zu", name, ws_bytes, need);
    hipStream_t st = (hipStream_t)stream;
    if (lg->dtype == AJ_BF16) {
      if (d_dtype == AJ_BF16) launch_step<bf16_t, bf16_t>(*lg, *t, loss, lse, err, dlogits, ldd, st);
      else launch_step<bf16_t, float>(*lg, *t, loss, lse, err, dlogits, ldd, st);
    } else {
      if (d_dtype == AJ_BF16) launch_step<float, bf16_t>(*lg, *t, loss, lse, err, dlogits, ldd, st);
      else launch_step<float, float>(*lg, *t, loss, lse, err, dlogits, ldd, st);
    }
    if (stats) distill_stats_kernel<<<1, 1024, 0, st>>>(loss, t->weight, lg->rows, t->coef, stats);
    return aj::check_launch(name);
  }
  if ((r = aj_distill_loss_fwd(lg, t, loss, lse, stats, err, ws, ws_bytes, stream))) return r;
  return aj_distill_loss_bwd(lg, t, lse, dlogits, ldd, d_dtype, stream);
}
