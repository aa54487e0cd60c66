// sample.hip -- gfx950 kernels of bridger_sample: a class of every row, drawn from its scores.
#include "scores.h"

namespace bridger {

// A value that all lanes agree on, in scalar registers.
__device__ inline uint32_t uniform(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ inline double uniform(double v) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  return __builtin_bit_cast(double, make_uint2(uniform(w.x), uniform(w.y)));
}
__device__ inline float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }

// A row's weights, e^((v - top) / T): 2^n times a polynomial in f, n + f = (v - top) log2(e) / T, |f| <=
// 1/2, that meets 2^f at eleven Chebyshev points and is off by at most 3.2e-16 of it; 1 for the largest,
// 0 below 2^-1075.  A draw compares sums of these with a random number, so they are held in double.
struct Weights {
  double top, factor;  // log2(e) / T
  double last;         // v - top of weight 0
  __device__ Weights(float top, double factor)
      : top(uniform((double)top)), factor(uniform(factor)), last(uniform(-1100.0 / factor)) {}
  // (a score of +infinity is its row's largest)
  __device__ double operator()(float v) const {
    return (double)v == top ? 1.0 : of((double)v - top);
  }
  __device__ double of(double d) const {
    double w[1];
    of<1>({d}, w);
    return w[0];
  }
  // N at a time, step by step, so that none waits for its own results.  Double instructions bound the
  // rows that need them for every class: 1 x 128,000 without cuts 69 us, a maximum alone 15.
  template <int N>
  __device__ void of(const double (&d)[N], double (&w)[N]) const {
    constexpr double round = 0x1.8p52;  // leaves whole numbers, in the lower word
    constexpr double c[] = {1.0208690299958306e-07, 1.321544258792169e-06, 1.5252657260200837e-05,
                            0.0001540353044173605,  0.0013333558230164974, 0.009618129107606888,
                            0.05550410866444772,    0.24022650695910097,   0.69314718055995, 1.0};
    double t[N], f[N], s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double x = fmax(d[i], last);  // (NaN: last)
      t[i] = __builtin_fma(x, factor, round);
      f[i] = __builtin_fma(x, factor, round - t[i]);
      s[i] = 7.072585949269223e-09;
    }
#pragma unroll
    for (int k = 0; k < 10; ++k) {
      double ck = c[k];
      asm("" : "+s"(ck));  // (in vector registers it would take a copy, too)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = __builtin_fma(s[i], f[i], ck);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      w[i] = __builtin_ldexp(s[i], (int)(uint32_t)__builtin_bit_cast(uint64_t, t[i]));
  }
  // The weights of four scores, those that are `in` (0 for others); their sum.
  __device__ void four(const float (&v)[4], const bool (&in)[4], double (&w)[4]) const {
    double d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      d[i] = in[i] ? (double)v[i] - top : last;
      d[i] = (double)v[i] == top && in[i] ? 0.0 : d[i];
    }
    of<4>(d, w);
  }
  __device__ double sum(const float (&v)[4], const bool (&in)[4]) const {
    double w[4];
    four(v, in, w);
    return (w[0] + w[1]) + (w[2] + w[3]);
  }
};

// The same relative to another score, quickly: the exponent in two floats, the exponential in one.  Off
// by 2^-23 times 0.36 of the exponent (the difference rounds by 2^-24 of it, times ln 2), 1 for the
// exponential and 1 for the product that follows.
struct QuickWeights {
  float high, low;  // log2(e) / T
  __device__ explicit QuickWeights(double factor)
      : high(uniform((float)factor)), low(uniform((float)(factor - (double)(float)factor))) {}
  // d = v - score (NaN: no weight); the exponent in `e`
  __device__ float operator()(float d, float *e) const {
    const float a = fmaxf(d * high, -200.0f);
    const float b = __builtin_fmaf(d, low, __builtin_fmaf(d, high, -a));
    const float w = __builtin_amdgcn_exp2f(a);
    *e = a;
    return a > -200.0f ? __builtin_fmaf(w, b * 0.693147181f, w) : 0.0f;
  }
};

template <int G>
constexpr int kSorted = G >= 1024 ? 2048 : G > 64 ? 1024 : 512;  // candidates that LDS holds

constexpr int kSegments = 16;  // of a row, whose sums the draw keeps
template <int G>
constexpr int kBins = G >= 512 ? 4 : 8;  // of a range that a cut is looked for in

template <int G>
struct SampleShared {
  union {
    uint64_t key[kSorted<G> + 8];
    unsigned long long bins[kSorted<G>];  // weights, by bins that all lanes share
    struct {  // a lane's weights and numbers of scores
      double weight[kBins<G>][G];
      int count[kBins<G>][G];
    } bin;
  };
  double segment[kSegments][G / 64];
  double part[kSegments];
  double wave[2][G / 64];
  double sum[G / 64];
  float bound[G / 64];
  int found[G / 64];
  int count, chosen, last;
  int32_t cls;   // what was drawn,
  double share;  // and its share of what stays
};

// What stays of a row: classes up to `cls` of score `score` and all of larger ones, at least `floor`.
struct Kept {
  float score, floor;
  int32_t cls;
  __device__ bool operator()(float v, int j) const {
    return (v > score || (v == score && j <= cls)) && v >= floor;
  }
};

// Sums over the workgroup, the same bits in all lanes.  `at` holds a value a wave.
template <int G, typename V>
__device__ inline V sum_all(V v, V *at) {
  v = lanes_reduce<Sum, 64>(v);
  if constexpr (G > 64) {
    __syncthreads();  // the last sum is read
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lanes_reduce<Sum, G / 64>(at[threadIdx.x & (G / 64 - 1)]);
  }
  return v;
}

// The sum of v over the lanes of the workgroup below this one; over all of them in `all`.
template <int G>
__device__ inline double lanes_before(double v, double *at, double *all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double sum = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double other = __shfl_up(sum, d, 64);
    if (lane >= d) sum += other;
  }
  double before = __shfl_up(sum, 1, 64);
  if (lane == 0) before = 0.0;
  if constexpr (G > 64) {
    __syncthreads();  // what `at` held is read
    if (lane == 63) at[wave] = sum;
    __syncthreads();
    double start = 0.0;
    *all = 0.0;
#pragma unroll 4
    for (int w = 0; w < G / 64; ++w) {
      if (w == wave) start = *all;
      *all += at[w];
    }
    return start + before;
  } else {
    *all = __shfl(sum, 63, 64);
    return before;
  }
}

// f(score, its place) for the scores of one load, two at a time: written out in full, the walks
// over a row's registers would not fit the instruction cache.
template <typename T, typename F>
__device__ inline void each_score(u32x4 raw, F f) {
#pragma unroll 1
  for (int i = 0; i < kPerLoad<T>; i += 2) {
    f(element<T>(raw, 0), i);
    f(element<T>(raw, 1), i + 1);
    if constexpr (sizeof(T) == 4) {
      raw = u32x4{raw[2], raw[3], 0, 0};
    } else {
      raw = u32x4{raw[1], raw[2], raw[3], 0};
    }
  }
}

// The same, four at a time: f(scores, the first one's place).
template <typename T, typename F>
__device__ inline void each_four(u32x4 raw, F f) {
#pragma unroll 1
  for (int i = 0; i < kPerLoad<T>; i += 4) {
    f({element<T>(raw, 0), element<T>(raw, 1), element<T>(raw, 2), element<T>(raw, 3)}, i);
    raw = u32x4{raw[2], raw[3], 0, 0};
  }
}

// A row's scores.  each(f): f(first class, 16 bytes of scores), in ascending order per lane, NaN past the
// row's end; all lanes make the same number of calls.  Every walk reads the row again, from the caches,
// with the next loads on their way while one is looked at: held in registers a long row leaves too few
// of them for the rest (2048 x 128,000 bfloat16, top_k 50: 221 to 241 us, 285 from registers).  kRing loads
// take turns, written out; each_again() is for walks that few rows take.
template <typename T, int G, int kRing>
struct Scores {
  const T *row;
  int n;
  static constexpr int V = kPerLoad<T>;
  __device__ int at(int64_t j0) const {
    const int64_t j = j0 + (int64_t)threadIdx.x * V;
    return (int)(j < n ? j : n);
  }
  template <typename F>
  __device__ void look(RowLoad<T> l, int64_t j0, F &f) const {
    const int j = at(j0);
    if (j0 + G * V > n) l.take(j, n, fill_of((T)__builtin_nanf("")));
    f(j, l.raw);
  }
  template <typename F>
  __device__ bool tiny(F &f) const {
    if (n >= V) return false;
    RowLoad<T> l;
    l.tiny(row, (int)threadIdx.x * V, n, (T)__builtin_nanf(""));
    f(at(0), l.raw);
    return true;
  }
  template <typename F>
  __device__ void each(F f) const {
    if (tiny(f)) return;
    constexpr int64_t step = G * V;
    RowLoad<T> ring[kRing];
#pragma unroll
    for (int u = 0; u < kRing; ++u)
      if (u * step < n) ring[u].issue(row, at(u * step), n);
#pragma unroll 1
    for (int64_t j0 = 0; j0 < n; j0 += kRing * step) {
#pragma unroll
      for (int u = 0; u < kRing; ++u)
        if (j0 + u * step < n) {
          look(ring[u], j0 + u * step, f);
          if (j0 + (u + kRing) * step < n) ring[u].issue(row, at(j0 + (u + kRing) * step), n);
        }
    }
  }
  template <typename F>
  __device__ void each_again(F f) const {
    if (tiny(f)) return;
    constexpr int64_t step = G * V;
    RowLoad<T> next;
    next.issue(row, at(0), n);
#pragma unroll 1
    for (int64_t j0 = 0; j0 < n; j0 += step) {
      const RowLoad<T> l = next;
      if (j0 + step < n) next.issue(row, at(j0 + step), n);
      look(l, j0, f);
    }
  }
};

// ---------------------------------------------------------------------------- candidates
// Scores of [lo, up) in the order that `kept` keeps go to the candidates; their number (it may pass
// kSorted, whose entries alone are there).
template <typename T, int G, int A, typename Keep>
__device__ inline int collect(const Scores<T, G, A> &x, SampleShared<G> &s, Keep kept, uint32_t lo, uint32_t up) {
  constexpr int V = kPerLoad<T>;
  const float low = value_of(lo);
  __syncthreads();
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
    float top = element<T>(raw, 0);
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, element<T>(raw, i));
    if (top >= low) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float v = element<T>(raw, i);
        if (v >= low && order_of(v) < up && kept(v, j + i)) {
          const int at = atomicAdd(&s.count, 1);
          if (at < kSorted<G>) s.key[at] = key_of(v, j + i);
        }
      }
    }
  });
  __syncthreads();
  return s.count;
}

template <int G>
constexpr int kRanked = G < 256 ? 256 : G < 512 ? G : 512;  // candidates that are ranked by counting

// Sorts the first `count` candidates, the largest first (some zeros behind).  Few: each goes where as
// many larger ones say.  More: compare and exchange over a network of the next power of two.
template <int G>
__device__ inline void sort_candidates(SampleShared<G> &s, int count) {
  constexpr int E = G < 256 ? 256 / G : 1;
  __syncthreads();
  if (count <= kRanked<G>) {
    if (threadIdx.x < 8) s.key[count + threadIdx.x] = 0;
    __syncthreads();
    uint64_t mine[E];
    int larger[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int t = e * G + threadIdx.x;
      if (e * G < count) {
        mine[e] = s.key[t < count ? t : count];
        larger[e] = 0;
      }
    }
    if ((threadIdx.x & ~63) < count)
#pragma unroll 1
      for (int q = 0; q < count; q += 8) {  // four loads on their way at once
        ulonglong2 other[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = *(const ulonglong2 *)&s.key[q + 2 * i];
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e * G < count)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              larger[e] += (other[i].x > mine[e]) + (other[i].y > mine[e]);
      }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * G + (int)threadIdx.x < count) s.key[larger[e]] = mine[e];
    __syncthreads();
    return;
  }
  int size = 64;
  while (size < count) size *= 2;
  for (int t = count + threadIdx.x; t < size; t += G) s.key[t] = 0;
#pragma unroll 1
  for (int run = 2; run <= size; run *= 2)
#pragma unroll 1
    for (int step = run / 2; step > 0; step /= 2) {
      __syncthreads();
#pragma unroll 1
      for (int t = threadIdx.x; t < size / 2; t += G) {
        const int i = (t & ~(step - 1)) * 2 + (t & (step - 1)), k = i + step;
        const uint64_t a = s.key[i], b = s.key[k];
        if ((a < b) == ((i & run) == 0)) s.key[i] = b, s.key[k] = a;
      }
    }
  __syncthreads();
}

// Weights of a lane's candidates, neighbours in the list, and what stands before them.
template <int G>
struct Listed {
  static constexpr int E = kSorted<G> / G;
  double w[E], before, all;
  __device__ Listed(SampleShared<G> &s, int count, const Weights &weight, int shift) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int t = threadIdx.x * E + i;
      w[i] = t < count ? weight(value_of((uint32_t)(s.key[t] >> shift))) : 0.0;
      sum += w[i];
    }
    before = lanes_before<G>(sum, s.sum, &all);
  }
  // how many of the first `count` have less than `target` before them
  __device__ int leading(SampleShared<G> &s, int count, double target) const {
    int stay = 0;
    double at = before;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      stay += (int)threadIdx.x * E + i < count && at < target;
      at += w[i];
    }
    return sum_all<G>(stay, s.found);
  }
};

// ------------------------------------------------------------------- cuts of whole rows
// The general way to a row's target-th score in the order (by weight: to the last one before which
// less than the target stands), among those of order [lo, up): parts the range into bins and goes on with
// the one that holds it, until LDS holds its scores or one score is left, that of many classes.  What is
// left of the target below `up` lies in [least, most]: by quick weights it is an interval, and false is
// returned where that does not tell, with the range so far.
struct Range {
  uint32_t lo, up;
  double least, most;
  int within;  // classes in the range (INT32_MAX: not known)
};

// One walk for a cut by quick weights: parts the scores of the range into bins of equal width, of which
// those that may hold the cut are left.  The weights are added up as whole numbers, whose sums do not
// depend on the order.  (512 x 50,257 float, top_p 0.95: 354 us with cut()'s bins alone, which take
// several walks, 244 with this one first.)
enum class Found { kRange, kUnclear, kPast };  // kPast: the whole range is less than the target
template <typename T, int G, int A>
__device__ inline Found narrow(const Scores<T, G, A> &x, SampleShared<G> &s, const Weights &weight,
                              Range &r) {
  constexpr int bins = kSorted<G>, lane_bins = bins / 64;
  const float top = (float)weight.top, first = value_of(r.lo), last = value_of(r.up - 1);
  const float scale = (float)bins / (last - first);
  if (!(scale > 0x1p-100f && scale < 0x1p100f)) return Found::kRange;  // (one score, or no finite range)
  const QuickWeights quick(weight.factor);
  auto bin = [&](float v) {  // no lower for a larger score
    const int b = (int)((v - first) * scale);
    return b < bins ? b : bins - 1;
  };
  // weights are multiples of 1 / unit, and n of them stay below 2^63
  const int digits = 31 + __builtin_clz((uint32_t)x.n);
  const double unit = __builtin_ldexp(1.0, digits < 50 ? digits : 50);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += G) s.bins[b] = 0;
  __syncthreads();
  x.each([&](int, const u32x4 &raw) __attribute__((always_inline)) {
    each_score<T>(raw, [&](float e, int) {
      if (e >= first && e <= last) {
        float exponent;
        const double w = __builtin_fma((double)quick(e - top, &exponent), unit, 0x1p52);
        atomicAdd(&s.bins[bin(e)], __builtin_bit_cast(uint64_t, w) & (~uint64_t(0) >> 12));
      }
    });
  });
  __syncthreads();
  // each wave finds the bins: a lane has lane_bins neighbours, the first lane the largest scores
  const int lane = threadIdx.x & 63, mine = bins - 1 - lane * lane_bins;
  unsigned long long sum = 0;
  for (int i = 0; i < lane_bins; ++i) sum += s.bins[mine - i];
  unsigned long long upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const unsigned long long other = __shfl_up(upto, d, 64);
    if (lane >= d) upto += other;
  }
  upto -= sum;
  const double rounding = (double)x.n / unit;
  auto off_from = [&](uint32_t lowest) {  // of the sum of weights of scores from there on
    return 0x1p-23 * (0.4 * (weight.top - (double)value_of(lowest)) * weight.factor + 2.5);
  };
  double off = off_from(r.lo), past = 0.0;
  int above = 0, reached = 0;  // bins wholly before the cut; that may be
  for (int i = 0; i < lane_bins; ++i) {
    upto += s.bins[mine - i];
    const double sums = (double)upto / unit;
    if (sums * (1.0 + off) + rounding < r.least) past += (double)s.bins[mine - i] / unit, ++above;
    reached += sums * (1.0 - off) - rounding < r.most;
  }
  above = lanes_reduce<Sum, 64>(above);
  reached = lanes_reduce<Sum, 64>(reached);
  past = uniform(lanes_reduce<Sum, 64>(past));
  __syncthreads();  // the bins are read
  if (reached >= bins) return above >= bins ? Found::kPast : Found::kUnclear;
  auto edge = [&](int b) {  // the lowest order of bin b and those after it
    uint32_t lo = r.lo, up = r.up;
    while (up - lo > 1) {
      const uint32_t mid = lo + (up - lo) / 2;
      if (bin(value_of(mid)) >= b) {
        up = mid;
      } else {
        lo = mid;
      }
    }
    return uniform(up);
  };
  const uint32_t up = above > 0 ? edge(bins - above) : r.up;
  const uint32_t lo = reached < bins - 1 ? edge(bins - 1 - reached) : r.lo;
  off = above > 0 ? off_from(up) : 0.0;
  r.most -= past > 0.0 ? past * (1.0 - off) - rounding : 0.0;
  r.least -= past > 0.0 ? past * (1.0 + off) + rounding : 0.0;
  r.lo = lo;
  r.up = up;
  r.within = 0;  // to be seen
  return Found::kRange;
}
// *at += v in LDS, without waiting for what was there; no other lane adds to it.
template <typename V>
__device__ inline void lane_add(V *at, V v) {
  __hip_atomic_fetch_add(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
enum class Measure { kCount, kWeight, kQuickWeight };
template <typename T, int G, int A>
__device__ inline bool cut(const Scores<T, G, A> &x, SampleShared<G> &s, Kept &kept,
                           const Weights &weight, Range &r, Measure by) {
  const float top = (float)weight.top;
  const QuickWeights quick(weight.factor);
  const bool whole = kept.score == -__builtin_inff() && kept.floor == -__builtin_inff();
  for (;;) {
    const bool one = r.up - r.lo == 1;
    if (one || r.within <= kSorted<G>) {
      const int count = collect<T, G, A>(x, s, kept, r.lo, r.up);
      if (count == 0) {  // rounding leaves the target past the range's last: it stays, and nothing below
        const float last = value_of(r.lo);
        if (last > kept.score) kept.score = last, kept.cls = INT32_MAX;
        return true;
      }
      if (count <= kSorted<G>) {
        sort_candidates<G>(s, count);
        int stay = r.most < count ? (int)r.most : count;
        if (by != Measure::kCount) {
          const Listed<G> l(s, count, weight, 32);
          stay = l.leading(s, count, r.most);
          if (by == Measure::kQuickWeight && stay != l.leading(s, count, r.least)) return false;
        }
        const uint64_t key = s.key[stay > 0 ? stay - 1 : 0];
        kept.score = value_of((uint32_t)(key >> 32));
        kept.cls = class_of(key);
        return true;
      }
    }
    if (one) {
      const float v = value_of(r.lo);
      const double each = by == Measure::kCount ? 1.0 : weight(v);
      double want = __builtin_ceil(r.most / each);
      if (want != __builtin_ceil(r.least / each)) return false;
      if (!(want >= 1.0)) want = 1.0;  // of its classes
      int32_t cls = 0;
      for (int bit = 30; bit >= 0; --bit) {  // the largest class with fewer than those before it
        const int32_t next = cls | 1 << bit;
        int below = 0;
        x.each_again([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
          each_score<T>(raw, [&](float e, int i) {
            below += e == v && j + i < next && kept(e, j + i);
          });
        });
        if ((double)sum_all<G>(below, s.found) < want) cls = next;
      }
      kept.score = v;
      kept.cls = cls;
      return true;
    }
    int shift = 0;
    while ((r.up - 1 - r.lo) >> shift >= kBins<G>) ++shift;
    const int bins = (int)((r.up - 1 - r.lo) >> shift) + 1;
    const float first = value_of(r.lo), past = value_of(r.up);
    __syncthreads();
    for (int b = 0; b < bins; ++b) {
      s.bin.weight[b][threadIdx.x] = 0.0;
      s.bin.count[b][threadIdx.x] = 0;
    }
    x.each_again([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
      each_score<T>(raw, [&](float e, int i) {
        if (e >= first && !(e >= past) && (whole || kept(e, j + i))) {  // (past +infinity: a NaN)
          const uint32_t bits = __float_as_uint(e + 0.0f);  // order_of a number
          const uint32_t o = bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
          const uint32_t b = (o - r.lo) >> shift;
          lane_add(&s.bin.count[b][threadIdx.x], 1);
          if (by == Measure::kQuickWeight) {
            float exponent;
            lane_add(&s.bin.weight[b][threadIdx.x], (double)quick(e - top, &exponent));
          } else if (by == Measure::kWeight) {
            lane_add(&s.bin.weight[b][threadIdx.x], weight(e));
          }
        }
      });
    });
    const double off = by != Measure::kQuickWeight ? 0.0
                       : 0x1p-23 * (0.4 * (weight.top - (double)value_of(r.lo)) * weight.factor + 2.5);
    // from the largest scores down: the bin that reaches the target, or the last
    int b = bins - 1;
    for (;; --b) {
      r.within = sum_all<G>(s.bin.count[b][threadIdx.x], s.found);
      const double reach = by == Measure::kCount
                               ? (double)r.within
                               : sum_all<G>(s.bin.weight[b][threadIdx.x], s.wave[0]);
      if (reach * (1.0 - off) >= r.most) break;
      if (!(reach * (1.0 + off) < r.least) || (b == 0 && by == Measure::kQuickWeight)) return false;
      if (b == 0) break;
      r.most -= reach * (1.0 - off);
      r.least -= reach * (1.0 + off);
    }
    const uint32_t begin = r.lo + ((uint32_t)b << shift);
    const uint64_t end = (uint64_t)begin + (uint64_t(1) << shift);
    r.up = end < r.up ? (uint32_t)end : r.up;
    r.lo = begin;
    __syncthreads();  // the bins are read
  }
}

// ------------------------------------------------------------------------------- draws
// The weights of a row's kept classes, by waves and segments (steps of a walk, whose classes ascend).
template <typename T, int G, int A>
__device__ inline double weigh_row(const Scores<T, G, A> &x, SampleShared<G> &s, const Kept &kept, const Weights &weight,
                                   int steps, int each) {
  constexpr int W = G / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  for (int t = threadIdx.x; t < kSegments * W; t += G) (&s.segment[0][0])[t] = 0.0;
  __syncthreads();
  int step = 0, segment = 0, within = 0;
  double sum = 0.0;
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
    each_four<T>(raw, [&](const float(&v)[4], int i) {
      sum += weight.sum(v, {kept(v[0], j + i), kept(v[1], j + i + 1), kept(v[2], j + i + 2),
                            kept(v[3], j + i + 3)});
    });
    ++step;
    if (++within == each || step == steps) {
      sum = lanes_reduce<Sum, 64>(sum);
      if (lane == 0) s.segment[segment][wave] = sum;
      ++segment;
      within = 0;
      sum = 0.0;
    }
  });
  __syncthreads();
  if (threadIdx.x < kSegments) {
    double part = 0.0;
#pragma unroll 4
    for (int w = 0; w < W; ++w) part += s.segment[threadIdx.x][w];
    s.part[threadIdx.x] = part;
  }
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int k = 0; k < kSegments; ++k) all += s.part[k];
  return all;
}

__device__ inline double target_of(const SampleArgs &a, int64_t row, double all) {
  const double u = (double)a.u[row];
  return (u > 0.0 ? (u < 1.0 ? u : 1.0 - 0x1p-24) : 0.0) * all;
}

// The weights of a row's kept classes, and of those among them that reach `from`.
template <typename T, int G, int A>
__device__ inline double weigh_from(const Scores<T, G, A> &x, SampleShared<G> &s, const Kept &kept,
                                    const Weights &weight, float from, double *reach) {
  double all = 0.0, part = 0.0;
  x.each_again([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
    each_four<T>(raw, [&](const float(&v)[4], int i) {
      double w[4];
      weight.four(v, {kept(v[0], j + i), kept(v[1], j + i + 1), kept(v[2], j + i + 2),
                      kept(v[3], j + i + 3)}, w);
#pragma unroll
      for (int q = 0; q < 4; ++q) part += v[q] >= from ? w[q] : 0.0;
      all += (w[0] + w[1]) + (w[2] + w[3]);
    });
  });
  *reach = sum_all<G>(part, s.wave[0]);
  return sum_all<G>(all, s.wave[1]);
}

// The first class whose weight, with that of the kept ones before it, passes the target, from the sums
// of weigh_row: first its segment, then the step and the lane.
template <typename T, int G, typename Keep>
__device__ inline void draw_row(const SampleArgs &a, int64_t row, SampleShared<G> &s, Keep kept,
                                const Weights &weight, double all, int steps, int each) {
  constexpr int V = kPerLoad<T>;
  const double target = target_of(a, row, all);
  // the last segment with weight that starts at the target or before it
  int segment = 0;
  double before = 0.0, start = 0.0;
  for (int k = 0; k < kSegments; ++k) {
    const double part = s.part[k];
    if (part > 0.0 && before <= target) segment = k, start = before;
    before += part;
  }
  if (threadIdx.x == 0) s.chosen = INT32_MAX, s.last = -1;
  const T *scores = (const T *)a.logits + row * a.ld;
  const int n = a.n_classes;
  for (int step = segment * each; step < steps && step < (segment + 1) * each; ++step) {
    const int64_t wanted = ((int64_t)step * G + threadIdx.x) * V;
    const int j = (int)(wanted < n ? wanted : n);
    RowLoad<T> l;
    if (n < V) {
      l.tiny(scores, j, n, (T)__builtin_nanf(""));
    } else {
      l.issue(scores, j, n);
      l.take(j, n, fill_of((T)__builtin_nanf("")));
    }
    double mine = 0.0, total;
    each_four<T>(l.raw, [&](const float(&v)[4], int i) {
      mine += weight.sum(v, {kept(v[0], j + i), kept(v[1], j + i + 1), kept(v[2], j + i + 2),
                             kept(v[3], j + i + 3)});
    });
    double at = start + lanes_before<G>(mine, s.sum, &total);
    start += total;
    // lanes near the target, whatever the order of their sums rounds to
    if (mine > 0.0) {
      const bool near = at <= target * (1.0 + 0x1p-40) && at + mine >= target * (1.0 - 0x1p-40);
      each_score<T>(l.raw, [&](float v, int i) {
        const double w = kept(v, j + i) ? weight(v) : 0.0;
        at += w;
        if (near && w > 0.0 && at > target) atomicMin(&s.chosen, j + i);
        if (w > 0.0) atomicMax(&s.last, j + i);
      });
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    // (where rounding leaves the target to no class of the segment: its last)
    const int chosen = s.chosen != INT32_MAX ? s.chosen : s.last;
    s.cls = chosen;
    s.share = weight(to_float(scores[chosen])) / all;
  }
}

// The same over the first `count` candidates, which are all that stays.
template <int G>
__device__ inline void draw_listed(const SampleArgs &a, int64_t row, SampleShared<G> &s, int count,
                                   const Weights &weight) {
  // in the order of their classes: the key's halves change places
  __syncthreads();
  for (int t = threadIdx.x; t < count; t += G) {
    const uint64_t key = s.key[t];
    s.key[t] = key << 32 | key >> 32;
  }
  sort_candidates<G>(s, count);
  if (threadIdx.x == 0) s.chosen = INT32_MAX, s.last = -1;
  const Listed<G> l(s, count, weight, 0);
  const double target = target_of(a, row, l.all);
  __syncthreads();
  double at = l.before;
#pragma unroll
  for (int i = 0; i < l.E; ++i) {
    at += l.w[i];
    if (l.w[i] > 0.0) {
      const int t = threadIdx.x * l.E + i;
      if (at > target) atomicMin(&s.chosen, t);
      atomicMax(&s.last, t);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint64_t key = s.key[s.chosen != INT32_MAX ? s.chosen : s.last];
    s.cls = class_of(key >> 32);
    s.share = weight(value_of((uint32_t)key)) / l.all;
  }
}

// The lowest class of the largest score.
template <typename T, int G, int A>
__device__ inline void first_of(const Scores<T, G, A> &x, SampleShared<G> &s, float top) {
  if (threadIdx.x == 0) s.chosen = INT32_MAX;
  __syncthreads();
  int first = INT32_MAX;
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
#pragma unroll
    for (int i = kPerLoad<T> - 1; i >= 0; --i)
      if (element<T>(raw, i) == top && j + i < first) first = j + i;
  });
  if (first < INT32_MAX) atomicMin(&s.chosen, first);
  __syncthreads();
  if (threadIdx.x == 0) s.cls = s.chosen, s.share = 1.0;
}

// What stays is found as a list of candidates in LDS wherever that holds it, and drawn from there; a
// row without cuts is drawn from the sums of its segments, the rest (more kept classes than LDS
// holds, cuts too near to call from quick sums) from memory.
template <typename T, int G, int A>
__device__ inline void sample_row(const SampleArgs &a, int64_t row, SampleShared<G> &s) {
  constexpr int V = kPerLoad<T>, W = G / 64;
  const float inf = __builtin_inff();
  const Scores<T, G, A> x = {(const T *)a.logits + row * a.ld, a.n_classes};
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double temperature = a.temperatures ? (double)a.temperatures[row] : a.temperature;
  const int k = a.top_ks ? a.top_ks[row] : a.top_k;
  const double p = a.top_ps ? (double)a.top_ps[row] : a.top_p;
  const double m = a.min_ps ? (double)a.min_ps[row] : a.min_p;
  const bool by_k = k > 0 && k < a.n_classes, by_p = p < 1.0;
  if (temperature > 1e6) temperature = 1e6;
  const double factor = uniform(1.4426950408889634 / temperature);
  float most = -inf;  // of the lane
  // The sum of its weights relative to its first load's largest, and of each times its exponent's size,
  // in quick floats: exact enough for most cuts by top_p, and done while the row's loads arrive.
  float from_score = 0.0f, lane_size = 0.0f;
  double lane_all = 0.0;
  const QuickWeights quick(factor);
  bool first = true;
  x.each([&](int, const u32x4 &raw) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < V; ++i) most = fmaxf(most, element<T>(raw, i));
    if (first && most > -inf) from_score = most;
    first = false;
    if (by_p && !by_k) {
      float w[V], e[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        w[i] = quick(element<T>(raw, i) - from_score, &e[i]);
        lane_size = __builtin_fmaf(w[i], fabsf(e[i]), lane_size);
      }
#pragma unroll
      for (int n = V / 2; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) w[i] += w[i + n];
      lane_all += (double)w[0];
    }
  });
  float top = lanes_reduce<Max, 64>(most);
  if constexpr (G > 64) {
    if (lane == 0) s.bound[wave] = top;
    __syncthreads();
    top = lanes_reduce<Max, W>(s.bound[threadIdx.x & (W - 1)]);
    __syncthreads();
  }
  top = uniform(top);
  if (top == -inf) {  // nothing to draw from
    if (threadIdx.x == 0) s.cls = -1, s.share = 0.0;
    return;
  }
  if (!(temperature >= 1e-6) || k == 1 || p <= 0.0) {
    first_of<T, G, A>(x, s, top);
    return;
  }
  const Weights weight(top, factor);
  const uint32_t lowest = order_of(-inf) + 1, all_up = order_of(top) + 1;
  // the order of the smallest score that is at least v
  auto order_from = [&](double v) {
    const float f = (float)v;
    const uint32_t o = uniform(order_of(f) + ((double)f < v));
    return o > lowest ? o : lowest;
  };
  // what min_p leaves
  const uint32_t reach_m =
      m > 0.0 ? order_from((double)top + temperature * log(m < 1.0 ? m : 1.0)) : lowest;
  const int steps = (int)(((int64_t)a.n_classes + G * V - 1) / (G * V));
  const int each = (steps + kSegments - 1) / kSegments;
  Kept kept = {-inf, -inf, -1};
  kept.floor = value_of(reach_m);
  if (!by_k && !by_p && reach_m == lowest) {
    const double all = weigh_row<T, G, A>(x, s, kept, weight, steps, each);
    draw_row<T, G>(a, row, s, kept, weight, all, steps, each);
    return;
  }

  // Where the candidates begin.  By top_p: the quick sum is off by what its weights are, and 2^-23 times
  // 1.5 for the sums of a load's weights (0.4 and 4 stand for 0.36 and 3.5).  Classes of a weight below
  // (1 - p) all / n hold less than 1 - p of it together: no cut below.
  uint32_t lo = by_k ? lowest : reach_m;
  double all = 0.0, off = 0.0;
  const bool finite = lane_all <= 0x1p100;
  if (by_p && !by_k) {
    // (rows whose first scores say nothing of the others: infinite sums are not quick)
    const double shift = ((double)from_score - (double)top) * factor;
    const double down = Weights(0.0f, factor).of((double)from_score - (double)top);
    const double lane_off = (double)lane_size + lane_all * fabs(shift);
    const bool held = __all(finite && shift <= 60.0);  // (false for NaN)
    all = held ? lane_all * down : (double)inf;
    off = held ? lane_off * down : (double)inf;
    all = uniform(sum_all<G>(all, s.wave[0]));
    off = uniform(0x1p-23 * (0.4 * sum_all<G>(off, s.wave[1]) + 4.0 * all));
    if (all < (double)inf && off < all) {
      const uint32_t o =
          order_from((double)top + temperature * (log((1.0 - p) * all / a.n_classes) - 1.0));
      lo = o > lo ? o : lo;
    } else {
      all = off = (double)inf;
    }
  }
  uint32_t from = lo;
  const int share = by_k ? (k - 1) / W + 1 : 32;
  if (by_k ? share <= 64 : by_p && a.n_classes > kSorted<G>) {
    // at least that many lanes a wave, so W times as many classes, reach the wave's bound: the upper
    // half of the order of its share-th largest maximum
    const uint32_t mine = order_of(most);
    uint32_t o = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit)
      if (__popcll(__ballot(mine >= (o | 1u << bit))) >= share) o |= 1u << bit;
    if constexpr (G > 64) {
      __syncthreads();
      if (lane == 0) s.found[wave] = (int)(o >> 16);
      __syncthreads();
      o = (uint32_t)-lanes_reduce<Max, W>(-s.found[threadIdx.x & (W - 1)]) << 16;
      __syncthreads();
    }
    o = uniform(o);
    from = o > from ? o : from;
  }
  int count = collect<T, G, A>(
      x, s, [&](float v, int) { return true; }, from, all_up);
  // Without top_k a list that would have to be sorted step by step is not taken: what min_p alone leaves is
  // drawn from memory (20,000 x 500 float, T 1.5, 120 us, sorted 382), a cut by top_p looked for in
  // narrow()'s few bins (top_p 0.95: 165 us, 336).
  bool listed = count <= (by_k ? kSorted<G> : kRanked<G>);
  // where a general cut by top_p is looked for
  Range range = {lo, all_up, p * (all - off), p * (all + off), INT32_MAX};
  bool exact = !(off < all);  // (sums of double weights are needed)
  if (listed) {
    if (by_k || by_p) sort_candidates<G>(s, count);
    if (by_k && count > k) count = k;
    if (by_p) {
      const Listed<G> l(s, count, weight, 32);
      if (by_k) all = l.all;
      const double least = p * (all - off), greatest = p * (all + off);
      if (!(off < all)) {
        listed = false;
      } else if (l.all >= greatest || from == lo) {
        const int stay = l.leading(s, count, least);
        if (off > 0.0 && stay != l.leading(s, count, greatest)) {
          listed = false;
          exact = true;
          range.lo = from;
          range.within = count;
        }
        count = stay;
      } else {
        listed = false;
        if (l.all < least) {
          range.up = from;
          range.least -= l.all;
          range.most -= l.all;
        }
      }
    }
  }
  if (listed) {
    int reach = 0;  // min_p
    for (int t = threadIdx.x; t < count; t += G) reach += (uint32_t)(s.key[t] >> 32) >= reach_m;
    draw_listed<G>(a, row, s, sum_all<G>(reach, s.found), weight);
    return;
  }
  // top_k, then top_p of what that keeps (by quick sums first, where no top_k is), then the draw
  for (int turn = by_k ? 0 : exact ? 2 : 1; turn < 4; ++turn) {
    if ((turn == 1 && by_k) || (turn < 3 && turn > 0 && !by_p)) continue;
    kept.floor = turn == 3 ? value_of(reach_m) : -inf;
    if (turn == 3) {
      const double weights = weigh_row<T, G, A>(x, s, kept, weight, steps, each);
      draw_row<T, G>(a, row, s, kept, weight, weights, steps, each);
      return;
    }
    if (turn == 0) range = {lowest, all_up, (double)k, (double)k, INT32_MAX};
    if (turn == 2) {
      if (by_k) range = {reach_m, all_up, 0.0, 0.0, INT32_MAX};
      double reach;
      const double weights = weigh_from<T, G, A>(x, s, kept, weight, value_of(range.up), &reach);
      range.least = range.most = p * weights - reach;
    }
    const Measure by = turn == 0   ? Measure::kCount
                       : turn == 1 ? Measure::kQuickWeight
                                   : Measure::kWeight;
    if (turn == 1) {
      const Found found = narrow<T, G, A>(x, s, weight, range);
      // (what min_p leaves stays: where no min_p is, the range goes down to where no cut can be)
      if (found == Found::kPast && range.lo == reach_m) turn = 2;
      if (found != Found::kRange) continue;
    }
    if (cut<T, G, A>(x, s, kept, weight, range, by) && turn == 1) turn = 2;
  }
}

template <int G>
__device__ inline void store_draw(const SampleArgs &a, int64_t row, const SampleShared<G> &s) {
  if (threadIdx.x) return;  // (the thread that left the draw there)
  a.ids[row] = s.cls;
  if (a.logp) a.logp[row] = (float)log(s.share);
}

// A workgroup of G lanes a row, with kRing loads on their way.  Many rows: few of them, in so few
// registers that two workgroups of 1024 lanes share a compute unit and hide each other's waits, though some
// registers spill (512 x 50,257 float, top_k 50: two loads 50 us, four 53, four with twice the registers 57;
// top_p 0.95: 245, 256, 260; 2048 x 128,000 without cuts 682, 744, 776).  A row or two for each compute
// unit: more, and twice the registers (1 x 128,000 bfloat16, top_k 50 and top_p 0.9: 25 us, with two loads
// 27; top_p 0.95 148, 165).
template <typename T, int G, int kRing>
__global__ __launch_bounds__(G, G >= 512 && kRing < 8 ? 8 : 4) void sample_kernel(SampleArgs a) {
  __shared__ __attribute__((aligned(16))) SampleShared<G> s;
  const int64_t row = a.first + blockIdx.x;
  sample_row<T, G, kRing>(a, row, s);
  store_draw<G>(a, row, s);
}

int launch_sample(const SampleArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t bytes = (int64_t)a.n_classes * (int)sizeof(T);
    auto of = [&](auto k, int threads) { return launch_each_row(k, threads, a, stream); };
    // top_k of more than a wave's 64 maxima, of more classes than its LDS holds: more waves, or there is
    // no bound (us, one wave / four: 8192 x 4000 bfloat16, top_k 200 326 / 272; 50,000 x 500 float, which
    // LDS holds, 630 / 1400)
    const int k = a.top_ks || a.top_k >= a.n_classes ? 0 : a.top_k;
    const int64_t most = k > 64 && a.n_classes > kSorted<64> && bytes <= 16384 ? 16384 : bytes;
    if (most <= 4096) return of(sample_kernel<T, 64, 4>, 64);
    if (most <= 8192) return of(sample_kernel<T, 128, 4>, 128);
    if (a.n_rows <= 256) return of(sample_kernel<T, 1024, 8>, 1024);
    if (most <= 32768) return of(sample_kernel<T, 256, 4>, 256);
    if (most <= 65536) return of(sample_kernel<T, 512, 2>, 512);
    return of(sample_kernel<T, 1024, 2>, 1024);
  });
}

}  // namespace bridger
