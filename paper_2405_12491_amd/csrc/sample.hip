// sample.hip -- gfx950 kernels of bridger_sample: a class of every row, drawn from its scores.
#include "scores.h"

namespace bridger {

// 2^x, x <= 0: 2^n times the series of e^(f ln 2), |f| <= 1/2, whose rest is below 7e-15 of it.  A
// draw compares sums of these with a random number, so they are held in double.
__device__ inline double exp2_of(double x) {
  if (!(x > -1100.0)) return 0.0;
  const double n = __builtin_rint(x), f = x - n;
  double s = 7.0549116208011233e-09;  // (ln 2)^k / k!, k = 11 to 0
  s = __builtin_fma(s, f, 1.0178086009239699e-07);
  s = __builtin_fma(s, f, 1.3215486790144309e-06);
  s = __builtin_fma(s, f, 1.5252733804059840e-05);
  s = __builtin_fma(s, f, 1.5403530393381610e-04);
  s = __builtin_fma(s, f, 1.3333558146428443e-03);
  s = __builtin_fma(s, f, 9.6181291076284772e-03);
  s = __builtin_fma(s, f, 5.5504108664821580e-02);
  s = __builtin_fma(s, f, 2.4022650695910071e-01);
  s = __builtin_fma(s, f, 6.9314718055994531e-01);
  s = __builtin_fma(s, f, 1.0);
  return __builtin_ldexp(s, (int)n);
}

template <int G>
constexpr int kSorted = G >= 1024 ? 2048 : G > 64 ? 1024 : 512;  // candidates that LDS holds

constexpr int kSegments = 16;  // of a row, whose sums the draw keeps

template <int G>
struct SampleShared {
  uint64_t key[kSorted<G>];
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

// A row's weights: e^((v - top) / T), 1 for the largest.
struct Weights {
  float top;
  double factor;  // log2(e) / T
  __device__ double operator()(float v) const {
    return v == top ? 1.0 : exp2_of(((double)v - (double)top) * factor);
  }
};

// ---------------------------------------------------------------------------- candidates
// Scores of [lo, up) in the order that `kept` keeps go to the candidates; their number (it may pass
// kSorted, whose entries alone are there).
template <typename T, int G, typename Source, typename Keep>
__device__ inline int collect(Source &x, SampleShared<G> &s, Keep kept, uint32_t lo, uint32_t up) {
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
      each_score<T>(raw, [&](float v, int i) {
        if (v >= low && order_of(v) < up && kept(v, j + i)) {
          const int at = atomicAdd(&s.count, 1);
          if (at < kSorted<G>) s.key[at] = key_of(v, j + i);
        }
      });
    }
  });
  __syncthreads();
  return s.count;
}

// Sorts the first `count` candidates, the largest first (zeros behind): compare and exchange over a
// network of the next power of two.
template <int G>
__device__ inline void sort_candidates(SampleShared<G> &s, int count) {
  int size = 64;
  while (size < count) size *= 2;
  __syncthreads();
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
// less than `target` of the weight stands): halves the range [lo, up) that holds it, `base` being
// what reaches up, until LDS holds it or one score is left, that of many classes.  Its walks read the
// row from memory again: held in registers they would make up most of the code.
template <typename T, int G>
__device__ inline void cut(InMemory<T, G> &x, SampleShared<G> &s, Kept &kept, const Weights &weight,
                           bool by_weight, double target) {
  const uint32_t lowest = order_of(-__builtin_inff()) + 1;
  uint32_t lo = lowest, up = order_of(weight.top) + 1;
  double base = 0.0;
  while (lo < up) {
    const uint32_t middle = lo + (up - lo) / 2;
    const int count = collect<T, G>(x, s, kept, middle, up);
    const float v = value_of(middle);
    double reach = base + count;
    if (count <= kSorted<G>) {
      sort_candidates<G>(s, count);
      int stay = target - base < count ? (int)(target - base) : count;
      if (by_weight) {
        const Listed<G> l(s, count, weight, 32);
        stay = l.leading(s, count, target - base);
        reach = base + l.all;
      }
      if (count && (reach >= target || middle == lo)) {
        const uint64_t key = s.key[stay > 0 ? stay - 1 : 0];
        kept.score = value_of((uint32_t)(key >> 32));
        kept.cls = class_of(key);
        return;
      }
    } else if (up - middle == 1) {
      const double one = by_weight ? weight(v) : 1.0;
      reach = base + count * one;
      if (reach >= target || middle == lo) {
        double want = __builtin_ceil((target - base) / one);  // of its classes
        if (!(want >= 1.0)) want = 1.0;
        int32_t cls = 0;
        for (int bit = 30; bit >= 0; --bit) {  // the largest class with fewer than those before it
          const int32_t next = cls | 1 << bit;
          int below = 0;
          x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
            each_score<T>(raw, [&](float e, int i) {
              below += e == v && j + i < next && kept(e, j + i);
            });
          });
          if ((double)sum_all<G>(below, s.found) < want) cls = next;
        }
        kept.score = v;
        kept.cls = cls;
        return;
      }
    } else if (by_weight) {
      double w = 0.0;
      x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
        each_score<T>(raw, [&](float e, int i) {
          if (e >= v && order_of(e) < up && kept(e, j + i)) w += weight(e);
        });
      });
      reach = base + sum_all<G>(w, s.wave[0]);
    }
    if (reach >= target) {
      if (middle == lo) return;  // (not reached: a range of one score is settled above)
      lo = middle;
    } else {
      base = reach;
      up = middle;
    }
  }
  // all of it stays: rounding leaves the target past the last
}

// ------------------------------------------------------------------------------- draws
// The weights of a row's kept classes, by waves and segments (steps of a walk, whose classes ascend).
template <typename T, int G, typename Source, typename Keep>
__device__ inline double weigh_row(Source &x, SampleShared<G> &s, Keep kept, const Weights &weight,
                                   int steps, int each) {
  constexpr int W = G / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  for (int t = threadIdx.x; t < kSegments * W; t += G) (&s.segment[0][0])[t] = 0.0;
  __syncthreads();
  int step = 0, segment = 0, within = 0;
  double sum = 0.0;
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
    each_score<T>(raw, [&](float v, int i) {
      if (kept(v, j + i)) sum += weight(v);
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
    each_score<T>(l.raw, [&](float v, int i) {
      if (kept(v, j + i)) mine += weight(v);
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
template <typename T, int G>
__device__ inline void first_of(const SampleArgs &a, int64_t row, SampleShared<G> &s, float top) {
  InMemory<T, G> x((const T *)a.logits + row * a.ld, a.n_classes);
  if (threadIdx.x == 0) s.chosen = INT32_MAX;
  __syncthreads();
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
#pragma unroll
    for (int i = kPerLoad<T> - 1; i >= 0; --i)
      if (element<T>(raw, i) == top) atomicMin(&s.chosen, j + i);
  });
  __syncthreads();
  if (threadIdx.x == 0) s.cls = s.chosen, s.share = 1.0;
}

// What stays is found as a list of candidates in LDS wherever that holds it, and drawn from there; a
// row without cuts is drawn from the sums of its segments, the rest (more kept classes than LDS
// holds) from memory.
template <typename T, int G, typename Source>
__device__ inline void sample_row(const SampleArgs &a, int64_t row, Source &x,
                                  SampleShared<G> &s) {
  constexpr int V = kPerLoad<T>, W = G / 64;
  const float inf = __builtin_inff();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double temperature = a.temperatures ? (double)a.temperatures[row] : a.temperature;
  const int k = a.top_ks ? a.top_ks[row] : a.top_k;
  const double p = a.top_ps ? (double)a.top_ps[row] : a.top_p;
  const double m = a.min_ps ? (double)a.min_ps[row] : a.min_p;
  float most = -inf;  // of the lane
  x.each([&](int, const u32x4 &raw) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < V; ++i) most = fmaxf(most, element<T>(raw, i));
  });
  float top = lanes_reduce<Max, 64>(most);
  if constexpr (G > 64) {
    if (lane == 0) s.bound[wave] = top;
    __syncthreads();
    top = lanes_reduce<Max, W>(s.bound[threadIdx.x & (W - 1)]);
    __syncthreads();
  }
  if (top == -inf) {  // nothing to draw from
    if (threadIdx.x == 0) s.cls = -1, s.share = 0.0;
    return;
  }
  if (!(temperature >= 1e-6) || k == 1 || p <= 0.0) {
    first_of<T, G>(a, row, s, top);
    return;
  }
  if (temperature > 1e6) temperature = 1e6;
  const Weights weight = {top, 1.4426950408889634 / temperature};
  const uint32_t lowest = order_of(-inf) + 1, all_up = order_of(top) + 1;
  float least = value_of(lowest);  // what min_p leaves
  if (m > 0.0) {
    const double v = (double)top + temperature * log(m < 1.0 ? m : 1.0);
    float f = (float)v;
    if ((double)f < v) f = value_of(order_of(f) + 1);
    least = f > least ? f : least;
  }
  const int steps = (int)(((int64_t)a.n_classes + G * V - 1) / (G * V));
  const int each = (steps + kSegments - 1) / kSegments;
  auto valid = [&](float v, int) { return v >= value_of(lowest); };
  auto stays = [&](float v, int) { return v >= least; };
  // at least j lanes a wave, so W j classes, reach the j-th largest of their maxima
  auto bound_of = [&](int j) {
    float b = wave_jth(most, j);
    if constexpr (G > 64) {
      __syncthreads();
      if (lane == 0) s.bound[wave] = b;
      __syncthreads();
      b = -lanes_reduce<Max, W>(-s.bound[threadIdx.x & (W - 1)]);
    }
    const uint32_t o = order_of(b);
    return o > lowest ? o : lowest;
  };
  const bool by_k = k > 0 && k < a.n_classes, by_p = p < 1.0;
  if (!by_k && !by_p) {
    const double all = weigh_row<T, G>(x, s, stays, weight, steps, each);
    draw_row<T, G>(a, row, s, stays, weight, all, steps, each);
    return;
  }
  double all = 0.0;
  if (!by_k) all = weigh_row<T, G>(x, s, valid, weight, steps, each);
  const int share = by_k ? (k + W - 1) / W : 32;
  const uint32_t bound =
      (by_k ? share > 64 : a.n_classes <= kSorted<G>) ? lowest : bound_of(share);
  int count = collect<T, G>(x, s, valid, bound, all_up);
  InMemory<T, G> row_again((const T *)a.logits + row * a.ld, a.n_classes);
  Kept kept = {-inf, least, -1};
  bool listed = count <= kSorted<G>;
  if (by_k) {
    if (!listed) {
      // (count of them reach the bound at least, more than LDS holds)
      Kept all_of = {-inf, -inf, -1};
      cut<T, G>(row_again, s, all_of, weight, false, (double)k);
      kept.score = all_of.score;
      kept.cls = all_of.cls;
      all_of.floor = -inf;
      if (k <= kSorted<G>) {
        count = collect<T, G>(row_again, s, all_of, lowest, all_up);
        listed = true;
      }
    }
    if (listed) {
      sort_candidates<G>(s, count);
      if (count > k) count = k;
      if (by_p) {
        const Listed<G> l(s, count, weight, 32);
        count = l.leading(s, count, p * l.all);
      }
    } else if (by_p) {
      Kept of_k = {kept.score, -inf, kept.cls};
      all = weigh_row<T, G>(row_again, s, of_k, weight, steps, each);
      cut<T, G>(row_again, s, of_k, weight, true, p * all);
      kept.score = of_k.score;
      kept.cls = of_k.cls;
    }
  } else {
    if (listed) {
      sort_candidates<G>(s, count);
      const Listed<G> l(s, count, weight, 32);
      const double target = p * all;
      listed = l.all >= target || bound == lowest;
      if (listed) count = l.leading(s, count, target);
    }
    if (!listed) {
      Kept all_of = {-inf, -inf, -1};
      cut<T, G>(row_again, s, all_of, weight, true, p * all);
      kept.score = all_of.score;
      kept.cls = all_of.cls;
    }
  }
  if (listed) {
    if (m > 0.0) {
      int reach = 0;
      for (int t = threadIdx.x; t < count; t += G)
        reach += value_of((uint32_t)(s.key[t] >> 32)) >= least;
      count = sum_all<G>(reach, s.found);
    }
    draw_listed<G>(a, row, s, count, weight);
  } else {
    all = weigh_row<T, G>(row_again, s, kept, weight, steps, each);
    draw_row<T, G>(a, row, s, kept, weight, all, steps, each);
  }
}

template <int G>
__device__ inline void store_draw(const SampleArgs &a, int64_t row, const SampleShared<G> &s) {
  if (threadIdx.x) return;  // (the thread that left the draw there)
  a.ids[row] = s.cls;
  if (a.logp) a.logp[row] = (float)log(s.share);
}

// A workgroup of G lanes a row, which stays in their registers.
template <typename T, int G, int C>
__global__ __launch_bounds__(G) void sample_kernel(SampleArgs a) {
  __shared__ __attribute__((aligned(16))) SampleShared<G> s;
  const int64_t row = a.first + blockIdx.x;
  InRegisters<T, G, C> x((const T *)a.logits + row * a.ld, a.n_classes);
  sample_row<T, G>(a, row, x, s);
  store_draw<G>(a, row, s);
}

// Rows below 16 bytes, and rows that do not fit a workgroup's registers: every walk reads the row.
template <typename T, int G>
__global__ __launch_bounds__(G) void sample_memory_kernel(SampleArgs a) {
  __shared__ __attribute__((aligned(16))) SampleShared<G> s;
  const int64_t row = a.first + blockIdx.x;
  InMemory<T, G> x((const T *)a.logits + row * a.ld, a.n_classes);
  sample_row<T, G>(a, row, x, s);
  store_draw<G>(a, row, s);
}

int launch_sample(const SampleArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t bytes = (int64_t)a.n_classes * (int)sizeof(T);
    auto of = [&](auto k, int threads) { return launch_each_row(k, threads, a, stream); };
    if (bytes < 16) return of(sample_memory_kernel<T, 64>, 64);
    if (bytes <= 1024) return of(sample_kernel<T, 64, 1>, 64);
    if (bytes <= 2048) return of(sample_kernel<T, 64, 2>, 64);
    if (bytes <= 4096) return of(sample_kernel<T, 64, 4>, 64);
    if (bytes <= 8192) return of(sample_kernel<T, 128, 4>, 128);
    if (bytes <= 16384) return of(sample_kernel<T, 256, 4>, 256);
    if (bytes <= 32768) return of(sample_kernel<T, 256, 8>, 256);
    if (bytes <= 65536) return of(sample_kernel<T, 512, 8>, 512);
    if (bytes <= 131072) return of(sample_kernel<T, 512, 16>, 512);
    if (bytes <= 262144) return of(sample_kernel<T, 1024, 16>, 1024);
    return of(sample_memory_kernel<T, 1024>, 1024);
  });
}

}  // namespace bridger
