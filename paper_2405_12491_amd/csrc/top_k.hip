// top_k.hip -- gfx950 kernels of bridger_top_k: the k largest scores of every row.
#include <utility>

#include "rows.h"

namespace bridger {

// A score's place in the order: larger is earlier.  Floats map to unsigned integers of the same
// order, -0 as +0, NaN (below -infinity) as 0.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t order) {
  return __uint_as_float(order ^ (order & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}
// With its class: of equal scores the lower class is the larger key.  Never 0.
__device__ inline uint64_t key_of(float x, int32_t cls) {
  return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - (uint32_t)cls);
}
__device__ inline int32_t class_of(uint64_t key) {
  return (int32_t)(0xFFFFFFFFu - (uint32_t)key);
}

template <typename T>
__device__ inline void store_slot(const TopKArgs &a, int64_t row, int at, T value, int32_t id) {
  if (a.values) ((T *)a.values)[row * a.k + at] = value;
  if (a.ids) a.ids[row * a.k + at] = id;
}

// ============================================================================ FEW CLASSES
// One lane a row: its K best so far stay sorted in registers.  Classes come in ascending order and
// a score goes behind its equals, so those stay in the order of their classes.  1M x 10 float, k =
// 4: 72 MB in 16 us (4.6 TB/s); with more slots bound by the insertion, classes x k steps of five
// instructions.
template <typename T, int K>
__global__ __launch_bounds__(256) void top_k_lane_kernel(TopKArgs a) {
  constexpr int V = kPerLoad<T>;
  const int64_t row = row_of<1>(a.first);
  if (row >= a.n_rows) return;
  const int n = a.n_classes;
  const T *x = (const T *)a.scores + row * a.ld;
  uint32_t best[K];
  int32_t id[K];
#pragma unroll
  for (int p = 0; p < K; ++p) best[p] = 0, id[p] = -1;
  for (int j = 0; j < n; j += V) {
    RowLoad<T> l;
    if (n < V) {
      l.tiny(x, j, n, (T)0.0f);
    } else {
      l.issue(x, j, n);
      l.take(j, n, 0);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t o = j + i < n ? order_of(element<T>(l.raw, i)) + 1 : 0;  // 0: an empty slot
#pragma unroll
      for (int p = K - 1; p >= 0; --p) {
        // past every slot that is not smaller; the smaller ones move down
        const bool here = o > best[p], above = p > 0 && o > best[p > 0 ? p - 1 : 0];
        best[p] = above ? best[p > 0 ? p - 1 : 0] : here ? o : best[p];
        id[p] = above ? id[p > 0 ? p - 1 : 0] : here ? j + i : id[p];
      }
    }
  }
  T value[K];
#pragma unroll
  for (int p = 0; p < K; ++p) {
    const float v = value_of(best[p] - 1);
    // the order holds a score's value, but not which zero or NaN it was
    value[p] = id[p] < 0 ? (T)-__builtin_inff()
               : v == 0.0f || v != v ? x[id[p]] : from_float<T>(v);
  }
  if (a.k == K) {  // whole slots of a lane in one store: a store of one slot each takes 64 cycles
    if (a.values) __builtin_memcpy((T *)a.values + row * K, value, sizeof(value));
    if (a.ids) __builtin_memcpy(a.ids + row * K, id, sizeof(id));
  } else {
#pragma unroll
    for (int p = 0; p < K; ++p)
      if (p < a.k) store_slot<T>(a, row, p, value[p], id[p]);
  }
}

// =========================================================================== MANY CLASSES
// One workgroup of G lanes a row.  Every wave takes the j-th largest of its 64 lanes' maxima, j the
// waves' share of k; the smallest of those bounds the k-th largest score from below, since at least
// k scores, one a lane, reach it.  The few scores that reach it are collected in LDS and ranked by
// counting the larger ones.  Rows where too many or too few reach it (many equal scores, masked or
// broken rows) take the general way below.
// Long rows are bound by memory: 2048 x 128,000 bfloat16, k = 64, read once, 524 MB in 120 us (4.4
// TB/s); short ones by a row's fixed steps (bound, collection, ranking): 100,000 x 1000, k = 10,
// 200 MB in 82.
template <int G>
constexpr int kCandidates = G == 64 ? 512 : 1024;  // of one wave: less LDS, so that many fit a CU

// Where the row's scores are.  each(f): f(first class, 16 bytes of scores), the classes kStep
// apart, in ascending order per lane; NaN past the row's end.  All lanes make the same number of
// calls. In registers, lane after lane with whole loads: rows of at least 16 bytes.
template <typename T, int G, int C>
struct InRegisters {
  static constexpr int kStep = 1;
  RowLoad<T> x[C];
  __device__ InRegisters(const T *row, int n) {
    const uint32_t nan = fill_of((T)__builtin_nanf(""));
#pragma unroll
    for (int c = 0; c < C; ++c) x[c].issue(row, (c * G + (int)threadIdx.x) * kPerLoad<T>, n);
#pragma unroll
    for (int c = 0; c < C; ++c) x[c].take((c * G + (int)threadIdx.x) * kPerLoad<T>, n, nan);
  }
  template <typename F>
  __device__ void each(F f) {
    each_of(f, std::make_integer_sequence<int, C>());
  }
  // written out: a loop that stayed one would index registers
  template <typename F, int... c>
  __device__ void each_of(F f, std::integer_sequence<int, c...>) {
    ((forget(x[c].raw), f((c * G + (int)threadIdx.x) * kPerLoad<T>, x[c].raw)), ...);
  }
};
// In registers, class after class on neighbouring lanes: short rows, whose whole loads would leave
// most lanes without a score, and their maxima without a bound.
template <typename T, int G>
struct InLanes {
  static constexpr int kStep = G;
  u32x4 raw;
  __device__ InLanes(const T *row, int n) {
    T e[kPerLoad<T>];
#pragma unroll
    for (int i = 0; i < kPerLoad<T>; ++i) {
      const int j = i * G + (int)threadIdx.x;
      e[i] = j < n ? row[j] : (T)__builtin_nanf("");
    }
    __builtin_memcpy(&raw, e, 16);
  }
  template <typename F>
  __device__ void each(F f) {
    f((int)threadIdx.x, raw);
  }
};
// In memory: every walk reads the row again.
template <typename T, int G>
struct InMemory {
  static constexpr int kStep = 1;
  const T *row;
  int n;
  __device__ InMemory(const T *row, int n) : row(row), n(n) {}
  template <typename F>
  __device__ void each(F f) {
    for (int64_t j0 = 0; j0 < n; j0 += G * kPerLoad<T>) {
      const int64_t j = j0 + (int64_t)threadIdx.x * kPerLoad<T>;
      const int at = (int)(j < n ? j : n);
      RowLoad<T> l;
      if (n < kPerLoad<T>) {
        l.tiny(row, at, n, (T)__builtin_nanf(""));
      } else {
        l.issue(row, at, n);
        l.take(at, n, fill_of((T)__builtin_nanf("")));
      }
      f(at, l.raw);
    }
  }
};

template <int G>
struct TopKShared {
  uint64_t key[kCandidates<G> + 8];
  float value[kCandidates<G>];
  float bound[G / 64];
  int wave[2][G / 64];
  int count;
};

// The waves' sum of v; all lanes call it.
template <int G>
__device__ inline int count_all(int v, TopKShared<G> &s) {
  v = lanes_reduce<Sum, 64>(v);
  if constexpr (G > 64) {
    __syncthreads();  // the last count is read
    if ((threadIdx.x & 63) == 0) s.wave[0][threadIdx.x >> 6] = v;
    __syncthreads();
    v = lanes_reduce<Sum, G / 64>(s.wave[0][threadIdx.x & (G / 64 - 1)]);
  }
  return v;
}

// Scores for which `reach` holds go to the candidates; their number (it may pass kCandidates, whose
// entries alone are kept).  `top` is the lane's largest score of one load.
template <typename T, int G, typename Source, typename Reach>
__device__ inline int collect(Source &x, TopKShared<G> &s, Reach reach) {
  constexpr int V = kPerLoad<T>;
  __syncthreads();
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
    float top = element<T>(raw, 0);
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, element<T>(raw, i));
    if (reach(top)) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float v = element<T>(raw, i);
        if (reach(v)) {
          const int at = atomicAdd(&s.count, 1);
          if (at < kCandidates<G>) {
            s.key[at] = key_of(v, j + i * Source::kStep);
            s.value[at] = v;
          }
        }
      }
    }
  });
  __syncthreads();
  return s.count;
}

// Ranks the first `count` candidates and stores those of rank below k.
template <typename T, int G>
__device__ inline void store_ranked(const TopKArgs &a, int64_t row, TopKShared<G> &s, int count,
                                    int k) {
  if (threadIdx.x < 8) s.key[count + threadIdx.x] = 0;
  __syncthreads();
  for (int t = threadIdx.x; t < count; t += G) {
    const uint64_t mine = s.key[t];
    int rank = 0;
    for (int q = 0; q < count; q += 8) {  // four loads on their way at once
      ulonglong2 other[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) other[i] = *(const ulonglong2 *)&s.key[q + 2 * i];
#pragma unroll
      for (int i = 0; i < 4; ++i) rank += (other[i].x > mine) + (other[i].y > mine);
    }
    if (rank < k) store_slot<T>(a, row, rank, from_float<T>(s.value[t]), class_of(mine));
  }
}

// Stores scores for which `is` holds in ascending class order from slot `at` on; the next free
// slot.
template <typename T, int G, typename Source, typename Is>
__device__ inline int store_in_order(const TopKArgs &a, int64_t row, Source &x, TopKShared<G> &s,
                                     int at, int k, Is is) {
  constexpr int V = kPerLoad<T>, W = G / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int turn = 0;
  x.each([&](int j, const u32x4 &raw) __attribute__((always_inline)) {
    if (at >= k) return;  // of the whole workgroup
    int before = 0, all = 0, mine = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool yes = i < a.n_classes - j && is(element<T>(raw, i));
      const uint64_t lanes = __ballot(yes);
      before += __popcll(lanes & ((uint64_t(1) << lane) - 1));
      all += __popcll(lanes);
      mine |= yes << i;
    }
    int first = at;
    if constexpr (G > 64) {
      if (lane == 0) s.wave[turn][wave] = all;
      __syncthreads();
      all = 0;
      for (int w = 0; w < W; ++w) {
        if (w < wave) first += s.wave[turn][w];
        all += s.wave[turn][w];
      }
      turn ^= 1;
    }
    int slot = first + before;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (mine >> i & 1) {
        if (slot < k) store_slot<T>(a, row, slot, from_float<T>(element<T>(raw, i)), j + i);
        ++slot;
      }
    at += all;
  });
  return at < k ? at : k;
}

// The j-th largest of a wave's 64 values (-infinity for those without one).
__device__ inline float wave_jth(float v, int j) {
  // as many larger ones as there are: the values with fewer than j of them are the j largest
  int larger = 0;
#pragma unroll
  for (int l = 0; l < 64; ++l)
    larger += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)) > v;
  return -lanes_reduce<Max, 64>(larger < j ? -v : -__builtin_inff());
}

// The general way, from any lower bound of the k-th largest score (-infinity where fewer than k are
// numbers): scores above it first, then those equal to it and at last NaN, in ascending class
// order. Where too many lie above it, the k-th largest score is found bit by bit and becomes the
// bound. Its walks read the row from memory again (from the caches): held in registers they would
// make up most of the kernel's code.
template <typename T, int G>
__device__ inline void store_general(const TopKArgs &a, int64_t row, InMemory<T, G> &x,
                                     TopKShared<G> &s, float bound, int k) {
  constexpr int V = kPerLoad<T>;
  int count = collect<T, G>(x, s, [&](float v) { return v > bound; });
  if (count > kCandidates<G>) {
    uint32_t order = 0;
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
      int reach = 0;
      x.each([&](int, const u32x4 &raw) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < V; ++i) reach += order_of(element<T>(raw, i)) >= (order | bit);
      });
      if (count_all<G>(reach, s) >= k) order |= bit;
    }
    bound = value_of(order);
    count = collect<T, G>(x, s, [&](float v) { return v > bound; });
  }
  store_ranked<T, G>(a, row, s, count, k);
  int stored = count < k ? count : k;
  __syncthreads();
  stored = store_in_order<T, G>(a, row, x, s, stored, k, [&](float v) { return v == bound; });
  __syncthreads();
  store_in_order<T, G>(a, row, x, s, stored, k, [&](float v) { return v != v; });
}

template <typename T, int G, typename Source>
__device__ inline void top_k_row(const TopKArgs &a, int64_t row, Source &x, TopKShared<G> &s) {
  constexpr int V = kPerLoad<T>, W = G / 64;
  const float inf = __builtin_inff();
  const int k = a.k < a.n_classes ? a.k : a.n_classes;
  float top = -inf;
  x.each([&](int, const u32x4 &raw) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < V; ++i) top = fmaxf(top, element<T>(raw, i));
  });
  // (a share is at most 64: launch_top_k gives more than 64 slots four waves or more)
  float bound = wave_jth(top, (k + W - 1) / W);
  if constexpr (G > 64) {
    if ((threadIdx.x & 63) == 0) s.bound[threadIdx.x >> 6] = bound;
    __syncthreads();
    bound = -lanes_reduce<Max, W>(-s.bound[threadIdx.x & (W - 1)]);
  }
  int count = collect<T, G>(x, s, [&](float v) { return v >= bound; });
  if (count >= k && count <= kCandidates<G>) {
    store_ranked<T, G>(a, row, s, count, k);
  } else {
    InMemory<T, G> m((const T *)a.scores + row * a.ld, a.n_classes);
    store_general<T, G>(a, row, m, s, bound, k);
  }
  for (int p = k + threadIdx.x; p < a.k; p += G) store_slot<T>(a, row, p, (T)-inf, -1);
}

template <typename T, int G, int C>
__global__ __launch_bounds__(G, C <= 8 ? 8 : 4) void top_k_kernel(TopKArgs a) {
  __shared__ __attribute__((aligned(16))) TopKShared<G> s;
  const int64_t row = a.first + blockIdx.x;
  InRegisters<T, G, C> x((const T *)a.scores + row * a.ld, a.n_classes);
  top_k_row<T, G>(a, row, x, s);
}

template <typename T, int G>
__global__ __launch_bounds__(G, 8) void top_k_short_kernel(TopKArgs a) {
  __shared__ __attribute__((aligned(16))) TopKShared<G> s;
  const int64_t row = a.first + blockIdx.x;
  InLanes<T, G> x((const T *)a.scores + row * a.ld, a.n_classes);
  top_k_row<T, G>(a, row, x, s);
}

// Rows that do not fit a workgroup's registers: they are read twice, for the bound and for the
// candidates.  2048 x 128,000 float, k = 64, 1.05 GB in 328 us; x 140,000 bfloat16, 573 MB in 213.
template <typename T>
__global__ __launch_bounds__(1024) void top_k_long_kernel(TopKArgs a) {
  __shared__ __attribute__((aligned(16))) TopKShared<1024> s;
  const int64_t row = a.first + blockIdx.x;
  InMemory<T, 1024> x((const T *)a.scores + row * a.ld, a.n_classes);
  top_k_row<T, 1024>(a, row, x, s);
}

int launch_top_k(const TopKArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t bytes = (int64_t)a.n_classes * (int)sizeof(T);
    // a lane's work is classes x k: beyond a few steps it takes many rows to pay (64 classes, k =
    // 16, us, a lane / a wave a row: 8192 rows 16 / 8, 100,000 27 / 56)
    if (a.k <= 32 && a.n_classes <= 64 &&
        ((int64_t)a.n_classes * a.k <= 64 || a.n_rows >= 32768)) {
      auto lane = [&](auto k) { return launch_rows(k, 1, a, stream); };
      return a.k == 1   ? lane(top_k_lane_kernel<T, 1>)
             : a.k == 2 ? lane(top_k_lane_kernel<T, 2>)
             : a.k <= 4 ? lane(top_k_lane_kernel<T, 4>)
             : a.k <= 8 ? lane(top_k_lane_kernel<T, 8>)
             : a.k <= 16 ? lane(top_k_lane_kernel<T, 16>)
                         : lane(top_k_lane_kernel<T, 32>);
    }
    auto of = [&](auto k, int threads) { return launch_each_row(k, threads, a, stream); };
    const int k = a.k < a.n_classes ? a.k : a.n_classes;
    // Few waves a row, each of which pays for its bound and its meetings, but so many that about
    // half of their lanes hold one of the k (bfloat16, us, one / two / four waves: 100,000 x 1000,
    // k = 10 82 / 133 / 216, k = 64 647 / 209 / 289; 10,000 x 8000, k = 20 37 / 36 / 40, k = 64 309
    // / 55 / 55).
    const bool small = a.n_classes <= 128;
    if (bytes <= 1024 && (k <= 32 || (small && k <= 64))) return of(top_k_short_kernel<T, 64>, 64);
    if (bytes <= 2048 && k > 32 && k <= 64) return of(top_k_short_kernel<T, 128>, 128);
    if (bytes <= 4096 && k > 64) return of(top_k_short_kernel<T, 256>, 256);
    if (bytes <= 2048 && k <= 32) return of(top_k_kernel<T, 64, 2>, 64);
    if (bytes <= 4096 && k <= 32) return of(top_k_kernel<T, 64, 4>, 64);
    if (bytes <= 8192 && k <= 32) return of(top_k_kernel<T, 64, 8>, 64);
    if (bytes <= 8192 && k <= 64) return of(top_k_kernel<T, 128, 4>, 128);
    if (bytes <= 16384 && k <= 32) return of(top_k_kernel<T, 128, 8>, 128);
    if (bytes <= 16384) return of(top_k_kernel<T, 256, 4>, 256);
    if (bytes <= 32768) return of(top_k_kernel<T, 256, 8>, 256);
    if (bytes <= 65536) return of(top_k_kernel<T, 512, 8>, 512);
    if (bytes <= 131072) return of(top_k_kernel<T, 512, 16>, 512);
    if (bytes <= 262144) return of(top_k_kernel<T, 1024, 16>, 1024);
    return of(top_k_long_kernel<T>, 1024);
  });
}

}  // namespace bridger
