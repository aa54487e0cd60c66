// scores.h -- rows of class scores as top_k and sample read them: their order, a workgroup's walk over
// one row, and a wave's j-th largest value.
#pragma once
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

// The j-th largest of a wave's 64 values (-infinity for those without one).
__device__ inline float wave_jth(float v, int j) {
  // as many larger ones as there are: the values with fewer than j of them are the j largest
  int larger = 0;
#pragma unroll
  for (int l = 0; l < 64; ++l)
    larger += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)) > v;
  return -lanes_reduce<Max, 64>(larger < j ? -v : -__builtin_inff());
}

}  // namespace bridger
