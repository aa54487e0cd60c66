// scores.h -- the order of a row's class scores, as top_k and sample keep it.
#pragma once
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

}  // namespace bridger
