// top_k.hip -- gfx950 kernels of bridger_top_k: the k largest scores of every row.
#include "rows.h"

namespace bridger {

// A score's place in the order, with its class: larger is earlier.  The upper word maps floats to
// unsigned integers of the same order (-0 as +0, NaN below -infinity as 0), the lower word is the
// class, inverted, so that equal scores rank by the lower class.  Never 0: classes are below 2^31.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ inline uint64_t key_of(float x, int32_t cls) {
  return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - (uint32_t)cls);
}
__device__ inline int32_t class_of(uint64_t key) {
  return (int32_t)(0xFFFFFFFFu - (uint32_t)key);
}

template <typename T>
__device__ inline T minus_infinity() {
  return (T)(-__builtin_inff());
}

// One workgroup a row: k times the largest key below the last one.
template <typename T>
__global__ __launch_bounds__(256) void top_k_kernel(TopKArgs a) {
  __shared__ uint64_t lds[4];
  const T *scores = (const T *)a.scores;
  for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
    const T *x = scores + row * a.ld;
    uint64_t last = ~uint64_t(0);
    for (int i = 0; i < a.k; ++i) {
      uint64_t best = 0;
      for (int64_t j = threadIdx.x; j < a.n_classes; j += 256) {
        const uint64_t key = key_of(to_float(x[j]), (int32_t)j);
        if (key < last && key > best) best = key;
      }
      last = block_reduce<Max, 4>(best, lds);
      if (threadIdx.x == 0) {
        const int32_t c = last ? class_of(last) : -1;
        if (a.values) ((T *)a.values)[row * a.k + i] = last ? x[c] : minus_infinity<T>();
        if (a.ids) a.ids[row * a.k + i] = c;
      }
    }
  }
}

int launch_top_k(const TopKArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    return launch(top_k_kernel<decltype(t)>, grid_of(a.n_rows), 256, 0, a, stream);
  });
}

}  // namespace bridger
