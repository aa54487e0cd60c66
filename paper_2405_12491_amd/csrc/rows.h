// rows.h -- what the kernels of the row operators share: element types, row loads and stores, and
// reductions over the lanes of a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "operators.h"

namespace bridger {

template <int32_t DTYPE>
struct ElementOf;
template <>
struct ElementOf<BRIDGER_F32> {
  using type = float;
};
template <>
struct ElementOf<BRIDGER_BF16> {
  using type = __bf16;
};
template <>
struct ElementOf<BRIDGER_F16> {
  using type = _Float16;
};

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(__bf16 x) { return (float)x; }
__device__ inline float to_float(_Float16 x) { return (float)x; }

// Rounds to nearest even (bfloat16: v_cvt_pk_bf16_f32).
template <typename T>
__device__ inline T from_float(float x) {
  return (T)x;
}

struct Sum {
  template <typename V>
  __device__ static V of(V a, V b) {
    return a + b;
  }
};
struct Max {  // the other operand where one is NaN
  __device__ static float of(float a, float b) { return fmaxf(a, b); }
  __device__ static uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; }
  __device__ static uint64_t of(uint64_t a, uint64_t b) { return a > b ? a : b; }
};

template <typename Op, typename V>
__device__ inline V wave_reduce(V v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = Op::of(v, __shfl_xor(v, d));
  return v;
}

// Over a workgroup of WAVES waves; every thread gets the result.  `lds` holds WAVES values and may
// be reused after the next barrier; all threads call it.
template <typename Op, int WAVES, typename V>
__device__ inline V block_reduce(V v, V *lds) {
  v = wave_reduce<Op>(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v = Op::of(v, lds[w]);
  return v;
}

// Calls f with the element type of dtype.
template <typename F>
int with_type(int32_t dtype, F f) {
  if (dtype == BRIDGER_F32) return f(float());
  if (dtype == BRIDGER_BF16) return f(__bf16());
  return f(_Float16());
}

// Launches k(args); returns its own error, never an earlier one.
template <typename Args>
int launch(void (*k)(Args), int64_t blocks, int threads, int lds_bytes, Args args, void *stream) {
  void *p[] = {&args};
  return (int)hipLaunchKernel((const void *)k, dim3((uint32_t)blocks), dim3((uint32_t)threads), p,
                              (size_t)lds_bytes, (hipStream_t)stream);
}

// Workgroups of a launch that walks `n` items with a stride of the grid: a dispatch counts its
// work-items in 32 bits.
constexpr int64_t kMaxBlocks = int64_t(1) << 20;
inline int64_t grid_of(int64_t n) { return n < kMaxBlocks ? n : kMaxBlocks; }

}  // namespace bridger
