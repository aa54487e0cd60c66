// rows.h -- what the kernels of the row operators share: element types, row loads and stores, and
// reductions over the lanes that hold a row.
//
// A row is held by G lanes (a power of two up to a wave, or a workgroup of whole waves), each with
// C loads of 16 bytes: load c of lane l holds the V elements from (c G + l) V, V = 16 / element
// size.  Rows need no alignment beyond the element's: the 16-byte loads and stores may lie at any
// element (the hardware splits them where they cross a line); only the last, partial one goes
// element by element.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "operators.h"

namespace bridger {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
constexpr int kPerLoad = 16 / (int)sizeof(T);

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(__bf16 x) { return (float)x; }
__device__ inline float to_float(_Float16 x) { return (float)x; }

// Rounds to nearest even (bfloat16: v_cvt_pk_bf16_f32).
template <typename T>
__device__ inline T from_float(float x) {
  return (T)x;
}

// Element i of 16 loaded bytes.
template <typename T>
__device__ inline float element(const u32x4 &raw, int i) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(raw[i]);
  } else {
    const uint32_t w = raw[i >> 1];
    if constexpr (__is_same(T, __bf16)) {
      return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    } else {
      return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w));
    }
  }
}

// Rows of at least 16 bytes (shorter ones: tiny).  The 16 bytes of elements from j on: the last,
// partial ones come from the 16 bytes that end the row, moved down, so that a lane's loads need no
// branch; `fill` (two elements' bits, or one's of 4 bytes) stands past the end.
template <typename T>
struct RowLoad {
  u32x4 raw;

  // a row below 16 bytes: j = 0 holds all of it
  __device__ void tiny(const T *row, int j, int n, T fill) {
    T e[kPerLoad<T>];
#pragma unroll
    for (int i = 0; i < kPerLoad<T>; ++i) e[i] = j + i < n ? row[j + i] : fill;
    __builtin_memcpy(&raw, e, 16);
  }
  // issues the load; take() completes it
  __device__ void issue(const T *row, int j, int n) {
    __builtin_memcpy(&raw, row + (j < n - kPerLoad<T> ? j : n - kPerLoad<T>), 16);
  }
  __device__ void take(int j, int n, uint32_t fill) {
    const int d = j - n + kPerLoad<T>;  // elements to move down, all of them from kPerLoad on
    if (d > 0) {
      const int words = sizeof(T) == 4 ? d : d >> 1;
      if (words >= 4) raw = u32x4{fill, fill, fill, fill};
      if (words & 2) raw = u32x4{raw[2], raw[3], fill, fill};
      if (words & 1) raw = u32x4{raw[1], raw[2], raw[3], fill};
      if (sizeof(T) == 2 && (d & 1))
        raw = u32x4{raw[0] >> 16 | raw[1] << 16, raw[1] >> 16 | raw[2] << 16,
                    raw[2] >> 16 | raw[3] << 16, raw[3] >> 16 | fill << 16};
    }
  }
};

// Two elements' bits of x (one's, of 4 bytes).
template <typename T>
__device__ inline uint32_t fill_of(T x) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(uint32_t, x);
  } else {
    return __builtin_bit_cast(uint16_t, x) * 0x10001u;
  }
}

// Hides where v comes from, so that what was computed from it is computed again rather than held
// in registers across a reduction.
__device__ inline void forget(u32x4 &v) {
  uint32_t a = v[0], b = v[1], c = v[2], d = v[3];
  asm volatile("" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
  v = u32x4{a, b, c, d};
}

// The first `left` of N elements of type E, packed in `w`, to p (N E's in whole words).
template <typename E, int N>
__device__ inline void store_packed(E *p, int left, uint32_t (&w)[N * sizeof(E) / 4]) {
  constexpr int words = N * sizeof(E) / 4;
  if (left >= N) {
    __builtin_memcpy(p, w, N * sizeof(E));
    return;
  }
  // falling powers of two: what is stored leaves the words
  if (words == 4 && (left * (int)sizeof(E) & 8)) {
    __builtin_memcpy(p, w, 8);
    p += 8 / sizeof(E);
    w[0] = w[words - 2], w[1] = w[words - 1];
  }
  if (words >= 2 && (left * (int)sizeof(E) & 4)) {
    __builtin_memcpy(p, w, 4);
    p += 4 / sizeof(E);
    w[0] = w[1 % words];
  }
  if (sizeof(E) <= 2 && (left * (int)sizeof(E) & 2)) {
    __builtin_memcpy(p, w, 2);
    p += 2 / sizeof(E);
    w[0] >>= 16;
  }
  if (sizeof(E) == 1 && (left & 1)) __builtin_memcpy(p, w, 1);
}

// The first `left` of kPerLoad floats, rounded, to p.
template <typename T>
__device__ inline void store16(T *p, int left, const float (&v)[kPerLoad<T>]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = __float_as_uint(v[i]);
    } else {  // two at a time: one instruction
      typedef T pair __attribute__((ext_vector_type(2)));
      typedef float floats __attribute__((ext_vector_type(2)));
      w[i] = __builtin_bit_cast(
          uint32_t, __builtin_convertvector((floats{v[2 * i], v[2 * i + 1]}), pair));
    }
  }
  store_packed<T, kPerLoad<T>>(p, left, w);
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
  __device__ static int of(int a, int b) { return a > b ? a : b; }
};

// The value of another lane: 1, 2: the lane's number with that bit flipped; 4, 8: a lane of the
// other half of the group of 8, 16 (mirrored; after the lower steps all lanes of a half agree).
template <int STEP>
__device__ inline uint32_t dpp_word(uint32_t v) {
  constexpr int ctrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, ctrl, 0xF, 0xF, true);
}
template <int STEP, typename V>
__device__ inline V dpp(V v) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, dpp_word<STEP>(__builtin_bit_cast(uint32_t, v)));
  } else {
    uint2 w = __builtin_bit_cast(uint2, v);
    w.x = dpp_word<STEP>(w.x);
    w.y = dpp_word<STEP>(w.y);
    return __builtin_bit_cast(V, w);
  }
}
// v of the lanes 16 (32) apart, for both: op(first, second) is the same in all of them.
template <int STEP, typename Op>
__device__ inline float swap_reduce(float v) {
  const uint32_t w = __float_as_uint(v);
  const auto p = STEP == 16 ? __builtin_amdgcn_permlane16_swap(w, w, false, false)
                            : __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return Op::of(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
template <int STEP, typename Op, typename I>
__device__ inline I swap_reduce_int(I v) {
  const auto p = STEP == 16
                     ? __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false)
                     : __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return Op::of((I)p[0], (I)p[1]);
}
template <int STEP, typename Op>
__device__ inline uint32_t swap_reduce(uint32_t v) {
  return swap_reduce_int<STEP, Op>(v);
}
template <int STEP, typename Op>
__device__ inline int swap_reduce(int v) {
  return swap_reduce_int<STEP, Op>(v);
}
template <int STEP, typename Op>
__device__ inline double swap_reduce(double v) {
  const uint2 w = __builtin_bit_cast(uint2, v);
  const auto x = STEP == 16 ? __builtin_amdgcn_permlane16_swap(w.x, w.x, false, false)
                            : __builtin_amdgcn_permlane32_swap(w.x, w.x, false, false);
  const auto y = STEP == 16 ? __builtin_amdgcn_permlane16_swap(w.y, w.y, false, false)
                            : __builtin_amdgcn_permlane32_swap(w.y, w.y, false, false);
  return Op::of(__builtin_bit_cast(double, make_uint2(x[0], y[0])),
                __builtin_bit_cast(double, make_uint2(x[1], y[1])));
}

// Over aligned groups of min(G, 64) lanes of a wave; every lane gets the result, the same bits.
template <typename Op, int G, typename V>
__device__ inline V lanes_reduce(V v) {
  if constexpr (G > 1) v = Op::of(v, dpp<1>(v));
  if constexpr (G > 2) v = Op::of(v, dpp<2>(v));
  if constexpr (G > 4) v = Op::of(v, dpp<4>(v));
  if constexpr (G > 8) v = Op::of(v, dpp<8>(v));
  if constexpr (G > 16) v = swap_reduce<16, Op>(v);
  if constexpr (G > 32) v = swap_reduce<32, Op>(v);
  return v;
}

// Over the G lanes of a row.  Beyond a wave: `lds` holds G / 64 values that nothing else uses
// until the next barrier, and the whole workgroup calls it.
template <typename Op, int G, typename V>
__device__ inline V row_reduce(V v, V *lds) {
  v = lanes_reduce<Op, G>(v);
  if constexpr (G > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lanes_reduce<Op, G / 64>(lds[threadIdx.x & (G / 64 - 1)]);
  }
  return v;
}

// Threads of a workgroup for rows of G lanes, and the rows it holds.
template <int G>
constexpr int kRowThreads = G > 256 ? G : 256;
template <int G>
constexpr int kRowsAWorkgroup = kRowThreads<G> / G;

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

// The row of a thread, where rows of G lanes start at `first`.
template <int G>
__device__ inline int64_t row_of(int64_t first) {
  return first + (int64_t)blockIdx.x * kRowsAWorkgroup<G> + threadIdx.x / G;
}

// Launches k over rows [0, args.n_rows), `rows` of them a workgroup.  A dispatch counts its
// work-items in 32 bits: more rows go out as several launches.  (A loop over rows in the kernel
// instead keeps every address and mask of a row's loads alive across it: 100 more registers.)
template <typename Args>
int launch_over(void (*k)(Args), int threads, int rows, Args args, void *stream) {
  const int64_t step = (int64_t)rows << 20;
  for (args.first = 0; args.first < args.n_rows; args.first += step) {
    const int64_t n = args.n_rows - args.first < step ? args.n_rows - args.first : step;
    const int err = launch(k, (n + rows - 1) / rows, threads, 0, args, stream);
    if (err) return err;
  }
  return 0;
}
// Rows of `lanes` lanes, as row_of finds them.
template <typename Args>
int launch_rows(void (*k)(Args), int lanes, const Args &args, void *stream) {
  const int threads = lanes > 256 ? lanes : 256;
  return launch_over(k, threads, threads / lanes, args, stream);
}
// A workgroup a row.
template <typename Args>
int launch_each_row(void (*k)(Args), int threads, const Args &args, void *stream) {
  return launch_over(k, threads, 1, args, stream);
}

}  // namespace bridger
