// rmsnorm_q8.hip -- gfx950 kernels of bridger_rmsnorm_q8.
#include "rows.h"

namespace bridger {

// q and scale need the row's largest |s w| and its mean square; both come from one walk, since the
// norm's factor 1 / rms is common to the row: q = rint(s w 127 / max|s w|) and scale = max|s w| /
// (127 rms).  Squares are added in double (a float square may overflow, and the mean loses
// nothing). Where extreme inputs take s w out of float's middle range, y is formed in double
// instead, which takes another walk.
__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ inline bool middle(uint32_t most) {
  return most >= __float_as_uint(0x1p-60f) && most <= __float_as_uint(0x1p60f);
}
__device__ inline double inverse_rms(double squares, int n, float eps) {
  const double mean = squares / n + (double)eps;
  return mean == 0.0 ? 0.0 : 1.0 / sqrt(mean);
}
__device__ inline int8_t to_q8(float v, float steps) {
  return (int8_t)(int)__builtin_rintf(v * steps);
}

// A row of G lanes by walks over memory, V elements at a time (V = 1: of any width).
template <typename T, int G, int V>
__device__ inline void walk_row(const RmsnormArgs &a, int64_t row, int lane, double *lds_sum,
                                uint32_t *lds_max, uint32_t *lds_again) {
  const T *x = (const T *)a.x + row * a.ldx;
  const T *res = a.residual ? (const T *)a.residual + row * a.ldr : nullptr;
  const T *w = (const T *)a.weight;
  T *total = a.total ? (T *)a.total + row * a.ldt : nullptr;
  int8_t *q = a.q + row * a.ldq;
  // f(first element, sums, weights); zeros past the row's end
  auto walk = [&](auto f) {
    for (int64_t j = (int64_t)lane * V; j < a.n_features; j += G * V) {
      float s[V], wi[V];
      if constexpr (V == 1) {
        s[0] = to_float(x[j]);
        if (res) s[0] += to_float(res[j]);
        wi[0] = w ? to_float(w[j]) : 1.0f;
      } else {
        RowLoad<T> xl, rl, wl;
        const int n = a.n_features;
        xl.issue(x, (int)j, n);
        if (res) rl.issue(res, (int)j, n);
        if (w) wl.issue(w, (int)j, n);
        xl.take((int)j, n, 0);
        if (res) rl.take((int)j, n, 0);
        if (w) wl.take((int)j, n, 0);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          s[i] = element<T>(xl.raw, i);
          if (res) s[i] += element<T>(rl.raw, i);
          wi[i] = w ? element<T>(wl.raw, i) : 1.0f;
        }
      }
      f(j, s, wi);
    }
  };
  double squares = 0.0;
  uint32_t most = 0;
  walk([&](int64_t, const float(&s)[V], const float(&wi)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      squares += (double)s[i] * (double)s[i];
      most = Max::of(most, magnitude(s[i] * wi[i]));
    }
  });
  squares = row_reduce<Sum, G>(squares, lds_sum);
  most = row_reduce<Max, G>(most, lds_max);
  const double per = inverse_rms(squares, a.n_features, a.eps);
  const bool wide = !middle(most);
  auto y = [&](float s, float wi) { return (float)((double)s * per * (double)wi); };
  if (wide) {
    most = 0;
    walk([&](int64_t, const float(&s)[V], const float(&wi)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) most = Max::of(most, magnitude(y(s[i], wi[i])));
    });
    most = row_reduce<Max, G>(most, lds_again);
  }
  const double top = (double)__uint_as_float(most) * (wide ? 1.0 : per);
  const bool fine = top <= (double)__FLT_MAX__;  // false for NaN
  const float raise = most < __float_as_uint(0x1p-60f) ? 0x1p90f : 1.0f;  // 127 / top stays finite
  const float steps = fine && most ? 127.0f / (__uint_as_float(most) * raise) : 0.0f;
  // The last walk stores the sum too, which may lie on x or the residual: an element at a time,
  // lane by lane, since a load of 16 bytes at the row's end reads another lane's elements.
  for (int64_t j = lane; j < a.n_features; j += G) {
    const float s = res ? to_float(x[j]) + to_float(res[j]) : to_float(x[j]);
    const float wi = w ? to_float(w[j]) : 1.0f;
    const float v = wide ? y(s, wi) : s * wi;
    q[j] = steps == 0.0f ? (int8_t)0 : to_q8(v * raise, steps);
    if (total) total[j] = from_float<T>(s);
  }
  if (lane == 0) a.scale[row] = fine ? (float)(top / 127.0) : __builtin_nanf("");
}

// Rows below 16 bytes (G = 4, V = 1), and rows that do not fit a workgroup's registers.  The latter
// are read twice and stored an element at a time: 3000 x 20,000 float, 300 MB in 105 us, 780 MB
// with a residual in 207; 3000 x 40,000 bfloat16, 360 MB in 195, 840 MB in 315.
template <typename T, int G, int V>
__global__ __launch_bounds__(kRowThreads<G>) void rmsnorm_q8_walk_kernel(RmsnormArgs a) {
  constexpr int W = G > 64 ? G / 64 : 1;
  __shared__ double lds_sum[W];
  __shared__ uint32_t lds_max[W], lds_again[W];
  const int64_t row = row_of<G>(a.first);
  if (row < a.n_rows)
    walk_row<T, G, V>(a, row, threadIdx.x & (G - 1), lds_sum, lds_max, lds_again);
}

// G lanes a row, C loads a lane of x, residual and weight; the row stays in registers from the one
// read to the 8-bit store.  Bound by memory: 8192 x 8192 bfloat16 with a residual, 470 MB, in 78 to
// 86 us (5.5 to 6.0 TB/s; part of what is written stays in the last cache), 100,000 x 784 float 392
// MB in 71 to 84.  Rows of a few elements are bound by instructions: 1M x 28 float 144 MB in 38 us.
template <typename T, int G, int C>
__global__ __launch_bounds__(kRowThreads<G>) void rmsnorm_q8_kernel(RmsnormArgs a) {
  constexpr int V = kPerLoad<T>, W = G > 64 ? G / 64 : 1;
  __shared__ double lds_sum[W], lds_sum2[W];
  __shared__ uint32_t lds_max[W], lds_max2[W], lds_again[W];
  const int lane = threadIdx.x & (G - 1), n = a.n_features;
  const T *w = (const T *)a.weight;
  const int64_t row = row_of<G>(a.first);
  if (row >= a.n_rows) return;
  const T *x = (const T *)a.x + row * a.ldx;
  const T *res = a.residual ? (const T *)a.residual + row * a.ldr : nullptr;
  T *total = a.total ? (T *)a.total + row * a.ldt : nullptr;
  float s[C][V];
  RowLoad<T> xl[C], rl[C], wl[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int j = (c * G + lane) * V;
    xl[c].issue(x, j, n);
    if (res) rl[c].issue(res, j, n);
    if (w) wl[c].issue(w, j, n);
  }
  double squares = 0.0;
  uint32_t most = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int j = (c * G + lane) * V;
    xl[c].take(j, n, 0);
    if (res) rl[c].take(j, n, 0);
    if (w) wl[c].take(j, n, 0);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s[c][i] = element<T>(xl[c].raw, i);
      if (res) s[c][i] += element<T>(rl[c].raw, i);
      squares += (double)s[c][i] * (double)s[c][i];
      most = Max::of(most, magnitude(w ? s[c][i] * element<T>(wl[c].raw, i) : s[c][i]));
    }
  }
  squares = row_reduce<Sum, G>(squares, lds_sum);
  most = row_reduce<Max, G>(most, lds_max);
  // (A row of zeros needs nothing more.)  The row's lanes agree, so whole workgroups do where they
  // hold one row.
  if (!middle(most) && !(most == 0 && squares == 0.0)) {
    walk_row<T, G, 1>(a, row, lane, lds_sum2, lds_max2, lds_again);
    return;
  }
  // in float where the mean square lies in its middle: half the instructions of a short row were
  // those of the double root and quotient (1M x 28 float: 48 -> 38 us)
  const double mean = squares * a.per_feature + (double)a.eps;
  double top;
  if (mean > 0x1p-100 && mean < 0x1p100) {
    top = (double)(__uint_as_float(most) / __builtin_sqrtf((float)mean));
  } else {
    top = (double)__uint_as_float(most) * inverse_rms(squares, n, a.eps);
  }
  const bool fine = top <= (double)__FLT_MAX__;
  const float steps = fine && most ? 127.0f / __uint_as_float(most) : 0.0f;
  int8_t *q = a.q + row * a.ldq;
  if (lane == 0) a.scale[row] = fine ? (float)top * (1.0f / 127.0f) : __builtin_nanf("");
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int j = (c * G + lane) * V;
    if (j >= n) return;
    // after the reductions: every lane of the row has read x and the residual, on which the
    // total may lie (a row's last load also reads elements of the lane before it)
    if (total) store16<T>(total + j, n - j, s[c]);
    if (w) forget(wl[c].raw);
    int8_t b[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
      b[i] = to_q8(w ? s[c][i] * element<T>(wl[c].raw, i) : s[c][i], steps);
    uint32_t words[V / 4];
    __builtin_memcpy(words, b, V);
    store_packed<int8_t, V>(q + j, n - j, words);
  }
}

// Few lanes a row, so that a wave's reductions serve many rows, but no more than four loads of each
// array in a lane's registers.  With (without) a residual, us, lanes x loads: 1M x 10 float 4 x 1
// 22, 8 x 1 42; 500,000 x 100 16 x 2 118 (45), 32 x 1 112 (69), 64 x 1 166 (139); 100,000 x 784 64
// x 4 180 (70), 256 x 1 176 (126); 16,384 x 4096 bfloat16 256 x 2 83, 512 x 2 101; 4096 x 11,008
// 512 x 4 57 (36), 1024 x 2 72 (48); 4096 x 16,384 85 (39) against 92 (54).
int launch_rmsnorm_q8(const RmsnormArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t bytes = (int64_t)a.n_features * (int)sizeof(T);
    auto of = [&](auto k, int lanes) { return launch_rows(k, lanes, a, stream); };
    if (bytes < 16) return of(rmsnorm_q8_walk_kernel<T, 4, 1>, 4);
    if (bytes <= 64) return of(rmsnorm_q8_kernel<T, 4, 1>, 4);
    if (bytes <= 128) return of(rmsnorm_q8_kernel<T, 8, 1>, 8);
    if (bytes <= 256) return of(rmsnorm_q8_kernel<T, 16, 1>, 16);
    if (bytes <= 512) return of(rmsnorm_q8_kernel<T, 16, 2>, 16);
    if (bytes <= 1024) return of(rmsnorm_q8_kernel<T, 64, 1>, 64);
    if (bytes <= 2048) return of(rmsnorm_q8_kernel<T, 64, 2>, 64);
    if (bytes <= 4096) return of(rmsnorm_q8_kernel<T, 64, 4>, 64);
    if (bytes <= 8192) return of(rmsnorm_q8_kernel<T, 256, 2>, 256);
    if (bytes <= 16384) return of(rmsnorm_q8_kernel<T, 256, 4>, 256);
    if (bytes <= 32768) return of(rmsnorm_q8_kernel<T, 512, 4>, 512);
    if (bytes <= 65536) return of(rmsnorm_q8_kernel<T, 1024, 4>, 1024);
    return of(rmsnorm_q8_walk_kernel<T, 1024, kPerLoad<T>>, 1024);
  });
}

}  // namespace bridger
