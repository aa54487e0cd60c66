// layer_norm.hip -- gfx950 kernels of bridger_layer_norm and bridger_layer_norm_backward.
#include "rows.h"

namespace bridger {

// The mean in two floats: what `high` leaves of it goes to `low`, since a row far from zero needs
// more of its mean than a float holds.
struct Moments {
  float high, low, inverse;  // 1 / sqrt(variance + eps)
};
__device__ inline bool moderate(float v) { return v > 0x1p-60f && v < 0x1p60f; }

__device__ inline Moments moments_of(double mean, double inverse) {
  const float high = (float)mean;
  return {high, (float)(mean - (double)high), (float)inverse};
}
__device__ inline void store_moments(float *stats, int64_t row, const Moments &m) {
  stats[3 * row] = m.high;
  stats[3 * row + 1] = m.low;
  stats[3 * row + 2] = m.inverse;
}

// Loads c of a lane's C: issue all, then take all.  G = 1: rows below 16 bytes.
template <typename T, int G, int C>
struct RowLoads {
  RowLoad<T> l[C];
  __device__ void issue(const T *row, int lane, int n) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (G == 1) {
        l[c].tiny(row, 0, n, (T)0.0f);
      } else {
        l[c].issue(row, (c * G + lane) * kPerLoad<T>, n);
      }
    }
  }
  // Past the row's end stand zeros, or where `repeat` is set its last element (zeros with G = 1).
  __device__ void take(int lane, int n, bool repeat = false) {
    if constexpr (G > 1) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t last = sizeof(T) == 4 ? l[c].raw[3] : (l[c].raw[3] >> 16) * 0x10001u;
        l[c].take((c * G + lane) * kPerLoad<T>, n, repeat ? last : 0);
      }
    }
  }
  __device__ float at(int c, int i) const { return element<T>(l[c].raw, i); }
};

// G lanes a row, C loads a lane; the row stays in registers from its one read to the store.  Sums
// in float: the first gives a mean m near the true one, the second those of t - m and its square,
// from which the mean's rest and the variance follow without cancellation.  Where a sum leaves
// float's middle range (rows of huge or tiny elements, broken ones), or m is off by more than a quarter
// of the deviation (elements 2^19 deviations and more from zero), both are taken in double.
// Bound by memory: 8192 x 4096 bfloat16 with a residual and its total 45 to 48 us (5.6 to 5.9 TB/s, part
// of it stays in the last cache), 1,000,000 x 28 float with the statistics 47 (5.1 TB/s).
template <typename T, int G, int C>
__global__ __launch_bounds__(kRowThreads<G>) void layer_norm_kernel(LayerNormArgs a) {
  constexpr int V = kPerLoad<T>, W = G > 64 ? G / 64 : 1;
  __shared__ float lds_sum[W], lds_rest[W], lds_square[W];
  __shared__ double lds_double[2][W];
  const int lane = threadIdx.x & (G - 1), n = a.n_features;
  const int64_t row = row_of<G>(a.first);
  if (row >= a.n_rows) return;
  const T *res = a.residual ? (const T *)a.residual + row * a.ldr : nullptr;
  RowLoads<T, G, C> x, r, w, b;
  x.issue((const T *)a.x + row * a.ldx, lane, n);
  if (res) r.issue(res, lane, n);
  if (a.weight) w.issue((const T *)a.weight, lane, n);
  if (a.bias) b.issue((const T *)a.bias, lane, n);
  x.take(lane, n);
  if (res) r.take(lane, n);
  float t[C][V], sum = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      t[c][i] = x.at(c, i);
      if (res) t[c][i] = to_float(from_float<T>(t[c][i] + r.at(c, i)));
      sum += t[c][i];
    }
  sum = row_reduce<Sum, G>(sum, lds_sum);
  const float m = sum / (float)n;
  float rest = 0.0f, square = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int left = n - (c * G + lane) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = i < left ? t[c][i] - m : 0.0f;
      rest += d;
      square += d * d;
    }
  }
  rest = row_reduce<Sum, G>(rest, lds_rest);
  square = row_reduce<Sum, G>(square, lds_square);
  const float low = rest / (float)n, spread = square / (float)n - low * low;
  const float variance = spread + a.eps;
  Moments k = {m, low, 1.0f / __builtin_sqrtf(variance)};
  // (where the first sum misses the mean by much of the deviation, too little of both is left)
  const bool fine = moderate(variance) && fabsf(m) < 0x1p100f && 16.0f * low * low <= spread;
  double mean = 0.0, inverse = 0.0;
  if (!fine) {  // of the whole row
    double s = 0.0, q = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) s += (double)t[c][i];
    mean = row_reduce<Sum, G>(s, lds_double[0]) / n;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int left = n - (c * G + lane) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const double d = i < left ? (double)t[c][i] - mean : 0.0;
        q += d * d;
      }
    }
    inverse = 1.0 / sqrt(row_reduce<Sum, G>(q, lds_double[1]) / n + (double)a.eps);
    k = moments_of(mean, inverse);
  }
  if (a.stats && lane == 0) store_moments(a.stats, row, k);
  if (a.weight) w.take(lane, n);
  if (a.bias) b.take(lane, n);
  T *total = a.total ? (T *)a.total + row * a.ldt : nullptr;
  T *out = (T *)a.out + row * a.ldo;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int j = (c * G + lane) * V;
    if (j >= n) return;
    // (every lane of the row has read x and the residual, on which the total may lie)
    if (total) store16<T>(total + j, n - j, t[c]);
    float y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      y[i] = fine ? (t[c][i] - k.high - k.low) * k.inverse
                  : (float)(((double)t[c][i] - mean) * inverse);
      if (a.weight) y[i] *= w.at(c, i);
      if (a.bias) y[i] += b.at(c, i);
    }
    store16<T>(out + j, n - j, y);
  }
}

// Rows that do not fit a workgroup's registers: read once for the sum, once for the squares and
// once for the norm, sums in double.  1000 x 40,000 bfloat16 60 to 65 us (2.6 TB/s; the second and third
// read are the caches' for the most part: 197 MB fetched).
constexpr int kLong = 1024;
template <typename T>
__global__ __launch_bounds__(kLong) void layer_norm_long_kernel(LayerNormArgs a) {
  constexpr int V = kPerLoad<T>, W = kLong / 64;
  __shared__ double lds_sum[W], lds_square[W];
  const int64_t row = a.first + blockIdx.x;
  const int n = a.n_features;
  const T *x = (const T *)a.x + row * a.ldx;
  const T *res = a.residual ? (const T *)a.residual + row * a.ldr : nullptr;
  const T *w = (const T *)a.weight, *b = (const T *)a.bias;
  T *total = a.total ? (T *)a.total + row * a.ldt : nullptr;
  T *out = (T *)a.out + row * a.ldo;
  auto sum_of = [&](float v, float r) { return to_float(from_float<T>(v + r)); };
  auto walk = [&](auto f) {
    for (int64_t j0 = 0; j0 < n; j0 += kLong * V) {
      const int64_t j = j0 + (int64_t)threadIdx.x * V;
      if (j >= n) break;
      RowLoad<T> xl, rl;
      xl.issue(x, (int)j, n);
      if (res) rl.issue(res, (int)j, n);
      xl.take((int)j, n, 0);
      if (res) rl.take((int)j, n, 0);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float t = element<T>(xl.raw, i);
        if (res) t = sum_of(t, element<T>(rl.raw, i));
        if (j + i < n) f(t);
      }
    }
  };
  double sum = 0.0, square = 0.0;
  walk([&](float t) { sum += (double)t; });
  const double mean = row_reduce<Sum, kLong>(sum, lds_sum) / n;
  walk([&](float t) {
    const double d = (double)t - mean;
    square += d * d;
  });
  const double inverse =
      1.0 / sqrt(row_reduce<Sum, kLong>(square, lds_square) / n + (double)a.eps);
  if (a.stats && threadIdx.x == 0) store_moments(a.stats, row, moments_of(mean, inverse));
  // The total may lie on x or the residual: each element is read by the lane that writes it.
  auto one = [&](int64_t j) {
    float t = to_float(x[j]);
    if (res) t = sum_of(t, to_float(res[j]));
    float y = (float)(((double)t - mean) * inverse);
    if (w) y *= to_float(w[j]);
    if (b) y += to_float(b[j]);
    if (total) total[j] = from_float<T>(t);
    out[j] = from_float<T>(y);
  };
  const int whole = n / V * V;
  for (int64_t j = (int64_t)threadIdx.x * V; j < whole; j += kLong * V) {
    RowLoad<T> xl, rl, wl, bl;
    xl.issue(x, (int)j, n);
    if (res) rl.issue(res, (int)j, n);
    if (w) wl.issue(w, (int)j, n);
    if (b) bl.issue(b, (int)j, n);
    float t[V], y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      t[i] = element<T>(xl.raw, i);
      if (res) t[i] = sum_of(t[i], element<T>(rl.raw, i));
      y[i] = (float)(((double)t[i] - mean) * inverse);
      if (w) y[i] *= element<T>(wl.raw, i);
      if (b) y[i] += element<T>(bl.raw, i);
    }
    if (total) store16<T>(total + j, V, t);
    store16<T>(out + j, V, y);
  }
  if (threadIdx.x < n - whole) one(whole + threadIdx.x);
}

int launch_layer_norm(const LayerNormArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t bytes = (int64_t)a.n_features * (int)sizeof(T);
    auto of = [&](auto k, int lanes) { return launch_rows(k, lanes, a, stream); };
    if (bytes < 16) return of(layer_norm_kernel<T, 1, 1>, 1);
    if (bytes <= 64) return of(layer_norm_kernel<T, 4, 1>, 4);
    if (bytes <= 128) return of(layer_norm_kernel<T, 8, 1>, 8);
    if (bytes <= 256) return of(layer_norm_kernel<T, 16, 1>, 16);
    if (bytes <= 512) return of(layer_norm_kernel<T, 16, 2>, 16);
    if (bytes <= 1024) return of(layer_norm_kernel<T, 64, 1>, 64);
    if (bytes <= 2048) return of(layer_norm_kernel<T, 64, 2>, 64);
    if (bytes <= 4096) return of(layer_norm_kernel<T, 64, 4>, 64);
    if (bytes <= 8192) return of(layer_norm_kernel<T, 256, 2>, 256);
    if (bytes <= 16384) return of(layer_norm_kernel<T, 256, 4>, 256);
    if (bytes <= 32768) return of(layer_norm_kernel<T, 512, 4>, 512);
    if (bytes <= 65536) return of(layer_norm_kernel<T, 1024, 4>, 1024);
    return launch_each_row(layer_norm_long_kernel<T>, kLong, a, stream);
  });
}

// ============================================================================== BACKWARD
// With h = (t - mean) / std and s = grad * weight, per row
//     dx = (s - mean(s) - h mean(s h)) / std + grad_total,
// and per column the sums of grad * h and of grad over the rows.  A workgroup takes every so many
// rows; its lanes keep the sums of their columns in registers, and a second kernel adds the
// workgroups' sums in their order: one read of the rows serves dx and both sums, and no atomics decide
// their order.  Bound by memory: 8192 x 4096 bfloat16 with grad_total 51 us and the sums' 4.7 (5.2 TB/s),
// 1,000,000 x 28 float 64 and 7.4 (5.4 TB/s).
template <typename T, int G, int C>
__global__ __launch_bounds__(kRowThreads<G>) void layer_norm_backward_kernel(LayerNormGradArgs a) {
  constexpr int V = kPerLoad<T>, W = G > 64 ? G / 64 : 1, slots = kRowsAWorkgroup<G>;
  __shared__ float lds[2][2][W];
  __shared__ float join[slots > 1 ? kRowThreads<G> * V : 1];
  const int lane = threadIdx.x & (G - 1), n = a.n_features;
  RowLoads<T, G, C> w;
  if (a.weight) {
    w.issue((const T *)a.weight, lane, n);
    w.take(lane, n);
  }
  float dw[C][V], db[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.0f;
  int turn = 0;
  const int64_t step = (int64_t)gridDim.x * slots;
  for (int64_t row = (int64_t)blockIdx.x * slots + threadIdx.x / G; row < a.n_rows; row += step) {
    RowLoads<T, G, C> x, g, s;
    x.issue((const T *)a.x + row * a.ldx, lane, n);
    g.issue((const T *)a.grad + row * a.ldg, lane, n);
    if (a.grad_total) s.issue((const T *)a.grad_total + row * a.lds, lane, n);
    const float *k = a.stats + 3 * row;
    const float high = k[0], low = k[1], inverse = k[2];
    x.take(lane, n, true);  // (a zero's h may be infinite)
    g.take(lane, n);
    float sum = 0.0f, along = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float h = G > 1 || i < n ? (x.at(c, i) - high - low) * inverse : 0.0f;
        const float v = a.weight ? g.at(c, i) * w.at(c, i) : g.at(c, i);
        sum += v;
        along += v * h;
        dw[c][i] += g.at(c, i) * h;
        db[c][i] += g.at(c, i);
      }
    // (the other turn's values are read before the next row's barrier)
    if constexpr (G > 64) {
      sum = lanes_reduce<Sum, 64>(sum);
      along = lanes_reduce<Sum, 64>(along);
      if ((threadIdx.x & 63) == 0) {
        lds[turn][0][threadIdx.x >> 6] = sum;
        lds[turn][1][threadIdx.x >> 6] = along;
      }
      __syncthreads();
      sum = lanes_reduce<Sum, W>(lds[turn][0][threadIdx.x & (W - 1)]);
      along = lanes_reduce<Sum, W>(lds[turn][1][threadIdx.x & (W - 1)]);
      turn ^= 1;
    } else {
      sum = lanes_reduce<Sum, G>(sum);
      along = lanes_reduce<Sum, G>(along);
    }
    sum /= (float)n;
    along /= (float)n;
    if (a.grad_total) s.take(lane, n);
    if (!a.dx) continue;
    T *dx = (T *)a.dx + row * a.ldd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int j = (c * G + lane) * V;
      if (j < n) {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float h = (x.at(c, i) - high - low) * inverse;
          v[i] = a.weight ? g.at(c, i) * w.at(c, i) : g.at(c, i);
          v[i] = (v[i] - sum - h * along) * inverse;
          if (a.grad_total) v[i] += s.at(c, i);
        }
        store16<T>(dx + j, n - j, v);
      }
    }
  }
  if (!a.partial) return;
  float *to = a.partial + (int64_t)blockIdx.x * 2 * n;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = k ? db[c][i] : dw[c][i];
      if constexpr (slots > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) join[i * kRowThreads<G> + threadIdx.x] = v[i];
        __syncthreads();
        if (threadIdx.x < G)
          for (int q = 1; q < slots; ++q)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += join[i * kRowThreads<G> + threadIdx.x + q * G];
      }
      const int j = (c * G + lane) * V;
      if (threadIdx.x < G || slots == 1)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (j + i < n) to[(int64_t)k * n + j + i] = v[i];
    }
}

// Long rows: dx from two walks, a workgroup a row.  1000 x 40,000 bfloat16 58 us, their columns' sums
// 49, what joins those 8.6.
template <typename T>
__global__ __launch_bounds__(kLong) void layer_norm_backward_long_kernel(LayerNormGradArgs a) {
  constexpr int V = kPerLoad<T>, W = kLong / 64;
  __shared__ double lds_sum[W], lds_along[W];
  const int64_t row = a.first + blockIdx.x;
  const int n = a.n_features;
  const T *x = (const T *)a.x + row * a.ldx, *grad = (const T *)a.grad + row * a.ldg;
  const T *w = (const T *)a.weight;
  const T *extra = a.grad_total ? (const T *)a.grad_total + row * a.lds : nullptr;
  T *dx = (T *)a.dx + row * a.ldd;
  const float high = a.stats[3 * row], low = a.stats[3 * row + 1], inverse = a.stats[3 * row + 2];
  auto walk = [&](auto f) {
    for (int64_t j = (int64_t)threadIdx.x * V; j < n; j += kLong * V) {
      RowLoad<T> xl, gl, wl, el;
      xl.issue(x, (int)j, n);
      gl.issue(grad, (int)j, n);
      if (w) wl.issue(w, (int)j, n);
      if (extra) el.issue(extra, (int)j, n);
      xl.take((int)j, n, 0);
      gl.take((int)j, n, 0);
      if (w) wl.take((int)j, n, 0);
      if (extra) el.take((int)j, n, 0);
      float h[V], v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[i] = j + i < n ? (element<T>(xl.raw, i) - high - low) * inverse : 0.0f;
        v[i] = element<T>(gl.raw, i);
        if (w) v[i] *= element<T>(wl.raw, i);
      }
      f(j, h, v, el.raw);
    }
  };
  double sum = 0.0, along = 0.0;
  walk([&](int64_t, const float(&h)[V], const float(&v)[V], const u32x4 &) {
    float s = 0.0f, q = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) s += v[i], q += v[i] * h[i];
    sum += (double)s;
    along += (double)q;
  });
  const float mean = (float)(row_reduce<Sum, kLong>(sum, lds_sum) / n);
  const float slope = (float)(row_reduce<Sum, kLong>(along, lds_along) / n);
  walk([&](int64_t j, const float(&h)[V], const float(&v)[V], const u32x4 &e) {
    float d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      d[i] = (v[i] - mean - h[i] * slope) * inverse;
      if (extra) d[i] += element<T>(e, i);
    }
    store16<T>(dx + j, (int)(n - j < V ? n - j : V), d);
  });
}
// Their columns' sums: a lane has V columns, a workgroup every so many rows.
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_columns_kernel(LayerNormGradArgs a) {
  constexpr int V = kPerLoad<T>, ahead = 4;
  const int tile = (int)(blockIdx.x % (uint32_t)a.tiles), part = (int)(blockIdx.x / (uint32_t)a.tiles);
  const int n = a.n_features;
  const int64_t wanted = ((int64_t)tile * 256 + threadIdx.x) * V;
  if (wanted >= n) return;
  const int j = (int)(wanted < n - V ? wanted : n - V);  // (two lanes may write the same sums)
  float dw[V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.0f;
  for (int64_t row0 = part; row0 < a.n_rows; row0 += (int64_t)ahead * a.parts) {
    u32x4 x[ahead], g[ahead];
    float k[ahead][3];
#pragma unroll
    for (int u = 0; u < ahead; ++u) {
      const int64_t row = row0 + (int64_t)u * a.parts, at = row < a.n_rows ? row : row0;
      __builtin_memcpy(&x[u], (const T *)a.x + at * a.ldx + j, 16);
      __builtin_memcpy(&g[u], (const T *)a.grad + at * a.ldg + j, 16);
#pragma unroll
      for (int q = 0; q < 3; ++q) k[u][q] = a.stats[3 * at + q];
    }
#pragma unroll
    for (int u = 0; u < ahead; ++u) {
      if (row0 + (int64_t)u * a.parts >= a.n_rows) break;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float v = element<T>(g[u], i);
        dw[i] += v * ((element<T>(x[u], i) - k[u][0] - k[u][1]) * k[u][2]);
        db[i] += v;
      }
    }
  }
  float *to = a.partial + (int64_t)part * 2 * n;
#pragma unroll
  for (int i = 0; i < V; ++i) to[j + i] = dw[i], to[(int64_t)n + j + i] = db[i];
}

// The sums of the workgroups' sums: 16 lanes a column, each with every 16th of them and 8 loads on
// their way, in double.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(LayerNormGradArgs a) {
  constexpr int columns = 64, lanes = 16, ahead = 8;
  __shared__ double join[lanes][columns];
  const int64_t j = (a.first + blockIdx.x) * columns + (threadIdx.x & 63);
  const int part = threadIdx.x >> 6, n = a.n_features;
  double sum = 0.0;
  if (j < 2 * (int64_t)n)
    for (int p0 = part; p0 < a.parts; p0 += ahead * lanes) {
      float v[ahead];
#pragma unroll
      for (int u = 0; u < ahead; ++u) {
        const int p = p0 + u * lanes;
        v[u] = a.partial[(int64_t)(p < a.parts ? p : p0) * 2 * n + j];
      }
#pragma unroll
      for (int u = 0; u < ahead; ++u) sum += p0 + u * lanes < a.parts ? (double)v[u] : 0.0;
    }
  join[part][threadIdx.x & 63] = sum;
  __syncthreads();
  if (part || j >= 2 * (int64_t)n) return;
#pragma unroll
  for (int p = 1; p < lanes; ++p) sum += join[p][threadIdx.x];
  T *to = (T *)(j < n ? a.dweight : a.dbias);
  if (to) to[j < n ? j : j - n] = from_float<T>((float)sum);
}

// Workgroups of the first kernel, whose sums the workspace holds.
static int parts_of(int64_t n_rows, int32_t n_features, int size) {
  const int64_t bytes = (int64_t)n_features * size;
  if (bytes > 65536) {
    const int64_t tile = 256 * (16 / size), tiles = (n_features + tile - 1) / tile;
    const int64_t parts = (2048 + tiles - 1) / tiles;
    return (int)(n_rows < 4 * parts ? (n_rows + 3) / 4 : parts);
  }
  const int64_t most = bytes > 4096 ? 512 : 1024;
  return (int)(n_rows < most ? n_rows : most);
}
int64_t layer_norm_backward_bytes(int64_t n_rows, int32_t n_features, int size) {
  return (int64_t)parts_of(n_rows, n_features, size) * 2 * n_features * 4;
}

int launch_layer_norm_backward(const LayerNormGradArgs &args, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    LayerNormGradArgs a = args;
    const int64_t bytes = (int64_t)a.n_features * (int)sizeof(T);
    a.parts = parts_of(a.n_rows, a.n_features, (int)sizeof(T));
    int err = 0;
    if (bytes > 65536) {
      constexpr int tile = 256 * kPerLoad<T>;
      a.tiles = (int)(((int64_t)a.n_features + tile - 1) / tile);
      if (a.partial && a.parts)
        err = launch(layer_norm_columns_kernel<T>, (int64_t)a.parts * a.tiles, 256, 0, a, stream);
      if (!err && a.dx)
        err = launch_each_row(layer_norm_backward_long_kernel<T>, kLong, a, stream);
    } else if (a.n_rows) {
      auto of = [&](auto k, int lanes) {
        const int threads = lanes > 256 ? lanes : 256;
        const int slots = threads / lanes;
        const int64_t blocks = (a.n_rows + slots - 1) / slots;
        if (blocks < a.parts) a.parts = (int)blocks;
        return launch(k, a.parts, threads, 0, a, stream);
      };
      err = bytes < 16       ? of(layer_norm_backward_kernel<T, 1, 1>, 1)
            : bytes <= 64    ? of(layer_norm_backward_kernel<T, 4, 1>, 4)
            : bytes <= 128   ? of(layer_norm_backward_kernel<T, 8, 1>, 8)
            : bytes <= 256   ? of(layer_norm_backward_kernel<T, 16, 1>, 16)
            : bytes <= 1024  ? of(layer_norm_backward_kernel<T, 64, 1>, 64)
            : bytes <= 2048  ? of(layer_norm_backward_kernel<T, 64, 2>, 64)
            : bytes <= 4096  ? of(layer_norm_backward_kernel<T, 256, 1>, 256)
            : bytes <= 8192  ? of(layer_norm_backward_kernel<T, 256, 2>, 256)
            : bytes <= 16384 ? of(layer_norm_backward_kernel<T, 512, 2>, 512)
            : bytes <= 32768 ? of(layer_norm_backward_kernel<T, 1024, 2>, 1024)
                             : of(layer_norm_backward_kernel<T, 1024, 4>, 1024);
    }
    if (err || (!a.dweight && !a.dbias)) return err;
    return launch_blocks(layer_norm_join_kernel<T>, (2 * (int64_t)a.n_features + 63) / 64, 1024, a,
                         stream);
  });
}

}  // namespace bridger
