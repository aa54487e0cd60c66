// rmsnorm_q8.hip -- gfx950 kernels of bridger_rmsnorm_q8.
#include "rows.h"

namespace bridger {

constexpr int kNormThreads = 256;

// One workgroup a row, three walks over it: the sums and their squares (in double: a float square
// may overflow), the largest |y|, then the 8-bit values.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_q8_kernel(RmsnormArgs a) {
  constexpr int W = kNormThreads / 64;
  __shared__ double lds_sum[W];
  __shared__ uint32_t lds_max[W];
  for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
    const T *x = (const T *)a.x + row * a.ldx;
    const T *r = a.residual ? (const T *)a.residual + row * a.ldr : nullptr;
    const T *w = (const T *)a.weight;
    auto sum_at = [&](int64_t j) {
      return r ? to_float(x[j]) + to_float(r[j]) : to_float(x[j]);
    };
    double v = 0.0;
    for (int64_t j = threadIdx.x; j < a.n_features; j += kNormThreads) {
      const float s = sum_at(j);
      v += (double)s * (double)s;
    }
    const double mean = block_reduce<Sum, W>(v, lds_sum) / a.n_features;
    const double per = mean + (double)a.eps == 0.0 ? 0.0 : 1.0 / sqrt(mean + (double)a.eps);
    auto y_at = [&](int64_t j) {
      return (float)((double)sum_at(j) * per * (w ? (double)to_float(w[j]) : 1.0));
    };
    // |y| as bits: NaN is above infinity, which is above every number
    uint32_t m = 0;
    for (int64_t j = threadIdx.x; j < a.n_features; j += kNormThreads) {
      const uint32_t b = __float_as_uint(y_at(j)) & 0x7FFFFFFFu;
      m = Max::of(m, b);
    }
    m = block_reduce<Max, W>(m, lds_max);
    const float most = __uint_as_float(m);
    const bool fine = m < 0x7F800000u;  // no NaN, no infinity
    // tiny values are raised first, so that 127 / most stays finite
    const float raise = most < 0x1p-60f ? 0x1p90f : 1.0f;
    const float steps = fine && m ? 127.0f / (most * raise) : 0.0f;
    T *total = a.total ? (T *)a.total + row * a.ldt : nullptr;
    for (int64_t j = threadIdx.x; j < a.n_features; j += kNormThreads) {
      a.q[row * a.ldq + j] = steps != 0.0f ? (int8_t)(int)__builtin_rintf(y_at(j) * raise * steps) : 0;
      if (total) total[j] = from_float<T>(sum_at(j));  // last: it may lie on x or the residual
    }
    if (threadIdx.x == 0) a.scale[row] = fine ? most / 127.0f : __builtin_nanf("");
  }
}

int launch_rmsnorm_q8(const RmsnormArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    return launch(rmsnorm_q8_kernel<decltype(t)>, grid_of(a.n_rows), kNormThreads, 0, a, stream);
  });
}

}  // namespace bridger
