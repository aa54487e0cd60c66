// distill.hip -- gfx950 kernels of bridger_distill and bridger_distill_backward.
#include "rows.h"

namespace bridger {

constexpr int kThreads = 256;

// A row's teacher: p = softmax(t / T) over the filled slots, thread i holding slot i.
struct Teacher {
  bool any;       // a filled slot above -infinity
  int32_t id;     // -1: not filled
  float p, logp;  // of this thread's slot (p = 0 where not filled)
};

template <typename U, int WAVES>
__device__ inline Teacher load_teacher(const DistillArgs &a, int64_t row, float *lds) {
  Teacher s = {false, -1, 0.0f, 0.0f};
  const int i = threadIdx.x;
  float t = -__builtin_inff();
  if (i < a.k) {
    const int32_t id = a.ids[row * a.k + i];
    if (id >= 0 && id < a.n_classes) {
      s.id = id;
      t = to_float(((const U *)a.teacher)[row * a.k + i]);
    }
  }
  s.any = __syncthreads_or(s.id >= 0 && t != -__builtin_inff());
  float most = block_reduce<Max, WAVES>(t, lds);
  if (most == -__builtin_inff()) most = 0.0f;  // nothing but NaN, or an empty row
  const float u = (t - most) / a.temperature;
  const float e = s.id >= 0 ? __expf(u) : 0.0f;
  const float mass = block_reduce<Sum, WAVES>(e, lds);
  s.p = e / mass;
  s.logp = u - __logf(mass);
  return s;
}

// One workgroup a row.  z - max(z) is formed before the division by T, so that neither overflows;
// exponents are at most 0.
template <typename T, typename U, bool BACKWARD>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  constexpr int W = kThreads / 64;
  __shared__ float lds[W];
  __shared__ int32_t slot_id[BRIDGER_MAX_TOP];
  __shared__ float slot_p[BRIDGER_MAX_TOP];
  const float inf = __builtin_inff();
  const float T_ = a.temperature;
  for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
    const T *z = (const T *)a.logits + row * a.ldl;
    T *grad = a.grad ? (T *)a.grad + row * a.ldg : nullptr;
    const Teacher s = load_teacher<U, W>(a, row, lds);
    const int i = threadIdx.x;
    const float z_id = s.id >= 0 ? to_float(z[s.id]) : 0.0f;
    float most, mass;
    if (BACKWARD) {
      most = a.stats[2 * row];
      mass = a.stats[2 * row + 1];
    } else {
      float v = -inf;
      for (int64_t j = i; j < a.n_classes; j += kThreads) v = fmaxf(v, to_float(z[j]));
      most = block_reduce<Max, W>(v, lds);
      if (most == -inf) most = 0.0f;
      v = 0.0f;
      for (int64_t j = i; j < a.n_classes; j += kThreads)
        v += __expf((to_float(z[j]) - most) / T_);
      mass = block_reduce<Sum, W>(v, lds);
      const float log_q = z_id == -inf ? -inf : (z_id - most) / T_ - __logf(mass);
      v = s.id >= 0 && s.p != 0.0f ? s.p * (s.logp - log_q) : 0.0f;
      v = block_reduce<Sum, W>(v, lds);
      if (i == 0) {
        if (a.loss) a.loss[row] = s.any ? T_ * T_ * v : 0.0f;
        if (a.stats) {
          a.stats[2 * row] = most;
          a.stats[2 * row + 1] = mass;
        }
      }
    }
    if (grad) {
      const float w = s.any ? T_ * (a.weight ? a.weight[row] : 1.0f) : 0.0f;
      const float per = mass == 0.0f ? 0.0f : 1.0f / mass;
      __syncthreads();
      if (i < a.k) {
        slot_id[i] = s.id;
        slot_p[i] = s.p;
      }
      __syncthreads();  // also: every slot's logit is read before the gradient may overwrite it
      for (int64_t j = i; j < a.n_classes; j += kThreads)
        grad[j] = from_float<T>(s.any ? w * (__expf((to_float(z[j]) - most) / T_) * per) : 0.0f);
      __syncthreads();
      if (s.any && s.id >= 0) {  // equal ids: every one of them writes the same value
        float p = 0.0f;
        for (int q = 0; q < a.k; ++q)
          if (slot_id[q] == s.id) p += slot_p[q];
        grad[s.id] = from_float<T>(w * (__expf((z_id - most) / T_) * per - p));
      }
    }
  }
}

int launch_distill(const DistillArgs &a, int32_t dtype, int32_t teacher_dtype, bool backward,
                   void *stream) {
  static_assert(kThreads >= BRIDGER_MAX_TOP, "a thread for each slot");
  return with_type(dtype, [&](auto t) {
    return with_type(teacher_dtype, [&](auto u) {
      using T = decltype(t);
      using U = decltype(u);
      return launch(backward ? distill_kernel<T, U, true> : distill_kernel<T, U, false>,
                    grid_of(a.n_rows), kThreads, 0, a, stream);
    });
  });
}

}  // namespace bridger
