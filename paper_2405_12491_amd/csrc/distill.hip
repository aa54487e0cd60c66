// distill.hip -- gfx950 kernels of bridger_distill and bridger_distill_backward.
#include "rows.h"

namespace bridger {

// With M = max z, e_j = exp((z_j - M) / T) and S = sum e_j:  q_j = e_j / S,
// loss = T^2 sum_i p_i (log p_i - (z_i - M) / T + log S),  grad_j = w T (q_j - p_j).
// z - M is formed before the division by T, so that neither overflows and exponents are at most 0;
// exp goes through exp2, 1 / T and log2(e) in one factor that is rounded once.  Every lane keeps
// the largest of its own logits and the sum relative to it; those pairs are joined across the row's
// lanes at once.  The gradient is first w T q everywhere; the few kept classes are then written
// again with their p taken off, by the row's first wave.
// Bound by memory from about 300 bytes a row on: 4096 x 32,000 bfloat16, loss and gradient from one
// read and one write of 262 MB, take 106 us (5.0 TB/s, a large copy's rate); 2048 x 50,257 float 92
// us for the loss and 138 for the gradient later.  Of shorter rows' time a row's slots and
// reductions are a part: 1M x 10 float, k = 4, 120 MB in 29 to 31 us (3.9 to 4.1 TB/s).
constexpr int kSlots = 4;  // a lane's share of the teacher's slots, lanes of one wave at most

template <int G>
constexpr int kSlotLanes = G < 64 ? G : 64;

struct Slots {
  int32_t id[kSlots];  // -1: not filled
  float z[kSlots], p[kSlots];
  float kl;  // this lane's sum of p log p
  bool any;  // some slot of the row is filled above -infinity
};

__device__ inline float teacher_at(const DistillArgs &a, int64_t at) {
  if (a.teacher_dtype == BRIDGER_F32) return ((const float *)a.teacher)[at];
  if (a.teacher_dtype == BRIDGER_BF16) return to_float(((const __bf16 *)a.teacher)[at]);
  return to_float(((const _Float16 *)a.teacher)[at]);
}

// p = softmax(t / T) over the row's filled slots; slot s L + l is lane l's.
template <typename T, int G>
__device__ inline Slots load_slots(const DistillArgs &a, int64_t row, const T *z, int lane) {
  constexpr int L = kSlotLanes<G>;
  const float inf = __builtin_inff();
  Slots s;
  float t[kSlots], most = -inf;
  int any = 0;
#pragma unroll
  for (int i = 0; i < kSlots; ++i) {
    s.id[i] = -1;
    s.z[i] = s.p[i] = 0.0f;
    t[i] = -inf;
  }
  // in this and the loops below: no work for the slots that no lane has
#pragma unroll
  for (int i = 0; i < kSlots; ++i) {
    if (i * L >= a.k) break;
    const int at = i * L + lane;
    if (at < a.k) {
      const int32_t id = a.ids[row * a.k + at];
      const float v = teacher_at(a, row * a.k + at);
      if (id >= 0 && id < a.n_classes) {
        s.id[i] = id;
        s.z[i] = to_float(z[id]);
        t[i] = v;
        any |= v != -inf;  // NaN is not
      }
    }
    most = fmaxf(most, t[i]);
  }
  s.any = lanes_reduce<Max, L>(any) != 0;
  most = lanes_reduce<Max, L>(most);
  if (most == -inf) most = 0.0f;  // an empty row, or nothing but NaN
  float mass = 0.0f;
#pragma unroll
  for (int i = 0; i < kSlots; ++i) {
    if (i * L >= a.k) break;
    t[i] = (t[i] - most) / a.temperature;
    s.p[i] = s.id[i] >= 0 ? __expf(t[i]) : 0.0f;
    mass += s.p[i];
  }
  mass = lanes_reduce<Sum, L>(mass);
  const float log_mass = __logf(mass);
  s.kl = 0.0f;
#pragma unroll
  for (int i = 0; i < kSlots; ++i) {
    if (i * L >= a.k) break;
    s.p[i] /= mass;
    if (s.id[i] >= 0 && s.p[i] != 0.0f) s.kl += s.p[i] * (t[i] - log_mass);
  }
  return s;
}

// How many pairs (slot of this wave's rows in groups below N, filled entry of the row's `ids`) hold
// one class.  A slot meets itself: no class is there twice where this is the number of filled
// slots.
template <int N>
__device__ inline int count_equal(const Slots &s, const int32_t *ids, int k) {
  int32_t id[N];
#pragma unroll
  for (int i = 0; i < N; ++i) id[i] = s.id[i] < 0 ? -2 : s.id[i];  // entries not filled are -1
  int equal = 0;
  for (int q = 0; q < k; q += 4) {
    const int4 other = *(const int4 *)(ids + q);
#pragma unroll
    for (int i = 0; i < N; ++i)
      equal += __popcll(__ballot(other.x == id[i])) + __popcll(__ballot(other.y == id[i])) +
               __popcll(__ballot(other.z == id[i])) + __popcll(__ballot(other.w == id[i]));
  }
  return equal;
}

// Of slots that hold one class, the first takes the sum of their p, in slot order, and the others
// are emptied.  `ids` and `ps`: the row's kSlots L slots, written and read by this wave.  All pairs
// are compared, and counted by the scalar unit; only rows that have such slots go on to find them.
template <int G>
__device__ inline void join_equal(const DistillArgs &a, Slots &s, int lane, int32_t *ids, float *ps) {
  constexpr int L = kSlotLanes<G>;
  int filled = 0;
#pragma unroll
  for (int i = 0; i < kSlots; ++i) {
    if (i * L >= a.k) break;
    ids[i * L + lane] = s.id[i];
    ps[i * L + lane] = s.p[i];
    filled += __popcll(__ballot(s.id[i] >= 0));
  }
  if constexpr (L < 4) {  // the last of four entries read at once
    if (lane == 0)
      for (int q = a.k; q < kSlots * L; ++q) ids[q] = -1;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int equal = a.k <= L ? count_equal<1>(s, ids, a.k)
                             : a.k <= 2 * L ? count_equal<2>(s, ids, a.k)
                                            : count_equal<kSlots>(s, ids, a.k);
  if (equal == filled) return;
#pragma unroll
  for (int i = 0; i < kSlots; ++i)
    if (s.id[i] >= 0) {
      float p = 0.0f;
      bool first = true;
      for (int q = 0; q < a.k; ++q)
        if (ids[q] == s.id[i]) {
          p += ps[q];
          first &= q >= i * L + lane;
        }
      s.p[i] = p;
      if (!first) s.id[i] = -1;
    }
}

// What a row's lanes share: the largest logit, the sum of the exponentials, and whether the row has
// a teacher.
struct RowStats {
  float most, mass;
  bool any;
};

// most and mass: a lane's; they are joined over the row.  The barrier between the waves of a row
// also makes `any`, which the first wave knows, known to all.
template <int G>
__device__ inline RowStats join_stats(float most, float mass, bool any, float factor, float2 *lds,
                                      int *lds_any) {
  const float inf = __builtin_inff();
  float all = lanes_reduce<Max, G>(most);
  float safe = all == -inf ? 0.0f : all;
  mass = lanes_reduce<Sum, G>(mass * __builtin_amdgcn_exp2f((most - safe) * factor));
  if constexpr (G > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[wave] = make_float2(all, mass);
    if (threadIdx.x == 0) *lds_any = any;
    __syncthreads();
    const float2 w = lds[threadIdx.x & (G / 64 - 1)];
    all = lanes_reduce<Max, G / 64>(w.x);
    safe = all == -inf ? 0.0f : all;
    mass = lanes_reduce<Sum, G / 64>(w.y * __builtin_amdgcn_exp2f((w.x - safe) * factor));
    any = *lds_any != 0;
  }
  return {safe, mass, any};
}

// The first wave's part after the row's sums: the loss, the stats.
template <int G>
__device__ inline void store_loss(const DistillArgs &a, int64_t row, const Slots &s,
                                  const RowStats &r, int lane) {
  const float inf = __builtin_inff();
  // T log q, then p (which may pass 1 by its rounding), and T where it makes the product larger last:
  // for logits of the type's lowest value nothing leaves float before the loss does
  const float log_mass = a.temperature * __logf(r.mass);
  const float low = fminf(a.temperature, 1.0f), high = fmaxf(a.temperature, 1.0f);
  float v = a.temperature * a.temperature * s.kl;
  const bool number = r.mass == r.mass;  // no class of a broken row has a log q, masked or not
#pragma unroll
  for (int i = 0; i < kSlots; ++i) {
    if (i * kSlotLanes<G> >= a.k) break;
    if (s.id[i] >= 0 && s.p[i] != 0.0f)
      v -= high *
           (s.p[i] * (low * (number && s.z[i] == -inf ? -inf : s.z[i] - r.most - log_mass)));
  }
  v = lanes_reduce<Sum, kSlotLanes<G>>(v);
  if (lane == 0) {
    if (a.loss) a.loss[row] = s.any ? v : 0.0f;
    if (a.stats) {
      a.stats[2 * row] = r.most;
      a.stats[2 * row + 1] = r.mass;
    }
  }
}

// Gradient of the kept classes, over what the whole row's lanes have written.
template <typename T>
__device__ inline void store_kept(T *grad, const Slots &s, const RowStats &r, float factor,
                                  float weight, float per) {
#pragma unroll
  for (int i = 0; i < kSlots; ++i)
    if (s.any && s.id[i] >= 0) {
      const float e = __builtin_amdgcn_exp2f((s.z[i] - r.most) * factor);
      grad[s.id[i]] = from_float<T>(weight * (e * per - s.p[i]));
    }
}

// G lanes a row, C loads a lane: the logits stay in registers between the sum and the gradient, so
// loss and gradient cost one read and one write of the row.
template <typename T, int G, int C, bool TINY, bool BACKWARD>
__global__ __launch_bounds__(kRowThreads<G>, C <= 4 ? 8 : 4) void distill_kernel(DistillArgs a) {
  constexpr int V = kPerLoad<T>, L = kSlotLanes<G>, W = G > 64 ? G / 64 : 1;
  __shared__ float2 lds[W];
  __shared__ int lds_any;
  __shared__ __attribute__((aligned(16))) int32_t slot_id[kRowsAWorkgroup<G> * L * kSlots];
  __shared__ float slot_p[kRowsAWorkgroup<G> * L * kSlots];
  const int lane = threadIdx.x & (G - 1), n = a.n_classes;
  const int64_t row = row_of<G>(a.first);
  if (row >= a.n_rows) return;
  const T *z = (const T *)a.logits + row * a.ldl;
  const float inf = __builtin_inff(), factor = a.factor;
  RowLoad<T> x[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int j = (c * G + lane) * V;
    if constexpr (TINY) {
      x[c].tiny(z, j, n, (T)-inf);
    } else {
      x[c].issue(z, j, n);
    }
  }
  const bool first_wave = G <= 64 || threadIdx.x < 64;
  const int slots_at = threadIdx.x / G * L * kSlots;
  Slots s;
  s.any = false;
  if (first_wave) {
    s = load_slots<T, G>(a, row, z, lane);
    join_equal<G>(a, s, lane, slot_id + slots_at, slot_p + slots_at);
    // the gradient may take the logits' place: they are here before any is stored
    asm volatile("" ::"v"(s.z[0]), "v"(s.z[1]), "v"(s.z[2]), "v"(s.z[3]));
  }
  float most = -inf, mass = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if constexpr (!TINY) x[c].take((c * G + lane) * V, n, fill_of((T)-inf));
    if constexpr (BACKWARD) forget(x[c].raw);  // here before any gradient is stored
    if constexpr (!BACKWARD) {
#pragma unroll
      for (int i = 0; i < V; ++i) most = fmaxf(most, element<T>(x[c].raw, i));
    }
  }
  RowStats r;
  if constexpr (BACKWARD) {
    if constexpr (G > 64) {
      if (threadIdx.x == 0) lds_any = s.any;
      __syncthreads();
      s.any = lds_any != 0;
    }
    r = {a.stats[2 * row], a.stats[2 * row + 1], s.any};
  } else {
    const float safe = most == -inf ? 0.0f : most;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      forget(x[c].raw);
#pragma unroll
      for (int i = 0; i < V; ++i)
        mass += __builtin_amdgcn_exp2f((element<T>(x[c].raw, i) - safe) * factor);
    }
    r = join_stats<G>(most, mass, s.any, factor, lds, &lds_any);
    s.any = r.any;
    if (first_wave) store_loss<G>(a, row, s, r, lane);
  }
  if (!a.grad) return;
  T *grad = (T *)a.grad + row * a.ldg;
  const float weight = r.any ? a.temperature * (a.weight ? a.weight[row] : 1.0f) : 0.0f;
  const float per = r.mass == 0.0f ? 0.0f : 1.0f / r.mass;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int j = (c * G + lane) * V;
    if (j >= n) break;
    forget(x[c].raw);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float e = __builtin_amdgcn_exp2f((element<T>(x[c].raw, i) - r.most) * factor);
      v[i] = r.any ? weight * (e * per) : 0.0f;
    }
    store16<T>(grad + j, n - j, v);
  }
  if constexpr (G > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
  }
  if (first_wave) store_kept<T>(grad, s, r, factor, weight, per);
}

// Rows that do not fit a workgroup's registers: one walk for the sums, one for the gradient.  2048
// x 160,000 bfloat16, 655 MB: the loss in 111 us (5.9 TB/s), loss and gradient in 335 (two reads
// and a write), the gradient later in 264.  A row has one workgroup, so few long rows leave the
// chip idle: 8 x 1,048,576 bfloat16 57, 122 and 79 us.
template <typename T, bool BACKWARD>
__global__ __launch_bounds__(1024) void distill_long_kernel(DistillArgs a) {
  constexpr int G = 1024, V = kPerLoad<T>, L = 64, U = 4;
  __shared__ float2 lds[G / 64];
  __shared__ int lds_any;
  __shared__ __attribute__((aligned(16))) int32_t slot_id[L * kSlots];
  __shared__ float slot_p[L * kSlots];
  const int lane = threadIdx.x, n = a.n_classes;
  const int64_t row = row_of<G>(a.first);
  const T *z = (const T *)a.logits + row * a.ldl;
  const float inf = __builtin_inff(), factor = a.factor;
  const int whole = n / V * V;  // the row's whole loads; the elements past them are lanes' own
  Slots s;
  s.any = false;
  if (lane < 64) {
    s = load_slots<T, G>(a, row, z, lane);
    join_equal<G>(a, s, lane, slot_id, slot_p);
    asm volatile("" ::"v"(s.z[0]), "v"(s.z[1]), "v"(s.z[2]), "v"(s.z[3]));
  }
  RowStats r;
  if constexpr (BACKWARD) {
    if (lane == 0) lds_any = s.any;
    __syncthreads();
    s.any = lds_any != 0;
    r = {a.stats[2 * row], a.stats[2 * row + 1], s.any};
  } else {
    // A lane adds n / 1024 exponentials, too many for one float (2^27 equal ones were off by 1e-3):
    // those of a step are added in float, the steps in double.  They are relative to `base`, which
    // goes up to the largest logit only once that is 2^kAhead ahead in the exponential: a change of
    // scale is off by a rounding, logits that rise slowly would make one at every step, and so no
    // more than a few of them reach what the sum ends with.
    constexpr float kAhead = 4.0f;
    float base = lane < n - whole ? to_float(z[whole + lane]) : -inf, most = base;
    double sum = base == -inf ? 0.0 : 1.0;
    if (base != base || base == inf) sum = __builtin_nan("");
    for (int64_t j = (int64_t)lane * V; j < whole; j += (int64_t)G * V * U) {
      u32x4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u * G * V < whole) {
          __builtin_memcpy(&raw[u], z + j + u * G * V, 16);
        } else {
          const uint32_t f = fill_of((T)-inf);
          raw[u] = u32x4{f, f, f, f};
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) most = fmaxf(most, element<T>(raw[u], i));
      // (a base that is NaN goes too, the sum being NaN already)
      if (most != -inf && !((most - base) * factor <= kAhead)) {
        sum *= (double)__builtin_amdgcn_exp2f((base - most) * factor);
        base = most;
      }
      const float safe = base == -inf ? 0.0f : base;
      float step = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i)
          step += __builtin_amdgcn_exp2f((element<T>(raw[u], i) - safe) * factor);
      sum += (double)step;
    }
    if (most != most) most = base = -inf;  // NaN is in the sum
    if (base != most) sum *= (double)__builtin_amdgcn_exp2f((base - most) * factor);
    const float mass = (float)sum;
    r = join_stats<G>(most, mass, s.any, factor, lds, &lds_any);
    s.any = r.any;
    if (lane < 64) store_loss<G>(a, row, s, r, lane);
  }
  if (!a.grad) return;
  T *grad = (T *)a.grad + row * a.ldg;
  const float weight = r.any ? a.temperature * (a.weight ? a.weight[row] : 1.0f) : 0.0f;
  const float per = r.mass == 0.0f ? 0.0f : 1.0f / r.mass;
  auto grad_of = [&](float x) {
    return r.any ? weight * (__builtin_amdgcn_exp2f((x - r.most) * factor) * per) : 0.0f;
  };
#pragma unroll 4
  for (int64_t j = (int64_t)lane * V; j < whole; j += G * V) {
    u32x4 raw;
    __builtin_memcpy(&raw, z + j, 16);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = grad_of(element<T>(raw, i));
    store16<T>(grad + j, V, v);
  }
  if (lane < n - whole) grad[whole + lane] = from_float<T>(grad_of(to_float(z[whole + lane])));
  __syncthreads();
  if (lane < 64) store_kept<T>(grad, s, r, factor, weight, per);
}

// Few lanes a row, so that a wave's reductions and slots serve many rows, but enough for its slots
// (four a lane), and no more loads a lane than leave the registers for many waves.  Loss and
// gradient, us, lanes x loads: 1M x 10 float (k = 4) 4 x 1 30, 8 x 1 58, 16 x 1 112; 1M x 64 (8) 8
// x 2 108, 16 x 1 148; 200,000 x 200 (10) 32 x 2 68, 16 x 4 74, 64 x 1 111; 100,000 x 347 (10) 32 x
// 4 55, 64 x 2 64; 100,000 x 500 (10) 64 x 2 74, 32 x 4 81; 20,000 x 1500 (20) 64 x 8 43, 256 x 2
// 44; 20,000 x 1700 (20) 256 x 2 47, 64 x 8 50; 20,000 x 4836 bfloat16 (84) 256 x 4 104, 512 x 2
// 161; 8192 x 12,000 (32) 512 x 4 75, 256 x 8 79, 1024 x 2 87; 4096 x 32,000 (64) 1024 x 4 100, 512
// x 8 107; 2048 x 128,000 (32) 1024 x 16 218, two walks over memory 257.
template <typename T, bool BACKWARD>
static int launch_pass(const DistillArgs &a, void *stream) {
  const int64_t bytes = (int64_t)a.n_classes * (int)sizeof(T);
  auto of = [&](auto k, int lanes) { return launch_rows(k, lanes, a, stream); };
  if (bytes < 16)
    return a.k <= 4 ? of(distill_kernel<T, 1, 1, true, BACKWARD>, 1)
                    : of(distill_kernel<T, 64, 1, true, BACKWARD>, 64);
  if (bytes <= 64 && a.k <= 16) return of(distill_kernel<T, 4, 1, false, BACKWARD>, 4);
  if (bytes <= 128 && a.k <= 32) return of(distill_kernel<T, 8, 1, false, BACKWARD>, 8);
  if (bytes <= 256 && a.k <= 32) return of(distill_kernel<T, 8, 2, false, BACKWARD>, 8);
  if (bytes <= 256 && a.k <= 64) return of(distill_kernel<T, 16, 1, false, BACKWARD>, 16);
  if (bytes <= 512 && a.k <= 64) return of(distill_kernel<T, 16, 2, false, BACKWARD>, 16);
  if (bytes <= 1024 && a.k <= 128) return of(distill_kernel<T, 32, 2, false, BACKWARD>, 32);
  if (bytes <= 1024) return of(distill_kernel<T, 64, 1, false, BACKWARD>, 64);
  if (bytes <= 1664 && a.k <= 128) return of(distill_kernel<T, 32, 4, false, BACKWARD>, 32);
  if (bytes <= 2048) return of(distill_kernel<T, 64, 2, false, BACKWARD>, 64);
  if (bytes <= 4096) return of(distill_kernel<T, 64, 4, false, BACKWARD>, 64);
  if (bytes <= 6144) return of(distill_kernel<T, 64, 8, false, BACKWARD>, 64);
  if (bytes <= 8192) return of(distill_kernel<T, 256, 2, false, BACKWARD>, 256);
  if (bytes <= 16384) return of(distill_kernel<T, 256, 4, false, BACKWARD>, 256);
  if (bytes <= 32768) return of(distill_kernel<T, 512, 4, false, BACKWARD>, 512);
  if (bytes <= 65536) return of(distill_kernel<T, 1024, 4, false, BACKWARD>, 1024);
  if (bytes <= 131072) return of(distill_kernel<T, 1024, 8, false, BACKWARD>, 1024);
  if (bytes <= 262144) return of(distill_kernel<T, 1024, 16, false, BACKWARD>, 1024);
  return of(distill_long_kernel<T, BACKWARD>, 1024);
}

int launch_distill(const DistillArgs &args, int32_t dtype, bool backward, void *stream) {
  DistillArgs a = args;
  a.factor = (float)(1.4426950408889634 / (double)a.temperature);
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return backward ? launch_pass<T, true>(a, stream) : launch_pass<T, false>(a, stream);
  });
}

}  // namespace bridger
