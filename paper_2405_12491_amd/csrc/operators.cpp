// operators.cpp -- C ABI of the row operators: argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "bridger.h"
#include "operators.h"

using namespace bridger;

namespace {

bridger_status invalid(const char *msg) { return report_error(BRIDGER_ERR_INVALID_ARGUMENT, msg); }

int bytes_of(int32_t dtype) {
  return dtype == BRIDGER_F32 ? 4 : dtype == BRIDGER_BF16 || dtype == BRIDGER_F16 ? 2 : 0;
}

// Rows of one array: `width` elements of `size` bytes, `ld` elements apart.
struct Rows {
  const void *p;
  int64_t n, width, ld;
  int size;

  uintptr_t at() const { return (uintptr_t)p; }
  int64_t pitch() const { return n > 1 ? ld * size : width * size; }
  // Bytes from the first element to the last; false if they do not fit an address.
  bool span(uint64_t *bytes) const {
    const __int128 s = (__int128)(n - 1) * pitch() + (__int128)width * size;
    *bytes = (uint64_t)s;
    return s <= (__int128)INT64_MAX - (__int128)at();
  }
  const char *fault() const {
    if (!p) return "null array";
    if (at() % (uintptr_t)size) return "an array is not aligned to its element size";
    if (n > 1 && (ld < width || ld > INT64_MAX / 4))
      return "the distance between rows is smaller than a row, or too large";
    uint64_t b;
    if (!span(&b)) return "an array does not fit the address space";
    return nullptr;
  }
};

// Whether two arrays share an element.  Rows of one pitch may lie side by side in one buffer.
bool overlap(const Rows &a, const Rows &b) {
  if (!a.p || !b.p) return false;
  uint64_t sa = 0, sb = 0;
  a.span(&sa);
  b.span(&sb);
  if (a.at() + sa <= b.at() || b.at() + sb <= a.at()) return false;
  if (a.n > 1 && b.n > 1 && a.pitch() == b.pitch()) {
    const int64_t pitch = a.pitch();
    const int64_t d = (int64_t)(b.at() - a.at());
    const int64_t off = ((d % pitch) + pitch) % pitch;  // b's rows within a's pitch
    if (off >= a.width * a.size && off + b.width * b.size <= pitch) return false;
  }
  return true;
}

bool same(const Rows &a, const Rows &b) {
  return a.p == b.p && a.size == b.size && a.width == b.width && a.n == b.n &&
         (a.n == 1 || a.ld == b.ld);
}

constexpr int64_t kMaxRows = INT32_MAX;

const char *count_fault(int64_t n_rows, int32_t width) {
  if (n_rows < 0) return "n_rows < 0";
  if (n_rows > kMaxRows) return "n_rows above 2^31 - 1";
  if (width < 1) return "a row's width must be >= 1";
  return nullptr;
}

bridger_status device_ready() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return report_error(BRIDGER_ERR_DEVICE, "no usable GPU");
  }
  return BRIDGER_OK;
}

// Runs a launcher; nothing throws across the interface.
template <typename F>
bridger_status launched(F f) {
  int err;
  try {
    err = f();
  } catch (...) {
    return report_error(BRIDGER_ERR_OUT_OF_MEMORY, "host allocation failed");
  }
  if (err == 0) return BRIDGER_OK;
  (void)hipGetLastError();
  return report_error(BRIDGER_ERR_DEVICE, hipGetErrorString((hipError_t)err));
}

// The arguments that both passes of the distillation have; nullptr when they are sound.
const char *distill_fault(const DistillArgs &a, int32_t dtype, int32_t teacher_dtype) {
  if (const char *f = count_fault(a.n_rows, a.n_classes)) return f;
  if (!bytes_of(dtype) || !bytes_of(teacher_dtype)) return "unknown dtype";
  if (a.k < 1 || a.k > BRIDGER_MAX_TOP) return "k must be between 1 and BRIDGER_MAX_TOP";
  if (!(a.temperature >= 1e-6f && a.temperature <= 1e6f))
    return "temperature must lie between 1e-6 and 1e6";
  return nullptr;
}

// What every row operator's arrays have to satisfy: sound inputs and outputs, and no output that
// shares an element with another array, but for the pairs in `alias` (equal arrays).
const char *arrays_fault(const Rows *in, int n_in, const Rows *out, int n_out,
                         bool (*alias)(int in, int out)) {
  for (int i = 0; i < n_in; ++i)
    if (const char *f = in[i].p ? in[i].fault() : nullptr) return f;
  for (int o = 0; o < n_out; ++o) {
    if (!out[o].p) continue;
    if (const char *f = out[o].fault()) return f;
    for (int i = 0; i < n_in; ++i)
      if (overlap(in[i], out[o]) && !(alias && alias(i, o) && same(in[i], out[o])))
        return "an output overlaps an input";
    for (int q = 0; q < o; ++q)
      if (overlap(out[q], out[o])) return "two outputs overlap";
  }
  return nullptr;
}

}  // namespace

extern "C" {

bridger_status bridger_top_k(const void *scores, int64_t ld, int32_t dtype, int64_t n_rows,
                             int32_t n_classes, int32_t k, void *values, int32_t *ids,
                             void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_classes)) return invalid(f);
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (k < 1 || k > BRIDGER_MAX_TOP) return invalid("k must be between 1 and BRIDGER_MAX_TOP");
  if (n_rows == 0) return BRIDGER_OK;
  if (!scores || (!values && !ids)) return invalid("null scores, or no output");
  const Rows in[] = {{scores, n_rows, n_classes, ld, size}};
  const Rows out[] = {{values, n_rows, k, k, size}, {ids, n_rows, k, k, 4}};
  if (const char *f = arrays_fault(in, 1, out, 2, nullptr)) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_top_k({scores, ld, n_rows, n_classes, k, values, ids, 0}, dtype, stream);
  });
}

bridger_status bridger_distill(const void *logits, int64_t ldl, int32_t dtype, const int32_t *ids,
                               const void *teacher, int32_t teacher_dtype, int64_t n_rows,
                               int32_t n_classes, int32_t k, float temperature,
                               const float *weight, float *loss, float *stats, void *grad,
                               int64_t ldg, void *stream) {
  clear_error();
  const DistillArgs a = {logits, ldl,    ids,  teacher, n_rows, n_classes, k, temperature,
                         weight, loss, stats, grad,    ldg, teacher_dtype, 0};
  if (const char *f = distill_fault(a, dtype, teacher_dtype)) return invalid(f);
  if (n_rows == 0) return BRIDGER_OK;
  if (!logits || !ids || !teacher) return invalid("null logits, ids or teacher");
  if (!loss && !stats && !grad) return invalid("no output");
  const int size = bytes_of(dtype);
  const Rows in[] = {{logits, n_rows, n_classes, ldl, size},
                     {ids, n_rows, k, k, 4},
                     {teacher, n_rows, k, k, bytes_of(teacher_dtype)},
                     {weight, n_rows, 1, 1, 4}};
  const Rows out[] = {
      {loss, n_rows, 1, 1, 4}, {stats, n_rows, 2, 2, 4}, {grad, n_rows, n_classes, ldg, size}};
  if (const char *f =
          arrays_fault(in, 4, out, 3, [](int i, int o) { return i == 0 && o == 2; }))
    return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_distill(a, dtype, false, stream);
  });
}

bridger_status bridger_distill_backward(const void *logits, int64_t ldl, int32_t dtype,
                                        const int32_t *ids, const void *teacher,
                                        int32_t teacher_dtype, int64_t n_rows, int32_t n_classes,
                                        int32_t k, float temperature, const float *stats,
                                        const float *weight, void *grad, int64_t ldg,
                                        void *stream) {
  clear_error();
  const DistillArgs a = {logits, ldl,     ids, teacher, n_rows, n_classes, k, temperature,
                         weight, nullptr, const_cast<float *>(stats), grad, ldg, teacher_dtype, 0};
  if (const char *f = distill_fault(a, dtype, teacher_dtype)) return invalid(f);
  if (n_rows == 0) return BRIDGER_OK;
  if (!logits || !ids || !teacher || !stats) return invalid("null logits, ids, teacher or stats");
  if (!grad) return invalid("null gradient");
  const int size = bytes_of(dtype);
  const Rows in[] = {{logits, n_rows, n_classes, ldl, size},
                     {ids, n_rows, k, k, 4},
                     {teacher, n_rows, k, k, bytes_of(teacher_dtype)},
                     {weight, n_rows, 1, 1, 4},
                     {stats, n_rows, 2, 2, 4}};
  const Rows out[] = {{grad, n_rows, n_classes, ldg, size}};
  if (const char *f = arrays_fault(in, 5, out, 1, [](int i, int) { return i == 0; }))
    return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_distill(a, dtype, true, stream);
  });
}

bridger_status bridger_rmsnorm_q8(const void *x, int64_t ldx, const void *residual, int64_t ldr,
                                  const void *weight, int32_t dtype, int64_t n_rows,
                                  int32_t n_features, float eps, void *total, int64_t ldt,
                                  int8_t *q, int64_t ldq, float *scale, void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_features)) return invalid(f);
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (!(eps >= 0.0f) || std::isinf(eps)) return invalid("eps must be finite and >= 0");
  if (n_rows == 0) return BRIDGER_OK;
  if (!x || !q || !scale) return invalid("null x, q or scale");
  const Rows in[] = {{x, n_rows, n_features, ldx, size},
                     {residual, n_rows, n_features, ldr, size},
                     {weight, 1, n_features, n_features, size}};
  const Rows out[] = {{total, n_rows, n_features, ldt, size},
                      {q, n_rows, n_features, ldq, 1},
                      {scale, n_rows, 1, 1, 4}};
  if (const char *f =
          arrays_fault(in, 3, out, 3, [](int i, int o) { return i < 2 && o == 0; }))
    return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_rmsnorm_q8({x, ldx, residual, ldr, weight, n_rows, n_features, eps, total,
                                     ldt, q, ldq, scale, 1.0 / n_features, 0},
                                    dtype, stream);
  });
}

bridger_status bridger_matmul_q8(const int8_t *a, int64_t lda, const float *a_scale,
                                 const int8_t *b, int64_t ldb, const float *b_scale,
                                 const float *bias, int64_t n_rows, int32_t n_outputs,
                                 int32_t n_features, int32_t dtype, void *out, int64_t ldo,
                                 void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_features)) return invalid(f);
  if (n_outputs < 1) return invalid("n_outputs must be >= 1");
  if (n_features > BRIDGER_MATMUL_Q8_MAX_FEATURES)
    return report_error(BRIDGER_ERR_UNSUPPORTED,
                        "n_features above BRIDGER_MATMUL_Q8_MAX_FEATURES: a sum could leave 32 bits");
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (n_rows == 0) return BRIDGER_OK;
  if (!a || !a_scale || !b || !b_scale || !out) return invalid("null array");
  const Rows in[] = {{a, n_rows, n_features, lda, 1},
                     {a_scale, n_rows, 1, 1, 4},
                     {b, n_outputs, n_features, ldb, 1},
                     {b_scale, n_outputs, 1, 1, 4},
                     {bias, n_outputs, 1, 1, 4}};
  const Rows o[] = {{out, n_rows, n_outputs, ldo, size}};
  if (const char *f = arrays_fault(in, 5, o, 1, nullptr)) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_matmul_q8({a, lda, a_scale, b, ldb, b_scale, bias, n_rows, n_outputs,
                                    n_features, out, ldo},
                                   dtype, stream);
  });
}

}  // extern "C"
