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

// The sizes that both passes of the lookup have; nullptr when they are sound.
const char *embed_fault(const EmbedArgs &a, int32_t dtype) {
  if (const char *f = count_fault(a.n_rows, a.n_features)) return f;
  if (a.n_slots < 1) return "n_slots must be >= 1";
  if (a.n_entries < 1) return "n_entries must be >= 1";
  if (!bytes_of(dtype)) return "unknown dtype";
  if (!std::isfinite(a.scale)) return "scale must be finite";
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

bridger_status bridger_embed(const int32_t *ids, int64_t ldi, const int64_t *offsets,
                             const void *table, int64_t ldt, int32_t dtype, int64_t n_rows,
                             int32_t n_slots, int32_t n_entries, int32_t n_features, float scale,
                             void *out, int64_t ldo, void *stream) {
  clear_error();
  const EmbedArgs a = {ids,        ldi,   offsets, table, ldt,     n_rows, n_slots, n_entries,
                       n_features, scale, out,     ldo,   nullptr, 1,      1,       0};
  if (const char *f = embed_fault(a, dtype)) return invalid(f);
  if (n_rows == 0) return BRIDGER_OK;
  if (!ids || !table || !out) return invalid("null ids, table or output");
  const int size = bytes_of(dtype);
  const Rows in[] = {{ids, n_rows, n_slots, ldi, 4},
                     {offsets, 1, (int64_t)n_slots + 1, (int64_t)n_slots + 1, 8},
                     {table, n_entries, n_features, ldt, size}};
  const Rows o[] = {{out, n_rows, n_features, ldo, size}};
  if (const char *f = arrays_fault(in, 3, o, 1, nullptr)) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] { return launch_embed(a, dtype, stream); });
}

int64_t bridger_embed_backward_workspace(int64_t n_rows, int32_t n_slots, int32_t n_entries,
                                         int32_t n_features) {
  const EmbedArgs a = {nullptr, 0,          nullptr, nullptr, 0, n_rows, n_slots, n_entries,
                       n_features, 1.0f, nullptr, 0,       nullptr, 1, 1,       0};
  if (embed_fault(a, BRIDGER_F32) || n_rows > INT32_MAX / (int64_t)n_slots) return 0;
  return embed_backward_bytes(n_rows, n_slots, n_entries, n_features);
}

bridger_status bridger_embed_backward(const int32_t *ids, int64_t ldi, const int64_t *offsets,
                                      const void *grad, int64_t ldg, int32_t dtype, int64_t n_rows,
                                      int32_t n_slots, int32_t n_entries, int32_t n_features,
                                      float scale, void *grad_table, int64_t ldt, void *workspace,
                                      int64_t workspace_bytes, void *stream) {
  clear_error();
  const EmbedArgs a = {ids,        ldi,   offsets,    grad, ldg,       n_rows, n_slots, n_entries,
                       n_features, scale, grad_table, ldt,  workspace, 1,      1,       0};
  if (const char *f = embed_fault(a, dtype)) return invalid(f);
  if (n_rows > INT32_MAX / (int64_t)n_slots)
    return report_error(BRIDGER_ERR_UNSUPPORTED, "more than 2^31 - 1 slots");
  if ((n_rows && (!ids || !grad)) || !grad_table || !workspace)
    return invalid("null ids, gradient, table's gradient or workspace");
  if ((uintptr_t)workspace % 16) return invalid("the workspace is not aligned to 16 bytes");
  const int64_t bytes = embed_backward_bytes(n_rows, n_slots, n_entries, n_features);
  if (workspace_bytes < bytes) return invalid("the workspace is too small");
  const int size = bytes_of(dtype);
  const Rows in[] = {{n_rows ? ids : nullptr, n_rows, n_slots, ldi, 4},
                     {n_rows ? offsets : nullptr, 1, (int64_t)n_slots + 1, (int64_t)n_slots + 1, 8},
                     {n_rows ? grad : nullptr, n_rows, n_features, ldg, size}};
  const Rows o[] = {{grad_table, n_entries, n_features, ldt, size}, {workspace, 1, bytes, bytes, 1}};
  if (const char *f = arrays_fault(in, 3, o, 2, nullptr)) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] { return launch_embed_backward(a, dtype, stream); });
}

bridger_status bridger_sample(const void *logits, int64_t ld, int32_t dtype, int64_t n_rows,
                              int32_t n_classes, const float *u, double temperature,
                              const float *temperatures, int32_t top_k, const int32_t *top_ks,
                              double top_p, const float *top_ps, double min_p, const float *min_ps,
                              int32_t *ids, float *logp, void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_classes)) return invalid(f);
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (!(temperature >= 0.0 && temperature <= 1e6))
    return invalid("temperature must lie between 0 and 1e6");
  if (top_k < 0) return invalid("top_k < 0");
  if (!(top_p >= 0.0 && top_p <= 1.0)) return invalid("top_p must lie between 0 and 1");
  if (!(min_p >= 0.0 && min_p <= 1.0)) return invalid("min_p must lie between 0 and 1");
  if (n_rows == 0) return BRIDGER_OK;
  if (!logits || !u || !ids) return invalid("null logits, u or ids");
  const Rows in[] = {{logits, n_rows, n_classes, ld, size}, {u, n_rows, 1, 1, 4},
                     {temperatures, n_rows, 1, 1, 4},       {top_ks, n_rows, 1, 1, 4},
                     {top_ps, n_rows, 1, 1, 4},             {min_ps, n_rows, 1, 1, 4}};
  const Rows out[] = {{ids, n_rows, 1, 1, 4}, {logp, n_rows, 1, 1, 4}};
  if (const char *f = arrays_fault(in, 6, out, 2, nullptr)) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_sample({logits, ld, n_rows, n_classes, u, temperature, top_p, min_p, top_k,
                          temperatures, top_ps, min_ps, top_ks, ids, logp, 0},
                         dtype, stream);
  });
}

bridger_status bridger_dropout(const void *x, int64_t ldx, const void *residual, int64_t ldr,
                               int32_t dtype, int64_t n_rows, int32_t n_features, double p,
                               const int64_t *seed, int32_t layer, void *out, int64_t ldo,
                               void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_features)) return invalid(f);
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (!(p >= 0.0 && p <= 1.0)) return invalid("p must lie between 0 and 1");
  if (layer < 0) return invalid("layer < 0");
  if (n_rows == 0) return BRIDGER_OK;
  if (!x || !seed || !out) return invalid("null x, seed or output");
  const Rows in[] = {{x, n_rows, n_features, ldx, size},
                     {residual, n_rows, n_features, ldr, size},
                     {seed, 1, 2, 2, 8}};
  const Rows o[] = {{out, n_rows, n_features, ldo, size}};
  if (const char *f = arrays_fault(in, 3, o, 1, [](int i, int) { return i < 2; })) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  const uint64_t limit = (uint64_t)std::nearbyint(p * 4294967296.0);
  const float scale = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f;
  return launched([&] {
    return launch_dropout({x, ldx, residual, ldr, n_rows, n_features, limit, scale, seed,
                           (uint32_t)layer, out, ldo, 1, 0},
                          dtype, stream);
  });
}

bridger_status bridger_layer_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr,
                                  const void *weight, const void *bias, int32_t dtype,
                                  int64_t n_rows, int32_t n_features, float eps, void *total,
                                  int64_t ldt, void *out, int64_t ldo, float *stats, void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_features)) return invalid(f);
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (!(eps >= 0.0f) || std::isinf(eps)) return invalid("eps must be finite and >= 0");
  if (n_rows == 0) return BRIDGER_OK;
  if (!x || !out) return invalid("null x or output");
  const Rows in[] = {{x, n_rows, n_features, ldx, size},
                     {residual, n_rows, n_features, ldr, size},
                     {weight, 1, n_features, n_features, size},
                     {bias, 1, n_features, n_features, size}};
  const Rows o[] = {{total, n_rows, n_features, ldt, size},
                    {out, n_rows, n_features, ldo, size},
                    {stats, n_rows, 3, 3, 4}};
  if (const char *f = arrays_fault(in, 4, o, 3, [](int i, int q) { return i < 2 && q == 0; }))
    return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_layer_norm({x, ldx, residual, ldr, weight, bias, n_rows, n_features, eps, total,
                              ldt, out, ldo, stats, 0},
                             dtype, stream);
  });
}

int64_t bridger_layer_norm_backward_workspace(int64_t n_rows, int32_t n_features, int32_t dtype) {
  const int size = bytes_of(dtype);
  if (count_fault(n_rows, n_features) || !size) return 0;
  return layer_norm_backward_bytes(n_rows, n_features, size);
}

bridger_status bridger_layer_norm_backward(const void *grad, int64_t ldg, const void *t, int64_t ldt,
                                           const float *stats, const void *weight,
                                           const void *grad_total, int64_t lds, int32_t dtype,
                                           int64_t n_rows, int32_t n_features, void *dx, int64_t ldd,
                                           void *dweight, void *dbias, void *workspace,
                                           int64_t workspace_bytes, void *stream) {
  clear_error();
  if (const char *f = count_fault(n_rows, n_features)) return invalid(f);
  const int size = bytes_of(dtype);
  if (!size) return invalid("unknown dtype");
  if (!dx && !dweight && !dbias) return invalid("no output");
  const bool weights = dweight || dbias;
  if (n_rows == 0 && !weights) return BRIDGER_OK;
  if (n_rows && (!grad || !t || !stats)) return invalid("null gradient, t or stats");
  const int64_t bytes = weights ? layer_norm_backward_bytes(n_rows, n_features, size) : 0;
  if (bytes && !workspace) return invalid("null workspace");
  if (bytes && (uintptr_t)workspace % 16) return invalid("the workspace is not aligned to 16 bytes");
  if (workspace_bytes < bytes) return invalid("the workspace is too small");
  const bool rows = n_rows > 0;
  const Rows in[] = {{rows ? grad : nullptr, n_rows, n_features, ldg, size},
                     {rows ? t : nullptr, n_rows, n_features, ldt, size},
                     {rows ? stats : nullptr, n_rows, 3, 3, 4},
                     {rows ? weight : nullptr, 1, n_features, n_features, size},
                     {rows ? grad_total : nullptr, n_rows, n_features, lds, size}};
  const Rows o[] = {{rows ? dx : nullptr, n_rows, n_features, ldd, size},
                    {dweight, 1, n_features, n_features, size},
                    {dbias, 1, n_features, n_features, size},
                    {bytes ? workspace : nullptr, 1, bytes, bytes, 1}};
  if (const char *f = arrays_fault(in, 5, o, 4, nullptr)) return invalid(f);
  if (bridger_status s = device_ready()) return s;
  return launched([&] {
    return launch_layer_norm_backward(
        {grad, ldg, t, ldt, stats, weight, grad_total, lds, n_rows, n_features, rows ? dx : nullptr,
         ldd, dweight, dbias, weights ? (float *)workspace : nullptr, 0, 1, 0},
        dtype, stream);
  });
}

}  // extern "C"
