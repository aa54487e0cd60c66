// operators.h -- launch descriptors of the row operators, shared by operators.cpp (the C ABI's
// checks) and the HIP kernels.
#pragma once
#include <stdint.h>

#include "bridger.h"

namespace bridger {

// Records the message for bridger_last_error and returns s (bridger_host.cpp).
bridger_status report_error(bridger_status s, const char *msg);
void clear_error();

struct TopKArgs {
  const void *scores;
  int64_t ld;
  int64_t n_rows;
  int32_t n_classes;
  int32_t k;
  void *values;  // may be null
  int32_t *ids;  // may be null
  int64_t first;  // the launch's first row
};

struct DistillArgs {
  const void *logits;
  int64_t ldl;
  const int32_t *ids;
  const void *teacher;
  int64_t n_rows;
  int32_t n_classes;
  int32_t k;
  float temperature;
  const float *weight;  // null: ones
  float *loss;          // may be null
  float *stats;         // written by the forward pass (may be null), read by the backward pass
  void *grad;           // may be null in the forward pass
  int64_t ldg;
  int32_t teacher_dtype;
  int64_t first;  // the launch's first row
  float factor;   // log2(e) / temperature, rounded once
};

struct RmsnormArgs {
  const void *x;
  int64_t ldx;
  const void *residual;  // null: none
  int64_t ldr;
  const void *weight;  // null: ones
  int64_t n_rows;
  int32_t n_features;
  float eps;
  void *total;  // may be null
  int64_t ldt;
  int8_t *q;
  int64_t ldq;
  float *scale;
  double per_feature;  // 1 / n_features
  int64_t first;  // the launch's first row
};

struct MatmulArgs {
  const int8_t *a;
  int64_t lda;
  const float *a_scale;
  const int8_t *b;
  int64_t ldb;
  const float *b_scale;
  const float *bias;  // null: none
  int64_t n_rows;
  int32_t n_outputs;
  int32_t n_features;
  void *out;
  int64_t ldo;
};

// Each returns a hipError_t as int.  Sizes are positive and every argument checked.
int launch_top_k(const TopKArgs &a, int32_t dtype, void *stream);
int launch_distill(const DistillArgs &a, int32_t dtype, bool backward, void *stream);
int launch_rmsnorm_q8(const RmsnormArgs &a, int32_t dtype, void *stream);
int launch_matmul_q8(const MatmulArgs &a, int32_t dtype, void *stream);

}  // namespace bridger
