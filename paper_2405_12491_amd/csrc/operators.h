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

struct EmbedArgs {
  const int32_t *ids;
  int64_t ldi;
  const int64_t *offsets;  // null: every slot reads the whole table
  const void *table;       // backward: the output's gradient
  int64_t ldt;
  int64_t n_rows;
  int32_t n_slots;
  int32_t n_entries;
  int32_t n_features;
  float scale;
  void *out;  // backward: the table's gradient
  int64_t ldo;
  void *workspace;  // backward
  int32_t tiles;    // parts of a row's features, one a workgroup
  int32_t parts;    // groups of lanes that share a row's slots
  int64_t first;    // the launch's first workgroup
};

struct DropoutArgs {
  const void *x;
  int64_t ldx;
  const void *residual;  // null: none
  int64_t ldr;
  int64_t n_rows;
  int32_t n_features;
  uint64_t limit;  // random numbers of 32 bits from here on keep their element
  float scale;     // of kept elements
  const int64_t *seed;
  uint32_t layer;
  void *out;
  int64_t ldo;
  int32_t tiles;  // parts of a row, one a workgroup
  int64_t first;  // the launch's first workgroup
};

struct LayerNormArgs {
  const void *x;
  int64_t ldx;
  const void *residual;  // null: none
  int64_t ldr;
  const void *weight;  // null: ones
  const void *bias;    // null: zeros
  int64_t n_rows;
  int32_t n_features;
  float eps;
  void *total;  // may be null
  int64_t ldt;
  void *out;
  int64_t ldo;
  float *stats;   // may be null
  int64_t first;  // the launch's first row
};

struct LayerNormGradArgs {
  const void *grad;
  int64_t ldg;
  const void *x;  // what the norm was taken of
  int64_t ldx;
  const float *stats;
  const void *weight;      // null: ones
  const void *grad_total;  // null: none
  int64_t lds;
  int64_t n_rows;
  int32_t n_features;
  void *dx;  // may be null
  int64_t ldd;
  void *dweight;   // may be null
  void *dbias;     // may be null
  float *partial;  // null: neither of both is wanted
  int32_t parts;   // workgroups whose sums `partial` holds
  int32_t tiles;   // parts of a long row, one a workgroup
  int64_t first;   // the launch's first row or workgroup
};

struct SampleArgs {
  const void *logits;
  int64_t ld;
  int64_t n_rows;
  int32_t n_classes;
  const float *u;
  double temperature, top_p, min_p;
  int32_t top_k;
  const float *temperatures, *top_ps, *min_ps;  // null: the values above for every row
  const int32_t *top_ks;
  int32_t *ids;
  float *logp;    // may be null
  int64_t first;  // the launch's first row
};

// Each returns a hipError_t as int.  Sizes are positive and every argument checked.
int launch_top_k(const TopKArgs &a, int32_t dtype, void *stream);
int launch_distill(const DistillArgs &a, int32_t dtype, bool backward, void *stream);
int launch_rmsnorm_q8(const RmsnormArgs &a, int32_t dtype, void *stream);
int launch_matmul_q8(const MatmulArgs &a, int32_t dtype, void *stream);
int launch_embed(const EmbedArgs &a, int32_t dtype, void *stream);
int launch_embed_backward(const EmbedArgs &a, int32_t dtype, void *stream);
// Bytes of workspace; n_rows * n_slots fits 31 bits.
int64_t embed_backward_bytes(int64_t n_rows, int32_t n_slots, int32_t n_entries,
                             int32_t n_features);

int launch_sample(const SampleArgs &a, int32_t dtype, void *stream);
int launch_dropout(const DropoutArgs &a, int32_t dtype, void *stream);
int launch_layer_norm(const LayerNormArgs &a, int32_t dtype, void *stream);
int launch_layer_norm_backward(const LayerNormGradArgs &a, int32_t dtype, void *stream);
int64_t layer_norm_backward_bytes(int64_t n_rows, int32_t n_features, int element_size);

}  // namespace bridger
