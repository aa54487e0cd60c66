// matmul_q8.hip -- gfx950 kernels of bridger_matmul_q8 (v_mfma_i32_16x16x64_i8).
#include "rows.h"

namespace bridger {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a row from `j`, zeros from `n` on.
__device__ inline i32x4 load_k16(const int8_t *p, int j, int n) {
  union {
    int8_t b[16];
    i32x4 v;
  } u;
#pragma unroll
  for (int i = 0; i < 16; ++i) u.b[i] = j + i < n ? p[j + i] : (int8_t)0;
  return u.v;
}

// One wave a tile of 16 x 16 outputs.  Lane l holds row (of a) and output (of b) l & 15 at the 16
// features from 16 (l >> 4) of each block of 64; rows and outputs past the end repeat the last one
// and are not stored.
template <typename T>
__global__ __launch_bounds__(64) void matmul_q8_kernel(MatmulArgs a) {
  const int lane = threadIdx.x, at = lane & 15, part = lane >> 4;
  const int64_t tiles_o = (a.n_outputs + 15) / 16, tiles = (a.n_rows + 15) / 16 * tiles_o;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t r0 = t / tiles_o * 16, o0 = t % tiles_o * 16;
    const int64_t r = r0 + at < a.n_rows ? r0 + at : a.n_rows - 1;
    const int64_t o = o0 + at < a.n_outputs ? o0 + at : a.n_outputs - 1;
    i32x4 c = {0, 0, 0, 0};
    for (int j = 0; j < a.n_features; j += 64)
      c = __builtin_amdgcn_mfma_i32_16x16x64_i8(
          load_k16(a.a + r * a.lda, j + 16 * part, a.n_features),
          load_k16(a.b + o * a.ldb, j + 16 * part, a.n_features), c, 0, 0, 0);
    if (o0 + at >= a.n_outputs) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = r0 + 4 * part + i;
      if (row >= a.n_rows) break;
      float y = (float)c[i] * a.a_scale[row] * a.b_scale[o0 + at];
      if (a.bias) y += a.bias[o0 + at];
      ((T *)a.out)[row * a.ldo + o0 + at] = from_float<T>(y);
    }
  }
}

int launch_matmul_q8(const MatmulArgs &a, int32_t dtype, void *stream) {
  const int64_t tiles = ((a.n_rows + 15) / 16) * (((int64_t)a.n_outputs + 15) / 16);
  return with_type(dtype, [&](auto t) {
    return launch(matmul_q8_kernel<decltype(t)>, (tiles < (1 << 20) ? tiles : 1 << 20), 64, 0, a, stream);
  });
}

}  // namespace bridger
