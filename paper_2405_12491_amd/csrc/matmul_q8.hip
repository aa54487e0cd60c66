// matmul_q8.hip -- gfx950 kernels of bridger_matmul_q8: 8-bit matrix cores, exact 32-bit sums.
//
// The matrix instructions take the weights as their first operand, so that a lane ends with four
// neighbouring outputs of one row.  Both operands share the order of the features within an
// instruction, so any fixed order of them gives the same sum.
#include "rows.h"

namespace bridger {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// 16 features of a row from j on; zeros from n on.  SHORT: n may be below 16.
template <bool SHORT>
__device__ inline i32x4 load_features(const int8_t *row, int j, int n) {
  i32x4 v;
  if (!SHORT || n >= 16) {  // the 16 bytes that end the row, moved down
    const int at = j < n - 16 ? j : n - 16;
    __builtin_memcpy(&v, row + at, 16);
    const int d = j - at;
    if (d > 0) {
      uint64_t lo = (uint32_t)v[0] | (uint64_t)(uint32_t)v[1] << 32;
      uint64_t hi = (uint32_t)v[2] | (uint64_t)(uint32_t)v[3] << 32;
      if (d >= 8) lo = hi, hi = 0;
      if (d >= 16) lo = 0;
      const int bits = 8 * (d & 7);
      if (bits) lo = lo >> bits | hi << (64 - bits), hi >>= bits;
      v = i32x4{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
    }
  } else {
    int8_t b[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) b[i] = j + i < n ? row[j + i] : (int8_t)0;
    __builtin_memcpy(&v, b, 16);
  }
  return v;
}

// Four neighbouring outputs of a row.
template <typename T>
__device__ inline void store_outputs(const MatmulArgs &a, int64_t row, int64_t o, i32x4 sum) {
  if (row >= a.n_rows || o >= a.n_outputs) return;
  const float row_scale = a.a_scale[row];
  T y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t at = o + i < a.n_outputs ? o + i : o;
    float v = (float)sum[i] * row_scale * a.b_scale[at];
    if (a.bias) v += a.bias[at];
    y[i] = from_float<T>(v);
  }
  T *out = (T *)a.out + row * a.ldo + o;
  if (o + 4 <= a.n_outputs) {
    __builtin_memcpy(out, y, sizeof(y));
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (o + i < a.n_outputs) out[i] = y[i];
  }
}

// ================================================================================ FEW ROWS
// A workgroup holds 16 R rows by 16 O outputs; its W waves share the features, each taking every
// W-th run of U x 64, straight from memory into the matrix instructions' registers (lane l: row or
// output l & 15, 16 features from 16 (l >> 4)), and join their sums in LDS.  So few rows still put
// enough waves on the chip to stream the weights, and nothing is shared beyond a workgroup.
template <typename T, int R, int O, int W, int U>
__global__ __launch_bounds__(64 * W) void matmul_q8_stream_kernel(MatmulArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15;
  const int n = a.n_features;
  const int64_t tiles_o = (a.n_outputs + 16 * O - 1) / (16 * O);
  const int64_t r0 = blockIdx.x / tiles_o * (16 * R), o0 = blockIdx.x % tiles_o * (16 * O);
  // past the end the last row, or output, stands in; its sums are not stored
  const int8_t *rows[R], *outs[O];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = r0 + 16 * r + at;
    rows[r] = a.a + (row < a.n_rows ? row : a.n_rows - 1) * a.lda + 16 * (lane >> 4);
  }
#pragma unroll
  for (int o = 0; o < O; ++o) {
    const int64_t out = o0 + 16 * o + at;
    outs[o] = a.b + (out < a.n_outputs ? out : a.n_outputs - 1) * a.ldb + 16 * (lane >> 4);
  }
  i32x4 sum[R][O] = {};
  int j = wave * U * 64;
  for (; j + U * 64 <= n; j += W * U * 64) {
    i32x4 x[U][R], w[U][O];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int o = 0; o < O; ++o) __builtin_memcpy(&w[u][o], outs[o] + j + 64 * u, 16);
#pragma unroll
      for (int r = 0; r < R; ++r) __builtin_memcpy(&x[u][r], rows[r] + j + 64 * u, 16);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int o = 0; o < O; ++o)
          sum[r][o] =
              __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][o], x[u][r], sum[r][o], 0, 0, 0);
  }
  // the last, partial run of features is one wave's
  for (const int end = j + U * 64; j < n && j < end; j += 64) {
    i32x4 x[R];
    const int part = 16 * (lane >> 4);
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = load_features<true>(rows[r] - part, j + part, n);
#pragma unroll
    for (int o = 0; o < O; ++o) {
      const i32x4 w = load_features<true>(outs[o] - part, j + part, n);
#pragma unroll
      for (int r = 0; r < R; ++r)
        sum[r][o] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x[r], sum[r][o], 0, 0, 0);
    }
  }
  i32x4 *lds = (i32x4 *)smem;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int o = 0; o < O; ++o) lds[((wave * R + r) * O + o) * 64 + lane] = sum[r][o];
  __syncthreads();
  for (int t = wave; t < R * O; t += W) {
    i32x4 all = lds[t * 64 + lane];
#pragma unroll
    for (int w = 1; w < W; ++w) all += lds[(w * R * O + t) * 64 + lane];
    store_outputs<T>(a, r0 + 16 * (t / O) + at, o0 + 16 * (t % O) + 4 * (lane >> 4), all);
  }
}

// =============================================================================== MANY ROWS
// A workgroup of 2 x 2 waves holds B x B outputs, each wave (B / 2) x (B / 2) in tiles of 32 x 32
// (v_mfma_i32_32x32x32_i8).  Stages of 128 features of its rows and weights go to LDS, two stages
// in turn, one being filled while the other is multiplied; a wave reads the operands of a step of
// 32 features while the matrix cores work on the step before.  In LDS a row's eight 16-byte chunks
// stand at chunk ^ (row & 7), so that the 32 rows that one instruction reads hit all banks.
constexpr int kStage = 128;

template <int B>
constexpr int kTileLds = 2 * 2 * B * kStage;

typedef __attribute__((address_space(3))) uint8_t lds_byte;

// ALIGNED: rows of a and b start at multiples of 16 bytes and lie within 2^32 bytes of the tile's
// first; stages then go to LDS without passing registers.
template <typename T, int B, bool ALIGNED>
__global__ __launch_bounds__(256) void matmul_q8_tile_kernel(MatmulArgs a) {
  constexpr int C = B / 64;       // 32 x 32 tiles of a wave, each way
  constexpr int P = B * 8 / 256;  // 16-byte chunks of a stage that a thread brings, for each matrix
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int n = a.n_features;
  // Workgroups of one XCD (every eighth) take neighbouring tiles, in columns of 8 tiles of rows:
  // those that run together share most of their rows and weights in the XCD's L2.
  const int64_t tiles_r = (a.n_rows + B - 1) / B, tiles_o = (a.n_outputs + B - 1) / B;
  const int64_t tiles = tiles_r * tiles_o;
  const int64_t share = tiles / 8, more = tiles % 8, xcd = blockIdx.x % 8;
  const int64_t tile = xcd * share + (xcd < more ? xcd : more) + blockIdx.x / 8;
  const int64_t group = tile / (8 * tiles_o), left = tiles_r - group * 8, height = left < 8 ? left : 8;
  const int64_t within = tile - group * 8 * tiles_o;
  const int64_t r0 = (group * 8 + within % height) * B, o0 = within / height * B;

  // thread t brings chunk (t & 7) ^ (row & 7) of rows t / 8 + 32 p to slot t & 7
  const int slot = t & 7, row_at = t >> 3, chunk = slot ^ (row_at & 7);
  const int8_t *from_a[P], *from_b[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t r = r0 + row_at + 32 * p, o = o0 + row_at + 32 * p;
    from_a[p] = a.a + (r < a.n_rows ? r : a.n_rows - 1) * a.lda;
    from_b[p] = a.b + (o < a.n_outputs ? o : a.n_outputs - 1) * a.ldb;
  }
  const int whole = n / kStage;
  uint8_t *lds_a = smem, *lds_b = smem + 2 * B * kStage;
  i32x4 hold_a[P], hold_b[P];  // a stage on its way through registers

  // starts to bring stage s
  auto fetch = [&](int s) __attribute__((always_inline)) {
    const int j = s * kStage + 16 * chunk;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if constexpr (ALIGNED) {
        lds_byte *to = (lds_byte *)smem + (s & 1) * B * kStage + wave * 1024 + p * 4096;
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void *)(from_a[p] + j),
            (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void *)(from_b[p] + j),
            (__attribute__((address_space(3))) void *)(to + 2 * B * kStage), 16, 0, 0);
      } else {
        __builtin_memcpy(&hold_a[p], from_a[p] + j, 16);
        __builtin_memcpy(&hold_b[p], from_b[p] + j, 16);
      }
    }
  };
  // a stage that is held in registers, to LDS
  auto put = [&](int s) __attribute__((always_inline)) {
    const int to = (s & 1) * B * kStage + t * 16;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      *(i32x4 *)(lds_a + to + p * 4096) = hold_a[p];
      *(i32x4 *)(lds_b + to + p * 4096) = hold_b[p];
    }
  };
  // lane l's operand: row (or output) l & 31, features from 16 (l >> 5) of a step of 32
  const int half = lane >> 5, row32 = lane & 31;
  const int base_a = ((wave >> 1) * (B / 2) + row32) * kStage;
  const int base_b = ((wave & 1) * (B / 2) + row32) * kStage;
  auto read = [&](int s, int step, i32x4(&x)[C], i32x4(&w)[C]) __attribute__((always_inline)) {
    const int at = (s & 1) * B * kStage + (((2 * step + half) ^ (row32 & 7)) << 4);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      x[c] = *(const i32x4 *)(lds_a + base_a + at + c * 32 * kStage);
      w[c] = *(const i32x4 *)(lds_b + base_b + at + c * 32 * kStage);
    }
  };
  i32x16 sum[C][C] = {};
  auto multiply = [&](const i32x4(&x)[C], const i32x4(&w)[C]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < C; ++r)
#pragma unroll
      for (int o = 0; o < C; ++o)
        sum[r][o] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[o], x[r], sum[r][o], 0, 0, 0);
  };
  // Every load to LDS issued so far is done, by all waves, and every read.
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  i32x4 x0[C], w0[C], x1[C], w1[C];
  if (whole > 0) {
    fetch(0);
    if (!ALIGNED) put(0);
    meet();
    read(0, 0, x0, w0);
    if (whole > 1) fetch(1);
    for (int s = 0; s < whole; ++s) {
      read(s, 1, x1, w1);
      multiply(x0, w0);
      read(s, 2, x0, w0);
      multiply(x1, w1);
      read(s, 3, x1, w1);
      if (!ALIGNED && s + 1 < whole) put(s + 1);
      multiply(x0, w0);
      if (s + 1 < whole) {
        meet();  // stage s + 1 is there, and nobody reads stage s any more
        read(s + 1, 0, x0, w0);
        if (s + 2 < whole) fetch(s + 2);
      }
      multiply(x1, w1);
    }
  }
  if (n % kStage) {  // the features past the last whole stage, filled up with zeros
    const int j = whole * kStage + 16 * chunk;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      hold_a[p] = load_features<false>(from_a[p], j, n);
      hold_b[p] = load_features<false>(from_b[p], j, n);
    }
    put(whole);  // nobody reads the other stage's place: it was left before the last meeting
    meet();
#pragma unroll 1
    for (int step = 0; step < (n % kStage + 31) / 32; ++step) {
      read(whole, step, x0, w0);
      multiply(x0, w0);
    }
  }
  // lane l holds row l & 31 and outputs 8 (i / 4) + 4 (l >> 5) + i % 4 of each tile
#pragma unroll
  for (int r = 0; r < C; ++r)
#pragma unroll
    for (int o = 0; o < C; ++o)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store_outputs<T>(a, r0 + (wave >> 1) * (B / 2) + 32 * r + row32,
                         o0 + (wave & 1) * (B / 2) + 32 * o + 8 * q + 4 * half,
                         i32x4{sum[r][o][4 * q], sum[r][o][4 * q + 1], sum[r][o][4 * q + 2],
                               sum[r][o][4 * q + 3]});
}

template <typename T, int R, int O, int W, int U>
static int launch_stream(const MatmulArgs &a, void *stream) {
  const int64_t tiles = ((a.n_rows + 16 * R - 1) / (16 * R)) *
                        (((int64_t)a.n_outputs + 16 * O - 1) / (16 * O));
  return launch_tiles(matmul_q8_stream_kernel<T, R, O, W, U>, tiles, 64 * W, W * R * O * 1024, a,
                      stream);
}
template <typename T, int B>
static int launch_tile(const MatmulArgs &a, void *stream) {
  const int64_t tiles =
      ((a.n_rows + B - 1) / B) * (((int64_t)a.n_outputs + B - 1) / B);
  const bool aligned = ((uintptr_t)a.a | (uintptr_t)a.b | (uint64_t)a.lda | (uint64_t)a.ldb) % 16 == 0;
  return aligned ? launch_tiles(matmul_q8_tile_kernel<T, B, true>, tiles, 256, kTileLds<B>, a, stream)
                 : launch_tiles(matmul_q8_tile_kernel<T, B, false>, tiles, 256, kTileLds<B>, a, stream);
}

int launch_matmul_q8(const MatmulArgs &a, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int64_t m = a.n_rows, o = a.n_outputs;
    if (a.n_features < 16) return launch_stream<T, 1, 1, 8, 4>(a, stream);
    if (m <= 16) return launch_stream<T, 1, 1, 8, 4>(a, stream);
    if (m <= 32) return launch_stream<T, 2, 1, 8, 4>(a, stream);
    if (m <= 64) return launch_stream<T, 4, 2, 4, 2>(a, stream);
    const int64_t wide = ((m + 255) / 256) * ((o + 255) / 256);
    const int64_t middle = ((m + 127) / 128) * ((o + 127) / 128);
    if (wide >= 192) return launch_tile<T, 256>(a, stream);
    if (middle >= 192) return launch_tile<T, 128>(a, stream);
    return launch_stream<T, 4, 4, 4, 1>(a, stream);
  });
}

}  // namespace bridger
