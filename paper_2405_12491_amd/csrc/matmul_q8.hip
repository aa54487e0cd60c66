// matmul_q8.hip -- gfx950 kernels of bridger_matmul_q8: 8-bit matrix cores, exact 32-bit sums.
//
// The matrix instructions take the weights as their first operand, so that a lane ends with four
// neighbouring outputs of one row.  Both operands share the order of the features within an
// instruction, so any fixed order of them gives the same sum.
#include <mutex>
#include <type_traits>

#include "rows.h"

namespace bridger {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// 16 features of a row (n of them, 16 at least) from j on; those that end the row where less is
// left.  move_down() brings the latter into place, zeros behind them.
__device__ inline i32x4 load_raw(const int8_t *row, int j, int n) {
  i32x4 v;
  __builtin_memcpy(&v, row + (j < n - 16 ? j : n - 16), 16);
  return v;
}
__device__ inline i32x4 move_down(i32x4 v, int j, int n) {
  const int d = j - n + 16;
  if (d <= 0) return v;
  uint64_t lo = (uint32_t)v[0] | (uint64_t)(uint32_t)v[1] << 32;
  uint64_t hi = (uint32_t)v[2] | (uint64_t)(uint32_t)v[3] << 32;
  if (d >= 8) lo = hi, hi = 0;
  if (d >= 16) lo = 0;
  const int bits = 8 * (d & 7);
  if (bits) lo = lo >> bits | hi << (64 - bits), hi >>= bits;
  return i32x4{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}
// A row below 16 features: j = 0 holds all of it.
__device__ inline i32x4 load_tiny(const int8_t *row, int j, int n) {
  i32x4 v;
  int8_t b[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) b[i] = j + i < n ? row[j + i] : (int8_t)0;
  __builtin_memcpy(&v, b, 16);
  return v;
}

// N neighbouring floats from `at` on; what lies past n is not read.
template <int N>
__device__ inline void load_floats(const float *p, int64_t at, int64_t n, float (&v)[N]) {
  if (at + N <= n) {
    __builtin_memcpy(v, p + at, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = at + i < n ? p[at + i] : 0.0f;
  }
}

// What four neighbouring outputs of a row take besides their sums.  Read ahead of the sums, so that
// a short call does not wait for memory twice.
struct Scales {
  float row, output[4], bias[4];

  __device__ void load(const MatmulArgs &a, int64_t r, int64_t o) {
    row = r < a.n_rows ? a.a_scale[r] : 0.0f;
    load_floats<4>(a.b_scale, o, a.n_outputs, output);
    if (a.bias) load_floats<4>(a.bias, o, a.n_outputs, bias);
  }
};

template <typename T>
__device__ inline void store_outputs(const MatmulArgs &a, int64_t row, int64_t o, i32x4 sum,
                                     const Scales &s) {
  if (row >= a.n_rows || o >= a.n_outputs) return;
  T y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v = (float)sum[i] * s.row * s.output[i];
    if (a.bias) v += s.bias[i];
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

// The tile of this workgroup: those of one XCD (every eighth workgroup) take neighbouring tiles.
__device__ inline int64_t tile_of(int64_t tiles) {
  const int64_t share = tiles / 8, more = tiles % 8, xcd = blockIdx.x % 8;
  return xcd * share + (xcd < more ? xcd : more) + blockIdx.x / 8;
}

// ================================================================================ FEW ROWS
// A workgroup holds 16 R rows by 16 O outputs; its W waves share the features, wave w taking stages
// w, w + W, .. of 64, and join their sums in LDS.  So few rows still put enough waves on the chip
// to stream the weights, and nothing is shared beyond a workgroup.  Each wave has a ring of S
// stages of its own in LDS and S - 1 of them on their way, without a barrier.  The detour through
// LDS is for the loads: an instruction that reads operands in place has neighbouring lanes in 16
// different rows, and takes 64 cycles; here four neighbouring lanes read 64 bytes of a row (16
// cycles).  A row's four 16-byte chunks stand at chunk ^ (row / 4 & 3): 16 rows of one chunk hit
// all banks.
// ALIGNED: rows go to LDS without passing registers (aligned_rows).
// One row is bound by memory: 1 x 32,000 x 4096, 131 MB in 25 us (5.3 TB/s).  Small
// products are bound by their chain of launch, first loads, stages and join: 77 x 4099 x 2047, 9
// MB, in 9.
typedef __attribute__((address_space(3))) uint8_t lds_byte;

// Rows [first, n) of a matrix, `ld` apart, for loads by 32-bit offsets from row `first`; what lies
// behind the matrix is out of its bounds.
__device__ inline __amdgpu_buffer_rsrc_t rows_from(const int8_t *p, int64_t ld, int64_t first,
                                                   int64_t n, int width) {
  const int64_t bytes = (n - 1 - first) * ld + width;
  return __builtin_amdgcn_make_buffer_rsrc((void *)(p + first * ld), 0,
                                           (int)(bytes < 0xFFFFFFFFll ? bytes : 0xFFFFFFFFll),
                                           0x27000);
}
// 16 bytes a lane to LDS, lane after lane from `to`.  (The buffer form: the compiler counts the
// global form among the LDS instructions too, and waits for all of those at every use of one.)
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t rows, int lane_offset, int offset,
                                   lds_byte *to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      rows, (__attribute__((address_space(3))) void *)to, 16, lane_offset, offset, 0, 0);
}

// At most V loads (and L LDS instructions) are still on their way.
template <int V, int L>
__device__ inline void wait_for() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((V & 15) | 7 << 4 | L << 8 | (V >> 4) << 14);
  asm volatile("" ::: "memory");
}

template <typename T, int R, int O, int W, int S, bool ALIGNED>
__global__ __launch_bounds__(64 * W) void matmul_q8_stream_kernel(MatmulArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  constexpr int N = R + O;  // 16-row parts of a stage, 1 KB and one load of a wave each
  const int lane = threadIdx.x & 63, at = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = a.n_features;
  // the tiles of one set of weights run side by side on one XCD, whose L2 they share
  const int64_t tiles_r = (a.n_rows + 16 * R - 1) / (16 * R);
  const int64_t tile = tile_of(gridDim.x);
  const int64_t r0 = tile % tiles_r * (16 * R), o0 = tile / tiles_r * (16 * O);
  // lane l brings chunk (l & 3) ^ (l / 16) of row l / 4 of each part to slot l & 3 of that row;
  // past the end the last row, or output, stands in: its sums are not stored
  auto row_of_part = [&](int p, int i) {
    const int64_t first = p < R ? r0 + 16 * p : o0 + 16 * (p - R), end = p < R ? a.n_rows : a.n_outputs;
    const int64_t row = first + i < end ? first + i : end - 1;
    return p < R ? a.a + row * a.lda : a.b + row * a.ldb;
  };
  const auto rows_a = rows_from(a.a, a.lda, r0, a.n_rows, n);
  const auto rows_b = rows_from(a.b, a.ldb, o0, a.n_outputs, n);
  const int8_t *from[N];
  int offset[N];
#pragma unroll
  for (int p = 0; p < N; ++p) {
    from[p] = row_of_part(p, lane >> 2) + 16 * ((lane & 3) ^ (lane >> 4)) + wave * 64;
    offset[p] = (int)(from[p] - (p < R ? a.a + r0 * a.lda : a.b + o0 * a.ldb));
  }
  const int whole = n / 64;                                     // stages without the last, partial one
  const int count = wave < whole ? (whole - wave + W - 1) / W : 0;  // this wave's
  constexpr int kRing = ALIGNED ? S : 1;
  uint8_t *ring = smem + wave * kRing * N * 1024;
  const uint8_t *operand = ring + at * 64 + (((lane >> 4) ^ (at >> 2)) << 4);
  i32x4 hold[ALIGNED ? 1 : S][N];
  auto issue = [&](int i, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < N; ++p)
      if constexpr (ALIGNED) {
        load_to_lds(p < R ? rows_a : rows_b, offset[p], i * (W * 64),
                    (lds_byte *)ring + (slot * N + p) * 1024);
      } else {
        __builtin_memcpy(&hold[slot][p], from[p] + (int64_t)i * (W * 64), 16);
      }
  };
  i32x4 sum[R][O] = {};
#pragma unroll
  for (int d = 0; d < S - 1; ++d)
    if (d < count) issue(d, d);
  // The features past the last whole stage, and what this wave's tiles take besides their sums:
  // asked for behind the first stages, where those do not fill the registers themselves.
  const bool tail = n % 64 && wave == whole % W;
  i32x4 last[N];
  const int last_at = whole * 64 + 16 * (lane >> 4);
  auto load_last = [&]() __attribute__((always_inline)) {
    if (tail && n >= 16) {
#pragma unroll
      for (int p = 0; p < N; ++p) last[p] = load_raw(row_of_part(p, at), last_at, n);
    }
  };
  constexpr int kTiles = (R * O + W - 1) / W;
  Scales scales[kTiles];
  auto load_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < kTiles; ++q) {
      const int t = wave + q * W;
      if (t < R * O) scales[q].load(a, r0 + 16 * (t / O) + at, o0 + 16 * (t % O) + 4 * (lane >> 4));
    }
  };
  if constexpr (ALIGNED) load_last(), load_scales();
  for (int i0 = 0; i0 < count; i0 += S) {
#pragma unroll
    for (int d = 0; d < S; ++d) {
      const int i = i0 + d;
      if (i >= count) break;
      wait_for<63, 0>();  // the slot that is filled next has been read
      if (i + S - 1 < count) {
        issue(i + S - 1, (d + S - 1) % S);
        if constexpr (ALIGNED) wait_for<(S - 1) * N, 15>();
      } else {
        if constexpr (ALIGNED) wait_for<0, 15>();
      }
      constexpr int kSlot = ALIGNED ? N * 1024 : 0;
      if constexpr (!ALIGNED) {
#pragma unroll
        for (int p = 0; p < N; ++p) *(i32x4 *)(ring + p * 1024 + lane * 16) = hold[d][p];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      i32x4 x[R], w[O];
#pragma unroll
      for (int o = 0; o < O; ++o) w[o] = *(const i32x4 *)(operand + d * kSlot + (R + o) * 1024);
#pragma unroll
      for (int r = 0; r < R; ++r) x[r] = *(const i32x4 *)(operand + d * kSlot + r * 1024);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int o = 0; o < O; ++o)
          sum[r][o] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[o], x[r], sum[r][o], 0, 0, 0);
    }
  }
  if constexpr (!ALIGNED) load_last(), load_scales();
  if (tail) {
#pragma unroll
    for (int p = 0; p < N; ++p)
      last[p] = n >= 16 ? move_down(last[p], last_at, n) : load_tiny(row_of_part(p, at), last_at, n);
#pragma unroll
    for (int o = 0; o < O; ++o)
#pragma unroll
      for (int r = 0; r < R; ++r)
        sum[r][o] =
            __builtin_amdgcn_mfma_i32_16x16x64_i8(last[R + o], last[r], sum[r][o], 0, 0, 0);
  }
  wait_for<0, 0>();
  __syncthreads();  // the rings are left
  i32x4 *lds = (i32x4 *)smem;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int o = 0; o < O; ++o) lds[((wave * R + r) * O + o) * 64 + lane] = sum[r][o];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kTiles; ++q) {
    const int t = wave + q * W;
    if (t >= R * O) break;
    i32x4 all = lds[t * 64 + lane];
#pragma unroll
    for (int w = 1; w < W; ++w) all += lds[(w * R * O + t) * 64 + lane];
    store_outputs<T>(a, r0 + 16 * (t / O) + at, o0 + 16 * (t % O) + 4 * (lane >> 4), all, scales[q]);
  }
}

// =============================================================================== MANY ROWS
// A workgroup of 2 x WO waves holds B x B outputs, each wave (B / 2) x (B / WO) in tiles of 32 x 32
// (v_mfma_i32_32x32x32_i8).  Stages of 128 features of its rows and weights go to a ring of stages
// in LDS, one being multiplied in steps of 32 features while the others are on their way.  In LDS a
// row's eight 16-byte chunks stand at chunk ^ (row / 2 & 7): the 16 lanes that are served in one
// cycle have 16 neighbouring rows, even ones in 32 of the 64 banks and odd ones in the others.
// 8192 x 8192 x 8192 in 443 to 452 us (2.43 to 2.48e15 operations/s).  The matrix cores are busy 76% of
// the cycles, and the clock falls to 1.6 GHz under random operands (2.2 with zeros, at the same
// count of cycles): power bounds it.
constexpr int kStage = 128;

template <int B, bool DEEP>
constexpr int kTileLds = (DEEP ? 4 : 2) * 2 * B * kStage;

// ALIGNED: stages go to LDS without passing registers (aligned_rows).
template <typename T, int B, int WO, bool DEEP, bool ALIGNED>
__global__ __launch_bounds__(128 * WO) void matmul_q8_tile_kernel(MatmulArgs a) {
  constexpr int kThreads = 128 * WO;
  constexpr int CR = B / 64, CO = B / (32 * WO);  // 32 x 32 tiles of a wave: of rows, of outputs
  constexpr int P = B * 8 / kThreads;  // 16-byte chunks of a stage that a thread brings, a matrix
  constexpr int S = DEEP ? 4 : 2;  // stages in LDS
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int n = a.n_features;
  // An XCD's tiles run in columns of 8 tiles of rows: those that run together share most of their
  // rows and weights in its L2.
  const int64_t tiles_r = (a.n_rows + B - 1) / B, tiles_o = (a.n_outputs + B - 1) / B;
  const int64_t tile = tile_of(tiles_r * tiles_o);
  const int64_t group = tile / (8 * tiles_o), left = tiles_r - group * 8, height = left < 8 ? left : 8;
  const int64_t within = tile - group * 8 * tiles_o;
  const int64_t r0 = (group * 8 + within % height) * B, o0 = within / height * B;

  // thread t brings chunk (t & 7) ^ (row / 2 & 7) of rows t / 8 + kThreads / 8 p to slot t & 7
  const int slot = t & 7, row_at = t >> 3, chunk = slot ^ (row_at >> 1 & 7);
  const auto rows_a = rows_from(a.a, a.lda, r0, a.n_rows, n);
  const auto rows_b = rows_from(a.b, a.ldb, o0, a.n_outputs, n);
  const int8_t *from[2 * P];
  int offset[2 * P];
#pragma unroll
  for (int p = 0; p < 2 * P; ++p) {
    const int64_t row = (p < P ? r0 : o0) + row_at + kThreads / 8 * (p % P);
    const int64_t end = p < P ? a.n_rows : a.n_outputs;
    from[p] = p < P ? a.a + (row < end ? row : end - 1) * a.lda
                    : a.b + (row < end ? row : end - 1) * a.ldb;
    offset[p] = (int)(from[p] - (p < P ? a.a + r0 * a.lda : a.b + o0 * a.ldb)) + 16 * chunk;
  }
  const int whole = n / kStage;
  uint8_t *lds_a = smem, *lds_b = smem + S * B * kStage;
  i32x4 hold[DEEP ? 2 : 1][2 * P];  // stages on their way through registers

  // starts to bring stage s: chunk p of a (p < P) or of b, into place h of hold
  auto fetch = [&](int s, int p, int h = 0) __attribute__((always_inline)) {
    if constexpr (ALIGNED) {
      lds_byte *to = (lds_byte *)smem + (p < P ? 0 : S * B * kStage) + (s & (S - 1)) * B * kStage +
                     wave * 1024 + p % P * (kThreads * 16);
      load_to_lds(p < P ? rows_a : rows_b, offset[p], s * kStage, to);
    } else {
      __builtin_memcpy(&hold[h][p], from[p] + s * kStage + 16 * chunk, 16);
    }
  };
  // a chunk that is held in registers, to LDS
  auto put = [&](int s, int p, int h = 0) __attribute__((always_inline)) {
    *(i32x4 *)((p < P ? lds_a : lds_b) + (s & (S - 1)) * B * kStage + t * 16 + p % P * (kThreads * 16)) =
        hold[h][p];
  };
  // lane l's operand: row (or output) l & 31, features from 16 (l >> 5) of a step of 32
  const int half = lane >> 5, row32 = lane & 31;
  const int base_a = (wave / WO * (32 * CR) + row32) * kStage;
  const int base_b = (wave % WO * (32 * CO) + row32) * kStage;
  struct Operands {
    i32x4 x[CR], w[CO];
  };
  constexpr int N = CR + CO;
  // operand i of a step: w, x in turn
  auto read = [&](int s, int step, int i, Operands &v) __attribute__((always_inline)) {
    const int at = (s & (S - 1)) * B * kStage + (((2 * step + half) ^ (row32 >> 1 & 7)) << 4);
    if (i < 2 * CO && i % 2 == 0) {
      v.w[i / 2] = *(const i32x4 *)(lds_b + base_b + at + i / 2 * 32 * kStage);
    } else {
      const int r = i < 2 * CO ? i / 2 : i - CO;
      v.x[r] = *(const i32x4 *)(lds_a + base_a + at + r * 32 * kStage);
    }
  };
  i32x16 sum[CR][CO] = {};
  // One step's matrix instructions, with beside(i) in the issue slots behind the i-th.  The order
  // is pinned: the scheduler would gather the loads ahead of them and leave the matrix cores idle.
  auto multiply = [&](const Operands &v, auto beside) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < CR; ++r)
#pragma unroll
      for (int o = 0; o < CO; ++o) {
        sum[r][o] = __builtin_amdgcn_mfma_i32_32x32x32_i8(v.w[o], v.x[r], sum[r][o], 0, 0, 0);
        beside(r * CO + o);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  constexpr int M = CR * CO;  // matrix instructions of a step
  // n things spread over a step's first instructions, `many` a time
  auto spread = [&](int i, int n, int many, auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < many; ++q)
      if (i * many + q < n) f(i * many + q);
  };
  // All waves are here; of this one's loads to LDS all but the latest `loads` are done, and of its
  // LDS instructions all but the latest `others`.
  auto meet = [&](auto loads, auto others) __attribute__((always_inline)) {
    wait_for<decltype(loads)::value, decltype(others)::value>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  typedef std::integral_constant<int, 0> none;
  constexpr int kReads = (N + M - 1) / M, kFetches = (2 * P + M - 1) / M;
  Operands u, v;
  if constexpr (!DEEP) {
    // A step's operands are read during the step before.  stage s, NEXT: with another after it,
    // FETCH: with stage s + 2 to be brought.
    auto stage = [&](int s, auto next, auto more) __attribute__((always_inline)) {
      constexpr bool NEXT = decltype(next)::value, FETCH = decltype(more)::value;
      multiply(u, [&](int i) {
        spread(i, N, kReads, [&](int q) { read(s, 1, q, v); });
      });
      multiply(v, [&](int i) {
        spread(i, N, kReads, [&](int q) { read(s, 2, q, u); });
      });
      multiply(u, [&](int i) {
        spread(i, N, kReads, [&](int q) { read(s, 3, q, v); });
        if (!ALIGNED && NEXT) spread(i, 2 * P, kFetches, [&](int p) { put(s + 1, p); });
      });
      // stage s + 1 is there, and nobody reads stage s any more
      if (NEXT) meet(none(), none());
      multiply(v, [&](int i) {
        if (NEXT) spread(i, N, kReads, [&](int q) { read(s + 1, 0, q, u); });
        if (FETCH) spread(i, 2 * P, kFetches, [&](int p) { fetch(s + 2, p); });
      });
    };
    if (whole > 0) {
#pragma unroll
      for (int p = 0; p < 2 * P; ++p) fetch(0, p);
      if (!ALIGNED)
#pragma unroll
        for (int p = 0; p < 2 * P; ++p) put(0, p);
      meet(none(), none());
#pragma unroll
      for (int q = 0; q < N; ++q) read(0, 0, q, u);
      if (whole > 1)
#pragma unroll
        for (int p = 0; p < 2 * P; ++p) fetch(1, p);
      int s = 0;
      for (; s + 2 < whole; ++s) stage(s, std::true_type(), std::true_type());
      if (s + 1 < whole) stage(s++, std::true_type(), std::false_type());
      stage(s, std::false_type(), std::false_type());
    }
  } else {
    // A step has few matrix instructions, too few to cover a read of LDS: operands are read
    // three steps ahead, into four sets, and the meeting of a stage (after its first step) makes
    // the next one readable.  Stages are on their way for two stages: in LDS, or in registers, from
    // where a stage goes to LDS two stages before its use.
    Operands set[4];
    auto stage = [&](int s, auto turn, auto next, auto two, auto three, auto four)
        __attribute__((always_inline)) {
      static_assert(2 * P <= 2 * M, "a stage's chunks go out beside two steps");
      constexpr int h = decltype(turn)::value;
      multiply(set[0], [&](int i) {
        spread(i, N, kReads, [&](int q) { read(s, 3, q, set[3]); });
      });
      if (next) {
        if constexpr (!ALIGNED) {
          meet(std::integral_constant<int, 63>(), std::integral_constant<int, N>());
        } else if (two) {
          meet(std::integral_constant<int, 2 * P>(), std::integral_constant<int, 15>());
        } else {
          meet(none(), std::integral_constant<int, 15>());
        }
      }
#pragma unroll
      for (int step = 1; step < 4; ++step)
        multiply(set[step], [&](int i) {
          if (next)
            spread(i, N, kReads, [&](int q) { read(s + 1, step - 1, q, set[step - 1]); });
          const int p = (step - 1) * M + i;
          if constexpr (ALIGNED) {
            if (three && p < 2 * P) fetch(s + 3, p);
          } else {
            if (two && p < 2 * P) put(s + 2, p, h);
            if (four && p >= M) fetch(s + 4, p - M, h);
          }
        });
    };
    typedef std::integral_constant<int, 0> even;
    typedef std::integral_constant<int, 1> odd;
    typedef std::true_type yes;
    if (whole > 0) {
#pragma unroll
      for (int f = 0; f < 3; ++f) {
        if (f < whole && (ALIGNED || f < 2))
#pragma unroll
          for (int p = 0; p < 2 * P; ++p) fetch(f, p, ALIGNED ? 0 : f);
      }
      if constexpr (ALIGNED) {
        if (whole >= 3) {
          meet(std::integral_constant<int, 4 * P>(), std::integral_constant<int, 15>());
        } else {
          meet(none(), none());
        }
      } else {
#pragma unroll
        for (int f = 0; f < 2; ++f)
          if (f < whole)
#pragma unroll
            for (int p = 0; p < 2 * P; ++p) put(f, p, f);
#pragma unroll
        for (int f = 2; f < 4; ++f)
          if (f < whole)
#pragma unroll
            for (int p = 0; p < 2 * P; ++p) fetch(f, p, f - 2);
        meet(std::integral_constant<int, 63>(), none());
      }
#pragma unroll
      for (int step = 0; step < 3; ++step)
#pragma unroll
        for (int q = 0; q < N; ++q) read(0, step, q, set[step]);
      int s = 0;
      for (; s + 5 < whole; s += 2) {
        stage(s, even(), yes(), yes(), yes(), yes());
        stage(s + 1, odd(), yes(), yes(), yes(), yes());
      }
      for (; s < whole; s += 2) {
        stage(s, even(), s + 1 < whole, s + 2 < whole, s + 3 < whole, s + 4 < whole);
        if (s + 1 < whole)
          stage(s + 1, odd(), s + 2 < whole, s + 3 < whole, s + 4 < whole, s + 5 < whole);
      }
    }
  }
  if (n % kStage) {  // the features past the last whole stage, filled up with zeros
    const int j = whole * kStage + 16 * chunk;
#pragma unroll
    for (int p = 0; p < 2 * P; ++p)
      hold[0][p] = move_down(load_raw(from[p], j, n), j, n);
#pragma unroll
    for (int p = 0; p < 2 * P; ++p) put(whole, p);  // not where the last whole stage is read
    meet(none(), none());
#pragma unroll 1
    for (int step = 0; step < (n % kStage + 31) / 32; ++step) {
#pragma unroll
      for (int q = 0; q < N; ++q) read(whole, step, q, u);
      multiply(u, [](int) {});
    }
  }

  // Lane l holds row l & 31 and outputs 8 (i / 4) + 4 (l >> 5) + i % 4 of each tile.  32 rows of a
  // wave at a time go through LDS, in the type they are stored in, and out as whole runs of a row.
  meet(none(), none());
  float *scales = (float *)smem;  // of the tile's rows, its outputs, and the bias
  for (int i = t; i < B; i += kThreads) {
    scales[i] = r0 + i < a.n_rows ? a.a_scale[r0 + i] : 0.0f;
    scales[B + i] = o0 + i < a.n_outputs ? a.b_scale[o0 + i] : 0.0f;
    scales[2 * B + i] = a.bias && o0 + i < a.n_outputs ? a.bias[o0 + i] : 0.0f;
  }
  meet(none(), none());
  constexpr int kPitch = 32 * CO * (int)sizeof(T) + 16;  // of a row of a wave's outputs, in bytes
  constexpr int kRun = 16 / (int)sizeof(T), kRunsARow = 32 * CO / kRun;
  uint8_t *part = smem + 3 * B * 4 + wave * 32 * kPitch;
  const int row_part = wave / WO * (32 * CR), out_part = wave % WO * (32 * CO);
  const int64_t row_first = r0 + row_part, out_first = o0 + out_part;
#pragma unroll
  for (int r = 0; r < CR; ++r) {
    const float row_scale = scales[row_part + 32 * r + row32];
#pragma unroll
    for (int o = 0; o < CO; ++o)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = 32 * o + 8 * q + 4 * half;
        const float4 scale = *(const float4 *)&scales[B + out_part + at];
        const float4 bias = *(const float4 *)&scales[2 * B + out_part + at];
        const float f[4] = {scale.x, scale.y, scale.z, scale.w};
        const float g[4] = {bias.x, bias.y, bias.z, bias.w};
        T y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float z = (float)sum[r][o][4 * q + i] * row_scale * f[i];
          if (a.bias) z += g[i];
          y[i] = from_float<T>(z);
        }
        __builtin_memcpy(part + row32 * kPitch + at * sizeof(T), y, sizeof(y));
      }
    // only this wave's own part: its LDS instructions are done in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 32 * kRunsARow / 64; ++i) {
      const int at = i * 64 + lane, in_row = at % kRunsARow * kRun;
      const int64_t row = row_first + 32 * r + at / kRunsARow, o = out_first + in_row;
      uint32_t w[4];
      __builtin_memcpy(w, part + at / kRunsARow * kPitch + in_row * sizeof(T), 16);
      if (row < a.n_rows && o < a.n_outputs) {
        const int64_t left = a.n_outputs - o;
        store_packed<T, kRun>((T *)a.out + row * a.ldo + o, left < kRun ? (int)left : kRun, w);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// A workgroup a tile, at most 2^22 of them.  More than 64 KB of LDS are allowed once per kernel
// (each has one size) and device.
static int launch_tiles(void (*k)(MatmulArgs), int64_t tiles, int threads, int lds_bytes,
                        const MatmulArgs &args, void *stream) {
  if (lds_bytes > 65536) {
    constexpr int kMost = 256;
    static std::mutex mu;
    static struct {
      void (*kernel)(MatmulArgs);
      int device;
    } allowed[kMost];
    static int count = 0;
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return (int)e;
    std::lock_guard<std::mutex> lock(mu);
    int at = 0;
    while (at < count && !(allowed[at].kernel == k && allowed[at].device == device)) ++at;
    if (at == count) {
      e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize,
                              lds_bytes);
      if (e != hipSuccess) return (int)e;
      if (count < kMost) allowed[count++] = {k, device};
    }
  }
  return launch(k, tiles, threads, lds_bytes, args, stream);
}

// Whether rows can go to LDS directly: 16-byte chunks, and a tile's offsets below 2^31.
static bool aligned_rows(const MatmulArgs &a) {
  return a.lda <= (1 << 22) && a.ldb <= (1 << 22) &&
         ((uintptr_t)a.a | (uintptr_t)a.b | (uint64_t)a.lda | (uint64_t)a.ldb) % 16 ==
             0;
}
template <typename T, int R, int O, int W, int S>
static int launch_stream(const MatmulArgs &a, void *stream) {
  const int64_t tiles = ((a.n_rows + 16 * R - 1) / (16 * R)) *
                        (((int64_t)a.n_outputs + 16 * O - 1) / (16 * O));
  constexpr int kSums = W * R * O * 1024, kPart = W * (R + O) * 1024;
  constexpr int kAligned = S * kPart > kSums ? S * kPart : kSums;
  constexpr int kOther = kPart > kSums ? kPart : kSums;
  return aligned_rows(a)
             ? launch_tiles(matmul_q8_stream_kernel<T, R, O, W, S, true>, tiles, 64 * W, kAligned, a,
                            stream)
             : launch_tiles(matmul_q8_stream_kernel<T, R, O, W, S, false>, tiles, 64 * W, kOther, a,
                            stream);
}
template <typename T, int B, int WO, bool DEEP>
static int launch_tile(const MatmulArgs &a, void *stream) {
  const int64_t tiles =
      ((a.n_rows + B - 1) / B) * (((int64_t)a.n_outputs + B - 1) / B);
  constexpr int kLds = kTileLds<B, DEEP>;
  return launch_tiles(aligned_rows(a) ? matmul_q8_tile_kernel<T, B, WO, DEEP, true>
                                      : matmul_q8_tile_kernel<T, B, WO, DEEP, false>,
                      tiles, 128 * WO, kLds, a, stream);
}

// Which kernel runs, by an estimate of each one's time in us on 256 CUs.  A streamed tile of 16 R
// rows by 16 O outputs takes its CU 1 us for 36 KB of rows and weights (28 KB where they pass
// through registers), no less than 0.36 us for a wave's stage, 0.2 us to begin, and 0.5 us to join
// 16 tiles of 16 x 16; more than two tiles a CU even out.  A stage of a 256 x 256 tile takes 1.1
// us, 1.7 where all CUs compute (the clock falls), of a 128 x 128 tile with four stages in LDS and
// one workgroup a CU 0.5, and 0.8 where all compute, and 0.7 for each of two workgroups a CU with
// two stages; rows through registers take 1.35 to 1.5 times as long.  No kernel is faster than
// memory.  Over 132 sizes (1 to 100,000 rows, 10 to 36,601 outputs, 64 to 16,256 features; two
// measurements of each, averaged) the choice takes 4% longer than the fastest of nine kernels on
// average, and 22% at most; 2% and 22% over the 61 sizes of 8 us or more.  Sides, us: 1 x
// 32000 x 4096 16 x 16 tiles 25, 16 x 32 26.3; 16 x 32000 x 4096 16 x 32 30.4, 16 x 16 32.9; 32 x
// 4096 x 4096 16 x 32 5.5, 32 x 32 6.9; 32 x 32000 x 4096 32 x 64 31.4, 64 x 64 32.8, 32 x 32 36;
// 64 x 4096 x 4096 32 x 32 6.6, 64 x 32 8; 128 x 4096 x 4096 64 x 32 8.6, 64 x 64 12.2; 256 x 4096
// x 4096 64 x 64 12.8, 128 x 128 14.9; 512 x 4096 x 4096 20.8 against 16.0; 2048 x 4096 x 4096 128
// x 128 38.6 with two workgroups a CU, 41.3 with one, 256 x 256 45.3; 8192 x 8192 x 1024 91.5
// against 85.8.  Rings of more stages, which leave room for fewer workgroups a CU, take longer (16
// x 4096 x 11,008 16 x 16 tiles with three stages 14.1, four 15.4; 32 x 4096 x 11,008 16 x 32 with
// two 15.8, four 18.7).
struct Estimate {
  const MatmulArgs &a;
  bool aligned;
  double memory, least = 1e30;
  int best = 0;

  explicit Estimate(const MatmulArgs &a) : a(a), aligned(aligned_rows(a)) {
    memory = ((double)a.n_rows * a.n_features + (double)a.n_outputs * a.n_features +
              2.0 * (double)a.n_rows * a.n_outputs) / 4.9e6;
  }
  double tiles(int rows, int outputs) const {
    return (double)((a.n_rows + rows - 1) / rows) *
           (double)(((int64_t)a.n_outputs + outputs - 1) / outputs);
  }
  void take(int kernel, double us, double after = 0.0) {
    us = (us > memory ? us : memory) + after;
    if (us < least) least = us, best = kernel;
  }
  void stream(int kernel, int R, int O, int W) {
    const double n = tiles(16 * R, 16 * O), rounds = n > 512 ? n / 256 : __builtin_ceil(n / 256);
    const double rows = a.n_rows < 16 * R ? (double)a.n_rows : 16 * R;
    const double moved = rounds * (rows + 16 * O) * a.n_features / (aligned ? 36e3 : 28e3);
    const double stages = (a.n_features + 64 * W - 1) / (64 * W) * 0.36;
    take(kernel, (moved > stages ? moved : stages) + 0.2 * rounds, 0.5 * rounds * R * O / 16);
  }
  void tile(int kernel, int B, bool deep) {
    const double n = tiles(B, B), rounds = __builtin_ceil(n / 256), busy = n < 256 ? n / 256 : 1.0;
    const double stages = (a.n_features + kStage - 1) / kStage;
    // the last stage moves the 16 bytes that end a row; few rows waste most of a tile (1 x 32000 x
    // 4096: 32 us against 28)
    if (a.n_features < 16 || a.n_rows < 48) return;
    if (B == 256) {
      take(kernel, rounds * (stages * (1.1 + 0.6 * busy) * (aligned ? 1.0 : 1.35) + 3.0));
    } else if (deep) {
      take(kernel, rounds * (stages * (0.5 + 0.3 * busy) * (aligned ? 1.0 : 1.4) + 1.0));
    } else if (n >= 256) {
      take(kernel, n / 256 * stages * 0.7 * (aligned ? 1.0 : 1.5));
    }
  }
};

static int launch_part(const MatmulArgs &a, int32_t dtype, void *stream) {
  Estimate e(a);
  e.stream(0, 1, 1, 8);
  e.stream(1, 1, 2, 8);
  e.stream(2, 2, 2, 8);
  e.stream(3, 4, 2, 4);
  e.stream(4, 4, 4, 4);
  e.stream(5, 2, 4, 8);
  e.tile(6, 128, false);
  e.tile(7, 256, false);
  e.tile(8, 128, true);
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    switch (e.best) {
      case 0: return launch_stream<T, 1, 1, 8, 3>(a, stream);
      case 1: return launch_stream<T, 1, 2, 8, 2>(a, stream);
      case 2: return launch_stream<T, 2, 2, 8, 2>(a, stream);
      case 3: return launch_stream<T, 4, 2, 4, 3>(a, stream);
      case 4: return launch_stream<T, 4, 4, 4, 2>(a, stream);
      case 5: return launch_stream<T, 2, 4, 8, 2>(a, stream);
      case 6: return launch_tile<T, 128, 4, false>(a, stream);
      case 7: return launch_tile<T, 256, 4, false>(a, stream);
      default: return launch_tile<T, 128, 4, true>(a, stream);
    }
  });
}

// A dispatch counts its work-items in 32 bits: no more than 2^22 tiles of 16 x 16 a launch.
int launch_matmul_q8(const MatmulArgs &a, int32_t dtype, void *stream) {
  constexpr int64_t kOutputs = int64_t(1) << 20, kSums = int64_t(1) << 30;
  const int64_t outputs = a.n_outputs < kOutputs ? a.n_outputs : kOutputs;
  const int64_t rows = kSums / ((outputs + 255) / 256 * 256) / 256 * 256;
  const int size = dtype == BRIDGER_F32 ? 4 : 2;
  for (int64_t o = 0; o < a.n_outputs; o += outputs)
    for (int64_t r = 0; r < a.n_rows; r += rows) {
      MatmulArgs part = a;
      part.a += r * a.lda;
      part.a_scale += r;
      part.b += o * a.ldb;
      part.b_scale += o;
      if (a.bias) part.bias += o;
      part.out = (uint8_t *)a.out + (r * a.ldo + o) * size;
      part.n_rows = a.n_rows - r < rows ? a.n_rows - r : rows;
      part.n_outputs = (int32_t)(a.n_outputs - o < outputs ? a.n_outputs - o : outputs);
      const int err = launch_part(part, dtype, stream);
      if (err) return err;
    }
  return 0;
}

}  // namespace bridger
