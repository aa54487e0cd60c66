// dropout.hip -- gfx950 kernels of bridger_dropout.
#include "rows.h"

namespace bridger {

// Philox4x32-10: ten rounds of two products and exclusive ors that turn a counter of four words and
// a key of two into four random words (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy
// as 1, 2, 3; 2011).
struct Words {
  uint32_t w[4];
};
__device__ inline Words random_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3,
                                     uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

constexpr int kUnit = 8;  // elements of a row that share a block of words

// A lane takes the kUnit elements from j on.  An element's 32 random bits are compared with
// p 2^32: the upper 16 decide but for one in 65536, so that one block of words serves kUnit elements;
// the lower 16 come from another block, which is made where some element needs it: ten rounds for 8
// elements leave memory as the bound.  8192 x 8192 bfloat16 with a residual 69 us (5.8 TB/s, part of what
// is written stays in the last cache), 100,000 x 347 float 54 to 56 (5.0 TB/s).
template <typename T, int G>
__global__ __launch_bounds__(kRowThreads<G>) void dropout_kernel(DropoutArgs a) {
  constexpr int V = kPerLoad<T>, L = kUnit / V;
  const int64_t b = a.first + blockIdx.x;
  int64_t block = b;
  int tile = 0;
  if (a.tiles > 1) {
    block = b / a.tiles;
    tile = (int)(b - block * a.tiles);
  }
  const int64_t row = block * kRowsAWorkgroup<G> + threadIdx.x / G;
  const int n = a.n_features;
  const int64_t unit = (int64_t)tile * G + threadIdx.x % G;
  if (row >= a.n_rows || unit * kUnit >= n) return;
  const int j = (int)unit * kUnit;
  const T *x = (const T *)a.x + row * a.ldx;
  const T *res = a.residual ? (const T *)a.residual + row * a.ldr : nullptr;
  RowLoad<T> xl[L], rl[L];
  if (n < V) {
    xl[0].tiny(x, 0, n, (T)0.0f);
    if (res) rl[0].tiny(res, 0, n, (T)0.0f);
  } else {
#pragma unroll
    for (int l = 0; l < L; ++l) {
      xl[l].issue(x, j + l * V, n);
      if (res) rl[l].issue(res, j + l * V, n);
    }
  }
  const uint32_t k0 = (uint32_t)a.seed[0], k1 = (uint32_t)((uint64_t)a.seed[0] >> 32);
  const uint32_t step = (uint32_t)a.seed[1];
  const Words r = random_words((uint32_t)unit, (uint32_t)row, step, 2 * a.layer, k0, k1);
  const uint32_t high = (uint32_t)(a.limit >> 16), low = (uint32_t)a.limit & 0xFFFFu;
  uint32_t keep = 0, tie = 0;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) {
    const uint32_t h = i & 1 ? r.w[i >> 1] >> 16 : r.w[i >> 1] & 0xFFFFu;
    keep |= (uint32_t)(h >= high) << i;
    tie |= (uint32_t)(h == high) << i;
  }
  if (tie && low) {
    const Words q = random_words((uint32_t)unit, (uint32_t)row, step, 2 * a.layer + 1, k0, k1);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) {
      const uint32_t h = i & 1 ? q.w[i >> 1] >> 16 : q.w[i >> 1] & 0xFFFFu;
      if (h < low) keep &= ~(tie & 1u << i);
    }
  }
  T *out = (T *)a.out + row * a.ldo;
#pragma unroll
  for (int l = 0; l < L; ++l) {
    const int at = j + l * V;
    if (at >= n) return;
    if (n >= V) {
      xl[l].take(at, n, 0);
      if (res) rl[l].take(at, n, 0);
    }
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = keep >> (l * V + i) & 1 ? element<T>(xl[l].raw, i) * a.scale : 0.0f;
      if (res) v[i] += element<T>(rl[l].raw, i);
    }
    store16<T>(out + at, n - at, v);
  }
}

int launch_dropout(const DropoutArgs &args, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    DropoutArgs a = args;
    const int64_t units = ((int64_t)a.n_features + kUnit - 1) / kUnit;
    auto of = [&](auto k, int lanes) {
      a.tiles = (int)((units + lanes - 1) / lanes);
      const int64_t rows = 256 / lanes;
      return launch_blocks(k, (a.n_rows + rows - 1) / rows * a.tiles, 256, a, stream);
    };
    if (units <= 1) return of(dropout_kernel<T, 1>, 1);
    if (units <= 4) return of(dropout_kernel<T, 4>, 4);
    if (units <= 16) return of(dropout_kernel<T, 16>, 16);
    if (units <= 64) return of(dropout_kernel<T, 64>, 64);
    return of(dropout_kernel<T, 256>, 256);
  });
}

}  // namespace bridger
