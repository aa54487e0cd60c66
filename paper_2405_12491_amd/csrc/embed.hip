// embed.hip -- gfx950 kernels of bridger_embed and bridger_embed_backward.
#include <type_traits>

#include "rows.h"

namespace bridger {

// W neighbouring elements of a row: 16 bytes, or one element where a row has less than 16 bytes.
template <typename T, int W>
struct Elements {
  u32x4 raw;
  T one;
  __device__ void load(const T *p) {
    if constexpr (W == 1) {
      one = *p;
    } else {
      __builtin_memcpy(&raw, p, 16);
    }
  }
  __device__ float at(int i) const {
    if constexpr (W == 1) {
      return to_float(one);
    } else {
      return element<T>(raw, i);
    }
  }
};
template <typename T, int W>
__device__ inline void store_elements(T *p, const float (&v)[W]) {
  if constexpr (W == 1) {
    *p = from_float<T>(v[0]);
  } else {
    store16<T>(p, W, v);
  }
}

// The entry that slot s of a row reads, or -1.
__device__ inline int32_t entry_of(const EmbedArgs &a, int64_t row, int s) {
  const int32_t id = a.ids[row * a.ldi + s];
  int64_t begin = 0, end = a.n_entries;
  if (a.offsets) {
    begin = a.offsets[s];
    const int64_t stop = a.offsets[s + 1];
    end = stop < end ? stop : end;
  }
  return id >= 0 && begin >= 0 && begin < end && id < end - begin ? (int32_t)(begin + id) : -1;
}

// A row's features are parted into tiles of G lanes with W elements each; the last lane of a row
// takes the W elements that end it, so that no load or store is partial (what two lanes hold of a
// row is the same, and no output lies on an input).
struct Place {
  int64_t block;  // the workgroup's number among those of its tile
  int column;     // the lane's first element
  bool inside;
};
template <int G, int W>
__device__ inline Place place_of(const EmbedArgs &a, int64_t first) {
  const int64_t b = first + blockIdx.x;
  int64_t block = b;
  int tile = 0;
  if (a.tiles > 1) {
    block = b / a.tiles;
    tile = (int)(b - block * a.tiles);
  }
  const int64_t j = ((int64_t)tile * G + threadIdx.x % G) * W;
  const int last = a.n_features - W;
  return {block, (int)(j < last ? j : last), j < a.n_features};
}

constexpr int kThreads = 256;
constexpr int kAhead = 8;  // loads that a lane has on their way

// One slot a row: G lanes copy kAhead rows at a time.
template <typename T, int G, int W>
__global__ __launch_bounds__(kThreads) void embed_rows_kernel(EmbedArgs a) {
  constexpr int groups = kThreads / G;
  const Place p = place_of<G, W>(a, a.first);
  if (!p.inside) return;
  const T *table = (const T *)a.table + p.column;
  T *out = (T *)a.out + p.column;
  const int64_t row0 = p.block * (groups * kAhead) + threadIdx.x / G;
  int32_t at[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t row = row0 + u * groups;
    at[u] = row < a.n_rows ? entry_of(a, row, 0) : -1;
  }
  Elements<T, W> e[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) e[u].load(table + (at[u] < 0 ? 0 : at[u]) * a.ldt);
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t row = row0 + u * groups;
    float v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = at[u] < 0 ? 0.0f : e[u].at(i) * a.scale;
    if (row < a.n_rows) store_elements<T, W>(out + row * a.ldo, v);
  }
}

// Several slots a row: a.parts groups of G lanes share a row's slots and join in LDS.
template <typename T, int G, int W>
__global__ __launch_bounds__(kThreads) void embed_bag_kernel(EmbedArgs a) {
  constexpr int groups = kThreads / G;
  __shared__ float join[kThreads * W];
  const Place p = place_of<G, W>(a, a.first);
  const int group = threadIdx.x / G, part = group & (a.parts - 1);
  const int64_t wanted = p.block * (groups / a.parts) + group / a.parts;
  const int64_t row = wanted < a.n_rows ? wanted : a.n_rows - 1;
  const T *table = (const T *)a.table + p.column;
  float sum[W];
#pragma unroll
  for (int i = 0; i < W; ++i) sum[i] = 0.0f;
  for (int64_t s0 = part * kAhead; s0 < a.n_slots; s0 += (int64_t)a.parts * kAhead) {
    int32_t at[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      at[u] = s0 + u < a.n_slots ? entry_of(a, row, (int)(s0 + u)) : -1;
    Elements<T, W> e[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) e[u].load(table + (at[u] < 0 ? 0 : at[u]) * a.ldt);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int i = 0; i < W; ++i) sum[i] += at[u] < 0 ? 0.0f : e[u].at(i);
  }
  if (a.parts > 1) {  // of the whole workgroup
#pragma unroll
    for (int i = 0; i < W; ++i) join[i * kThreads + threadIdx.x] = sum[i];
    __syncthreads();
    for (int q = 1; part == 0 && q < a.parts; ++q)
#pragma unroll
      for (int i = 0; i < W; ++i) sum[i] += join[i * kThreads + threadIdx.x + q * G];
  }
  if (part || !p.inside || wanted >= a.n_rows) return;
#pragma unroll
  for (int i = 0; i < W; ++i) sum[i] *= a.scale;
  store_elements<T, W>((T *)a.out + row * a.ldo + p.column, sum);
}

// Calls f(lanes, elements a lane) as types, for rows of `width` elements of T.
template <typename T, typename F>
int with_lanes(int width, F f) {
  constexpr int V = kPerLoad<T>;
  using std::integral_constant;
  if (width < V) return f(integral_constant<int, 8>(), integral_constant<int, 1>());
  const int lanes = (width + V - 1) / V;
  if (lanes <= 4) return f(integral_constant<int, 4>(), integral_constant<int, V>());
  if (lanes <= 8) return f(integral_constant<int, 8>(), integral_constant<int, V>());
  if (lanes <= 16) return f(integral_constant<int, 16>(), integral_constant<int, V>());
  if (lanes <= 32) return f(integral_constant<int, 32>(), integral_constant<int, V>());
  return f(integral_constant<int, 64>(), integral_constant<int, V>());
}
int tiles_of(int width, int lanes, int elements) {
  const int64_t tile = (int64_t)lanes * elements;
  return (int)((width + tile - 1) / tile);
}

int launch_embed(const EmbedArgs &args, int32_t dtype, void *stream) {
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(args.n_features, [&](auto lanes, auto elements) {
      constexpr int G = decltype(lanes)::value, W = decltype(elements)::value;
      constexpr int groups = kThreads / G;
      EmbedArgs a = args;
      a.tiles = tiles_of(a.n_features, G, W);
      if (a.n_slots == 1) {
        const int64_t rows = groups * kAhead;
        return launch_blocks(embed_rows_kernel<T, G, W>, (a.n_rows + rows - 1) / rows * a.tiles,
                             kThreads, a, stream);
      }
      // groups share a row's slots while rows alone leave compute units idle
      a.parts = 1;
      while (a.parts < groups && a.n_rows * a.tiles * a.parts < 2048 * groups &&
             a.parts * kAhead < a.n_slots)
        a.parts *= 2;
      const int64_t rows = groups / a.parts;
      return launch_blocks(embed_bag_kernel<T, G, W>, (a.n_rows + rows - 1) / rows * a.tiles,
                           kThreads, a, stream);
    });
  });
}

// ============================================================================== BACKWARD
// Pairs (entry, row), one a slot, are sorted by entry: a radix sort whose passes keep the order of
// equal keys, so that an entry's rows stand in the order of their slots.  Then groups of lanes add
// an entry's rows.  Empty slots have the key n_entries and end up behind all others.
constexpr int kTile = 4096;     // pairs that a workgroup sorts at once
constexpr int kMaxDigit = 11;   // bits a pass
constexpr int kChunk = 64;      // pairs that are added beforehand where they belong to one entry

struct SortPlan {
  int passes, bits;  // of one digit
  int64_t pairs, tiles, chunks, supers;
};
static SortPlan plan_of(int64_t pairs, int32_t n_entries) {
  SortPlan p;
  int bits = 0;
  while ((int64_t)n_entries >> bits) ++bits;  // the largest key is n_entries
  p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.pairs = pairs;
  p.tiles = (pairs + kTile - 1) / kTile;
  p.chunks = pairs / kChunk;
  p.supers = p.chunks / kChunk;
  return p;
}

struct GradArgs {
  EmbedArgs e;
  int64_t pairs, tiles;
  const uint32_t *keys, *rows;  // sorted so far; null: the slots themselves
  uint32_t *keys_to, *rows_to;
  uint32_t *counts;  // [digit values][tiles]
  uint32_t *totals;  // [digit values]
  float *chunk, *super;  // sums of whole chunks, and of kChunk chunks, that belong to one entry
  int64_t chunks, supers;
  int shift, bits;
  int each;       // entries of a group
  int64_t first;  // the launch's first workgroup
};

struct Pair {
  uint32_t key, row;
};
__device__ inline Pair pair_of(const GradArgs &a, int64_t i) {
  if (a.keys) return {a.keys[i], a.rows[i]};
  uint32_t row = (uint32_t)i, s = 0;
  if (a.e.n_slots > 1) {
    row = (uint32_t)i / (uint32_t)a.e.n_slots;
    s = (uint32_t)i - row * (uint32_t)a.e.n_slots;
  }
  const int32_t at = entry_of(a.e, row, (int)s);
  return {at < 0 ? (uint32_t)a.e.n_entries : (uint32_t)at, row};
}
__device__ inline uint32_t digit_of(const GradArgs &a, uint32_t key) {
  return key >> a.shift & ((1u << a.bits) - 1);
}

// How many of a tile's pairs have each digit.
__global__ __launch_bounds__(kThreads) void embed_count_kernel(GradArgs a) {
  __shared__ uint32_t count[1 << kMaxDigit];
  const int values = 1 << a.bits;
  for (int d = threadIdx.x; d < values; d += kThreads) count[d] = 0;
  __syncthreads();
  const int64_t tile = a.first + blockIdx.x, begin = tile * kTile;
#pragma unroll
  for (int u = 0; u < kTile / kThreads; ++u) {
    const int64_t i = begin + u * kThreads + threadIdx.x;
    if (i < a.pairs) atomicAdd(&count[digit_of(a, pair_of(a, i).key)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < values; d += kThreads) a.counts[d * a.tiles + tile] = count[d];
}

// The sum of v over the lanes below this one, and over all.
__device__ inline uint32_t lanes_before(uint32_t v, uint32_t *all) {
  const int lane = threadIdx.x & 63;
  uint32_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t other = __shfl_up(sum, d, 64);
    if (lane >= d) sum += other;
  }
  *all = __shfl(sum, 63, 64);
  return sum - v;
}

// Per digit: its count in every tile becomes that of the tiles before.  A wave a digit.
__global__ __launch_bounds__(kThreads) void embed_scan_kernel(GradArgs a) {
  const int d = blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  if (d >= 1 << a.bits) return;
  uint32_t *count = a.counts + d * a.tiles;
  uint32_t before = 0;
  for (int64_t t0 = 0; t0 < a.tiles; t0 += 256) {
    const int64_t t = t0 + (threadIdx.x & 63) * 4;
    uint32_t c[4], all;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = t + i < a.tiles ? count[t + i] : 0;
    uint32_t at = before + lanes_before(c[0] + c[1] + c[2] + c[3], &all);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (t + i < a.tiles) count[t + i] = at;
      at += c[i];
    }
    before += all;
  }
  if ((threadIdx.x & 63) == 0) a.totals[d] = before;
}

// Lanes of the wave whose digit is this lane's (`live` lanes only).
__device__ inline uint64_t lanes_alike(uint32_t digit, int bits, bool live) {
  uint64_t same = __ballot(live);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  return same;
}

// Moves a tile's pairs to their places.  Every wave has a run of the tile's pairs and, for each
// digit, the place of its next pair: those of smaller digits, of the tiles before, of the waves
// before, and its own so far.
__global__ __launch_bounds__(kThreads) void embed_move_kernel(GradArgs a) {
  constexpr int waves = kThreads / 64, rounds = kTile / kThreads;
  __shared__ uint32_t next[waves][1 << kMaxDigit];
  __shared__ uint32_t wave_sum[waves];
  const int values = 1 << a.bits, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int64_t tile = a.first + blockIdx.x;
  const int64_t begin = tile * kTile + wave * (rounds * 64) + lane;
  for (int d = threadIdx.x; d < values; d += kThreads)
#pragma unroll
    for (int w = 0; w < waves; ++w) next[w][d] = 0;
  Pair p[rounds];
#pragma unroll
  for (int u = 0; u < rounds; ++u) {
    const int64_t i = begin + u * 64;
    p[u] = i < a.pairs ? pair_of(a, i) : Pair{0, 0};
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < rounds; ++u)
    if (begin + u * 64 < a.pairs) atomicAdd(&next[wave][digit_of(a, p[u].key)], 1u);
  // each thread takes a run of digits
  constexpr int run = (1 << kMaxDigit) / kThreads;
  const int d0 = threadIdx.x * run;
  uint32_t own = 0, all;
  for (int i = 0; i < run; ++i) own += d0 + i < values ? a.totals[d0 + i] : 0;
  uint32_t before = lanes_before(own, &all);
  if (lane == 0) wave_sum[wave] = all;
  __syncthreads();
  for (int w = 0; w < wave; ++w) before += wave_sum[w];
  for (int i = 0; i < run && d0 + i < values; ++i) {
    const int d = d0 + i;
    uint32_t at = before + a.counts[d * a.tiles + tile];
#pragma unroll
    for (int w = 0; w < waves; ++w) {
      const uint32_t c = next[w][d];
      next[w][d] = at;
      at += c;
    }
    before += a.totals[d];
  }
  __syncthreads();
  volatile uint32_t *mine = next[wave];
#pragma unroll
  for (int u = 0; u < rounds; ++u) {
    const bool live = begin + u * 64 < a.pairs;
    const uint32_t d = digit_of(a, p[u].key);
    const uint64_t same = lanes_alike(d, a.bits, live);
    const int earlier = __popcll(same & ((uint64_t(1) << lane) - 1));
    if (live) {
      const uint32_t at = mine[d];
      // the wave's lanes have all read it; the first of those alike moves it on
      __builtin_amdgcn_wave_barrier();
      if (earlier == 0) mine[d] = at + __popcll(same);
      __builtin_amdgcn_wave_barrier();
      a.keys_to[at + earlier] = p[u].key;
      a.rows_to[at + earlier] = p[u].row;
    }
  }
}

// The first pair whose key reaches `key`, found by all lanes of a wave together.
__device__ inline int64_t first_pair(const uint32_t *keys, int64_t n, uint32_t key) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t step = (hi - lo + 63) / 64, i = lo + (threadIdx.x & 63) * step;
    const int below = __popcll(__ballot(i < hi && keys[i < hi ? i : lo] < key));
    if (below == 0) {
      hi = lo;
    } else {
      const int64_t end = lo + below * step;
      lo = end - step + 1;
      hi = end < hi ? end : hi;
    }
  }
  return lo;
}

// sum += rows [i, end) of `width` floats apart, from their first element `p`.
template <int W>
__device__ inline void add_sums(float (&sum)[W], const float *p, int64_t width, int64_t i,
                                int64_t end) {
  for (; i < end; i += kAhead) {
    float v[kAhead][W];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      __builtin_memcpy(v[u], p + (i + u < end ? i + u : i) * width, sizeof(v[u]));
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int k = 0; k < W; ++k) sum[k] += i + u < end ? v[u][k] : 0.0f;
  }
}
template <typename T, int W>
__device__ inline void add_rows(float (&sum)[W], const GradArgs &a, const T *grad, int64_t i,
                                int64_t end) {
  for (; i < end; i += kAhead) {
    uint32_t row[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) row[u] = a.rows[i + u < end ? i + u : i];
    Elements<T, W> e[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) e[u].load(grad + (int64_t)row[u] * a.e.ldt);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int k = 0; k < W; ++k) sum[k] += i + u < end ? e[u].at(k) : 0.0f;
  }
}

// Sums of the chunks whose pairs all belong to one entry, for entries with many rows.
template <typename T, int G, int W>
__global__ __launch_bounds__(kThreads) void embed_chunk_kernel(GradArgs a) {
  const Place p = place_of<G, W>(a.e, a.first);
  const int64_t c = p.block * (kThreads / G) + threadIdx.x / G;
  if (c >= a.chunks || !p.inside) return;
  const uint32_t key = a.keys[c * kChunk];
  if (key != a.keys[c * kChunk + kChunk - 1] || key >= (uint32_t)a.e.n_entries) return;
  float sum[W];
#pragma unroll
  for (int k = 0; k < W; ++k) sum[k] = 0.0f;
  add_rows<T, W>(sum, a, (const T *)a.e.table + p.column, c * kChunk, (c + 1) * kChunk);
  __builtin_memcpy(a.chunk + c * a.e.n_features + p.column, sum, sizeof(sum));
}
template <int G, int W>
__global__ __launch_bounds__(kThreads) void embed_super_kernel(GradArgs a) {
  constexpr int64_t pairs = kChunk * kChunk;
  const Place p = place_of<G, W>(a.e, a.first);
  const int64_t c = p.block * (kThreads / G) + threadIdx.x / G;
  if (c >= a.supers || !p.inside) return;
  const uint32_t key = a.keys[c * pairs];
  if (key != a.keys[c * pairs + pairs - 1] || key >= (uint32_t)a.e.n_entries) return;
  float sum[W];
#pragma unroll
  for (int k = 0; k < W; ++k) sum[k] = 0.0f;
  add_sums<W>(sum, a.chunk + p.column, a.e.n_features, c * kChunk, (c + 1) * kChunk);
  __builtin_memcpy(a.super + c * a.e.n_features + p.column, sum, sizeof(sum));
}

// A workgroup's groups of lanes take a.each entries each: rows up to the first whole chunk, chunks
// up to the first whole super chunk, those, and the rest likewise.
constexpr int kMostEntries = kThreads;
template <typename T, int G, int W>
__global__ __launch_bounds__(kThreads) void embed_entries_kernel(GradArgs a) {
  constexpr int groups = kThreads / G;
  __shared__ int64_t bound[2];
  __shared__ uint32_t start[kMostEntries + 1];
  const Place p = place_of<G, W>(a.e, a.first);
  const int n = groups * a.each;
  const int64_t e0 = p.block * n;
  const int64_t e1 = e0 + n < a.e.n_entries ? e0 + n : a.e.n_entries;
  if (threadIdx.x < 128) {
    const int64_t at =
        first_pair(a.keys, a.pairs, (uint32_t)(threadIdx.x < 64 ? e0 : e1));
    if ((threadIdx.x & 63) == 0) bound[threadIdx.x / 64] = at;
  }
  __syncthreads();
  for (int t = threadIdx.x; t <= e1 - e0; t += kThreads) {
    int64_t lo = bound[0], hi = bound[1];
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (a.keys[mid] < (uint32_t)(e0 + t)) {
        lo = mid + 1;
      } else {
        hi = mid;
      }
    }
    start[t] = (uint32_t)lo;
  }
  __syncthreads();
  if (!p.inside) return;
  const T *grad = (const T *)a.e.table + p.column;
  T *out = (T *)a.e.out + p.column;
  const int width = a.e.n_features;
  for (int t = threadIdx.x / G; t < e1 - e0; t += groups) {
    float sum[W];
#pragma unroll
    for (int k = 0; k < W; ++k) sum[k] = 0.0f;
    const int64_t i0 = start[t], i1 = start[t + 1];
    const int64_t c0 = (i0 + kChunk - 1) / kChunk, c1 = i1 / kChunk;  // whole chunks
    if (c0 >= c1) {
      add_rows<T, W>(sum, a, grad, i0, i1);
    } else {
      add_rows<T, W>(sum, a, grad, i0, c0 * kChunk);
      const int64_t s0 = (c0 + kChunk - 1) / kChunk, s1 = c1 / kChunk;
      const float *chunk = a.chunk + p.column;
      if (s0 >= s1) {
        add_sums<W>(sum, chunk, width, c0, c1);
      } else {
        add_sums<W>(sum, chunk, width, c0, s0 * kChunk);
        add_sums<W>(sum, a.super + p.column, width, s0, s1);
        add_sums<W>(sum, chunk, width, s1 * kChunk, c1);
      }
      add_rows<T, W>(sum, a, grad, c1 * kChunk, i1);
    }
#pragma unroll
    for (int k = 0; k < W; ++k) sum[k] *= a.e.scale;
    store_elements<T, W>(out + (e0 + t) * a.e.ldo, sum);
  }
}

// The workspace's parts, each from a multiple of 16 bytes.
struct Parts {
  int64_t keys[2], rows[2], counts, totals, chunk, super, bytes;
};
static Parts parts_of(const SortPlan &p, int64_t width) {
  Parts w;
  int64_t at = 0;
  auto take = [&](int64_t words) {
    const int64_t begin = at;
    at += (words * 4 + 15) / 16 * 16;
    return begin;
  };
  for (int i = 0; i < 2; ++i) w.keys[i] = take(p.pairs), w.rows[i] = take(p.pairs);
  w.counts = take(p.tiles << p.bits);
  w.totals = take(int64_t(1) << p.bits);
  w.chunk = take(p.chunks * width);
  w.super = take(p.supers * width);
  w.bytes = at;
  return w;
}

int64_t embed_backward_bytes(int64_t n_rows, int32_t n_slots, int32_t n_entries,
                             int32_t n_features) {
  return parts_of(plan_of(n_rows * n_slots, n_entries), n_features).bytes;
}

int launch_embed_backward(const EmbedArgs &args, int32_t dtype, void *stream) {
  const SortPlan plan = plan_of(args.n_rows * args.n_slots, args.n_entries);
  const Parts parts = parts_of(plan, args.n_features);
  char *ws = (char *)args.workspace;
  uint32_t *keys[2], *rows[2];
  for (int i = 0; i < 2; ++i) {
    keys[i] = (uint32_t *)(ws + parts.keys[i]);
    rows[i] = (uint32_t *)(ws + parts.rows[i]);
  }
  GradArgs a = {};
  a.e = args;
  a.pairs = plan.pairs;
  a.tiles = plan.tiles;
  a.counts = (uint32_t *)(ws + parts.counts);
  a.totals = (uint32_t *)(ws + parts.totals);
  a.chunk = (float *)(ws + parts.chunk);
  a.super = (float *)(ws + parts.super);
  a.chunks = plan.chunks;
  a.supers = plan.supers;
  a.bits = plan.bits;
  int err = 0;
  for (int pass = 0; pass < plan.passes && plan.pairs; ++pass) {
    a.shift = pass * plan.bits;
    a.keys_to = keys[pass & 1];
    a.rows_to = rows[pass & 1];
    err = launch_blocks(embed_count_kernel, a.tiles, kThreads, a, stream);
    if (!err) {
      const int waves = kThreads / 64;
      err = launch(embed_scan_kernel, ((1 << a.bits) + waves - 1) / waves, kThreads, 0, a, stream);
    }
    if (!err) err = launch_blocks(embed_move_kernel, a.tiles, kThreads, a, stream);
    if (err) return err;
    a.keys = a.keys_to;
    a.rows = a.rows_to;
  }
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(args.n_features, [&](auto lanes, auto elements) {
      constexpr int G = decltype(lanes)::value, W = decltype(elements)::value;
      constexpr int groups = kThreads / G;
      GradArgs g = a;
      g.e.tiles = tiles_of(g.e.n_features, G, W);
      int e = 0;
      auto blocks = [&](int64_t n) { return (n + groups - 1) / groups * g.e.tiles; };
      if (g.chunks) e = launch_blocks(embed_chunk_kernel<T, G, W>, blocks(g.chunks), kThreads, g, stream);
      if (!e && g.supers)
        e = launch_blocks(embed_super_kernel<G, W>, blocks(g.supers), kThreads, g, stream);
      if (e) return e;
      // several entries a group where the chip is full without
      g.each = 1;
      while (g.each * groups < 64 && (int64_t)g.e.n_entries * g.e.tiles > (int64_t)g.each * groups * 4096)
        g.each *= 2;
      const int64_t n = groups * g.each;
      return launch_blocks(embed_entries_kernel<T, G, W>, (g.e.n_entries + n - 1) / n * g.e.tiles,
                           kThreads, g, stream);
    });
  });
}

}  // namespace bridger
