// embed.hip -- gfx950 kernels of bridger_embed and bridger_embed_backward.
#include <type_traits>

#include "rows.h"

namespace bridger {

// W neighbouring elements of a row: 16 bytes, or one element where a row has less than 16 bytes.
template <typename T, int W>
struct Elements {
  u32x4 raw;
  T one;
  __device__ void clear() {
    raw = u32x4{0, 0, 0, 0};
    one = (T)0.0f;
  }
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

// The entry that slot s reads where it holds `id`, or -1.
__device__ inline int32_t entry_at(const EmbedArgs &a, int32_t id, int s) {
  if (!a.offsets) return (uint32_t)id < (uint32_t)a.n_entries ? id : -1;
  const int64_t begin = a.offsets[s], stop = a.offsets[s + 1];
  const int64_t end = stop < a.n_entries ? stop : a.n_entries;
  return id >= 0 && begin >= 0 && begin < end && id < end - begin ? (int32_t)(begin + id) : -1;
}
__device__ inline int32_t entry_of(const EmbedArgs &a, int64_t row, int s) {
  return entry_at(a, a.ids[row * a.ldi + s], s);
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

// One slot a row: G lanes copy kAhead rows at a time, eight loads a lane on their way.  Bound by memory:
// 16,384 x 4096 bfloat16 41 us (134 MB written at 3.3 TB/s, frequent rows read from the caches).
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

// Lane u's value for all lanes of its group of G.
template <int G>
__device__ inline uint32_t of_lane(uint32_t v, int u) {
  if constexpr (G == 64) {
    return (uint32_t)__builtin_amdgcn_readlane((int)v, u);
  } else {
    return (uint32_t)__shfl((int)v, u, G);
  }
}

// Several slots a row: a.parts groups of G lanes share a row's slots and join in LDS.  Each lane of a
// group finds the entry of one of the next slots, and all of them take each entry in turn.  16,384 rows of
// 100 slots, 64 floats each of a table of 13 MB: 28 us, 419 MB from the caches.  Their rate (15 TB/s) and the
// instructions (13 us of the vector units, as many for 8 bfloat16 a lane as for 4 floats) share the bound:
// with bfloat16 19 us; of a table of 1.5 MB, which any L2 holds, 22, and 16 with bfloat16.
template <typename T, int G, int W>
__global__ __launch_bounds__(kThreads) void embed_bag_kernel(EmbedArgs a) {
  constexpr int groups = kThreads / G, U = G < 16 ? G : 16;
  __shared__ float join[kThreads * W];
  const Place p = place_of<G, W>(a, a.first);
  const int lane = threadIdx.x % G, group = threadIdx.x / G, part = group & (a.parts - 1);
  const int64_t wanted = p.block * (groups / a.parts) + group / a.parts;
  const int64_t row = wanted < a.n_rows ? wanted : a.n_rows - 1;
  const char *table = (const char *)((const T *)a.table + p.column);
  float sum[W];
#pragma unroll
  for (int i = 0; i < W; ++i) sum[i] = 0.0f;
  for (int64_t s0 = part * U; s0 < a.n_slots; s0 += (int64_t)a.parts * U) {
    int32_t at = -1;
    if (lane < U && s0 + lane < a.n_slots) at = entry_of(a, row, (int)(s0 + lane));
    // below 0: none (whatever the distance of a table's only entry is)
    const int64_t offset = at < 0 ? -1 : at * a.ldt * (int64_t)sizeof(T);
    Elements<T, W> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t low = of_lane<G>((uint32_t)offset, u);
      const int32_t high = (int32_t)of_lane<G>((uint32_t)(offset >> 32), u);
      e[u].clear();
      if (high >= 0) e[u].load((const T *)(table + ((int64_t)high << 32 | low)));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < W; ++i) sum[i] += e[u].at(i);
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
      auto bag = [&](auto lanes) {
        constexpr int G = decltype(lanes)::value, groups = kThreads / G;
        a.tiles = tiles_of(a.n_features, G, W);
        // groups share a row's slots while rows alone leave compute units idle
        a.parts = 1;
        while (a.parts < groups && a.n_rows * a.tiles * a.parts < 2048 * groups &&
               a.parts * (G < 16 ? G : 16) < a.n_slots)
          a.parts *= 2;
        const int64_t rows = groups / a.parts;
        return launch_blocks(embed_bag_kernel<T, G, W>, (a.n_rows + rows - 1) / rows * a.tiles,
                             kThreads, a, stream);
      };
      // A table that passes an XCD's L2: neighbouring workgroups run on neighbouring XCDs, so with a row in 8
      // tiles each L2 holds columns of its own.  Tiles of 128 to 512 bytes (us, whole rows / tiles of 128,
      // 256, 512 bytes, 100 slots: 16,384 x 64 float of a table of 13 MB 35 / 29; 4096 x 256 float, 52 MB
      // 53 / 33, 36, 45; 2048 x 1024 float, 41 MB 48 / 52, 41, 41; 16,384 x 64, 1.5 MB 22.6 / 23.5).
      if constexpr (G > 8) {
        const int64_t bytes = (int64_t)a.n_entries * a.n_features * (int)sizeof(T);
        const int64_t eighth = ((int64_t)a.n_features + 8 * W - 1) / (8 * W);  // lanes
        if (bytes > 4 << 20 && eighth <= 8) return bag(std::integral_constant<int, 8>());
        if constexpr (G > 16)
          if (bytes > 4 << 20 && eighth <= 16) return bag(std::integral_constant<int, 16>());
        if constexpr (G > 32)
          if (bytes > 4 << 20) return bag(std::integral_constant<int, 32>());
      }
      return bag(lanes);
    });
  });
}

// ============================================================================== BACKWARD
// Pairs (entry, row), one a slot, are sorted by entry: a radix sort whose passes keep the order of
// equal keys, so that an entry's rows stand in the order of their slots.  Groups of lanes then add
// the rows of blocks of neighbouring pairs; an entry whose pairs lie in one block is finished there,
// those of several blocks are joined afterwards, block after block.  The rest of the table is zero:
// workgroups that would wait for the sort fill it.  Empty slots have the key n_entries and end up
// behind all others.
constexpr int kFew = 16384;    // pairs that a workgroup holds
constexpr int kTile = 2048;    // pairs that a workgroup sorts at once where there are more
constexpr int kMaxDigit = 9;   // bits a pass of many pairs,
constexpr int kFewDigit = 10;  // and of few
constexpr int kBucketBits = 6, kBuckets = 1 << kBucketBits, kPlaceBits = 14;
constexpr int kFewThreads = 1024;
constexpr int kMostSlots = 1024;  // that are sorted one by one
static_assert(kFew == 1 << kPlaceBits, "a place fits its bits");

struct Pair {
  uint32_t key, row;
};

struct SortPlan {
  int passes, bits;  // of one digit
  bool few;
  int64_t pairs, tiles;
  int length;  // pairs of a block
  int64_t blocks;
};
static SortPlan plan_of(int64_t pairs, int32_t n_entries, int32_t n_features) {
  SortPlan p;
  int bits = 0;
  while ((int64_t)n_entries >> bits) ++bits;  // the largest key is n_entries
  p.few = pairs <= kFew && bits <= 32 - kPlaceBits + kBucketBits;
  if (p.few) bits = bits > kBucketBits ? bits - kBucketBits : 1;
  const int most = p.few ? kFewDigit : kMaxDigit;
  p.passes = (bits + most - 1) / most;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.pairs = pairs;
  p.tiles = (pairs + kTile - 1) / kTile;
  // blocks as long as leaves every compute unit several waves' work
  const int64_t lanes = n_features > 128 ? n_features / 8 : 16;
  p.length = 16;
  while (p.length < 128 && pairs / p.length * lanes > 512 * 1024) p.length *= 2;
  p.blocks = (pairs + p.length - 1) / p.length;
  return p;
}

struct GradArgs {
  EmbedArgs e;
  int64_t pairs, tiles;
  const Pair *sorted;  // so far; null: the slots themselves
  Pair *to;
  uint32_t *counts;  // [digit values][tiles]
  uint32_t *totals;  // [digit values]
  float *partial;    // [blocks][2]: of the entry that goes on from the block before; that goes on
  int64_t blocks;
  int length;
  int shift, bits, passes;
  int fill;       // workgroups that write zeros, 0: none
  int bytes;      // of an element
  int64_t first;  // the launch's first workgroup
};

// The pairs of slots (or of what is sorted) begin, begin + step, ... before `end`: all loads first, since
// one inside a branch is waited for there; past the end those of the last.
template <int N>
__device__ inline void load_pairs(const GradArgs &a, int64_t begin, int step, int64_t end, int rounds,
                                  Pair (&p)[N]) {
  auto index = [&](int u) {
    const int64_t i = begin + u * step;
    return i < end ? i : end - 1;
  };
  if (a.sorted) {
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (u < rounds) p[u] = a.sorted[index(u)];
    return;
  }
  int32_t id[N];
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (u < rounds) {
      const uint32_t i = (uint32_t)index(u);
      uint32_t s = 0;
      p[u].row = i;
      if (a.e.n_slots > 1) {
        p[u].row = i / (uint32_t)a.e.n_slots;
        s = i - p[u].row * (uint32_t)a.e.n_slots;
      }
      p[u].key = s;
      id[u] = a.e.ids[(int64_t)p[u].row * a.e.ldi + s];
    }
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (u < rounds) {
      const int32_t at = entry_at(a.e, id[u], (int)p[u].key);
      p[u].key = at < 0 ? (uint32_t)a.e.n_entries : (uint32_t)at;
    }
}
__device__ inline uint32_t digit_of(uint32_t key, int shift, int bits) {
  return key >> shift & ((1u << bits) - 1);
}

// Zeros, 16 bytes a lane where a row has them: workgroup `part` of a.fill.
__device__ inline void fill_zeros(const GradArgs &a, int part, int threads) {
  const int64_t row_bytes = (int64_t)a.e.n_features * a.bytes, pitch = a.e.ldo * a.bytes;
  char *out = (char *)a.e.out;
  const int64_t lane = (int64_t)part * threads + threadIdx.x, lanes = (int64_t)a.fill * threads;
  const u32x4 zero = {0, 0, 0, 0};
  if (pitch == row_bytes || a.e.n_entries == 1) {  // one run, but for its first and last bytes
    const int64_t bytes = row_bytes * a.e.n_entries;
    const int64_t head = bytes < 16 ? bytes : (int64_t)(-(uintptr_t)out & 15);
    const int64_t whole = (bytes - head) / 16;
    for (int64_t i = lane; i < whole; i += lanes) *(u32x4 *)(out + head + i * 16) = zero;
    const int64_t tail = bytes - head - whole * 16;
    for (int64_t i = lane; i < (head + tail) / a.bytes; i += lanes) {
      char *p = out + (i * a.bytes < head ? i * a.bytes : bytes - tail + (i * a.bytes - head));
      if (a.bytes == 4) {
        *(uint32_t *)p = 0;
      } else {
        *(uint16_t *)p = 0;
      }
    }
    return;
  }
  for (int64_t row = (int64_t)part * (threads / 64) + threadIdx.x / 64; row < a.e.n_entries;
       row += (int64_t)a.fill * (threads / 64)) {
    char *p = out + row * pitch;
    if (row_bytes < 16) {
      for (int64_t i = (threadIdx.x & 63) * a.bytes; i < row_bytes; i += 64 * a.bytes)
        __builtin_memcpy(p + i, &zero, 2), __builtin_memcpy(p + i + a.bytes - 2, &zero, 2);
    } else {
      for (int64_t i = (threadIdx.x & 63) * 16; i < row_bytes; i += 64 * 16)
        __builtin_memcpy(p + (i < row_bytes - 16 ? i : row_bytes - 16), &zero, 16);
    }
  }
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

// How many of the lanes in the mask are below this one.
__device__ inline int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Lanes of the wave whose digit is this lane's (`live` lanes only).
__device__ inline uint64_t lanes_alike(uint32_t digit, int bits, bool live) {
  const uint64_t all = __ballot(live);
  uint32_t low = (uint32_t)all, high = (uint32_t)(all >> 32);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    const uint32_t unset = (digit >> b & 1) - 1;  // all bits where the lane's is 0
    low &= (uint32_t)set ^ unset;
    high &= (uint32_t)(set >> 32) ^ unset;
  }
  return (uint64_t)high << 32 | low;
}

// The place of the lane's pair of digit d, from next[d], which moves on by the lanes alike; all lanes
// of a wave call it.
__device__ inline uint32_t take_place(volatile uint32_t *next, uint32_t d, int bits, bool live) {
  const uint64_t same = lanes_alike(d, bits, live);
  const int earlier = lanes_below(same);
  uint32_t at = 0;
  if (live) {
    at = next[d] + earlier;
    // the wave's lanes have all read it; the first of those alike moves it on
    __builtin_amdgcn_wave_barrier();
    if (earlier == 0) next[d] = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  return at;
}

// The counts of the waves' digits become the places of each wave's first pair, behind those of smaller
// digits and of the waves before.  Each thread takes a run of digits.
template <int kWaves, int kValues>
__device__ inline void places(uint32_t (&next)[kWaves][kValues], uint32_t *wave_sum, int values) {
  const int run = (values + kWaves * 64 - 1) / (kWaves * 64);
  const int d0 = threadIdx.x * run, wave = threadIdx.x / 64;
  uint32_t own = 0, all;
  for (int d = d0; d < d0 + run && d < values; ++d)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) own += next[w][d];
  uint32_t at = lanes_before(own, &all);
  if ((threadIdx.x & 63) == 0) wave_sum[wave] = all;
  __syncthreads();
  for (int w = 0; w < wave; ++w) at += wave_sum[w];
  for (int d = d0; d < d0 + run && d < values; ++d)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = next[w][d];
      next[w][d] = at;
      at += c;
    }
  __syncthreads();
}

// The items of `held`, sorted by what stands above their kPlaceBits, `bits` a pass; f(place, item) for each
// after the last.
template <typename F>
__device__ inline void sort_held(uint32_t (&held)[kFew],
                                 uint32_t (&next)[kFewThreads / 64][1 << kFewDigit],
                                 uint32_t *wave_sum, int count, int bits, int passes, F f) {
  constexpr int waves = kFewThreads / 64, most = kFew / kFewThreads;
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int rounds = (count + kFewThreads - 1) / kFewThreads, values = 1 << bits;
  const int begin = wave * rounds * 64 + lane;
  for (int pass = 0; pass < passes; ++pass) {
    __syncthreads();
    for (int d = lane; d < values; d += 64) next[wave][d] = 0;
    const int shift = kPlaceBits + pass * bits;
    uint32_t item[most];
#pragma unroll
    for (int u = 0; u < most; ++u)
      if (u < rounds && begin + u * 64 < count) {
        item[u] = held[begin + u * 64];
        atomicAdd(&next[wave][digit_of(item[u], shift, bits)], 1u);
      }
    __syncthreads();
    places<waves, 1 << kFewDigit>(next, wave_sum, values);
#pragma unroll
    for (int u = 0; u < most; ++u)
      if (u < rounds) {
        const bool live = begin + u * 64 < count;
        const uint32_t at = take_place(next[wave], digit_of(item[u], shift, bits), bits, live);
        if (live && pass < passes - 1) {
          held[at] = item[u];
        } else if (live) {
          f(at, item[u]);
        }
      }
  }
}

// Few pairs: what the sums need is that an entry's pairs stand together, in their order, so kBuckets
// workgroups take the entries of one remainder each.  Each reads all slots, keeps its own, whose
// place among all it learns from the count of lower remainders, and sorts them by the rest of the key
// in one pass (tables below 2^16 entries) or two.  The other workgroups fill the table with zeros
// meanwhile.  16,384 slots: 14 us, of which 8 are the walk over all slots and bound by instructions
// (32 workgroups of 512 lanes: 22); beside 103 MB of zeros 21, at which those alone are 18.
__global__ __launch_bounds__(kFewThreads) void embed_group_kernel(GradArgs a) {
  constexpr int waves = kFewThreads / 64, most = kFew / kFewThreads;
  __shared__ uint32_t held[kFew];  // rest of the key, place among the slots
  __shared__ uint32_t next[waves][1 << kFewDigit];
  __shared__ uint32_t wave_sum[2][waves];
  if (blockIdx.x >= kBuckets) {
    fill_zeros(a, blockIdx.x - kBuckets, kFewThreads);
    return;
  }
  const uint32_t bucket = blockIdx.x;
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  int base = 0, count = 0;  // pairs of lower remainders; of this one
  {
    const int n = (int)a.pairs, rounds = (n + kFewThreads - 1) / kFewThreads;
    const int begin = wave * rounds * 64 + lane;
    Pair p[most];
    load_pairs<most>(a, begin, 64, n, rounds, p);
    int own = 0, lower = 0;
#pragma unroll
    for (int u = 0; u < most; ++u)
      if (u < rounds) {
        const bool live = begin + u * 64 < n;
        own += __popcll(__ballot(live && p[u].key % kBuckets == bucket));
        lower += __popcll(__ballot(live && p[u].key % kBuckets < bucket));
      }
    if (lane == 0) wave_sum[0][wave] = own, wave_sum[1][wave] = lower;
    __syncthreads();
    int at = 0;
    for (int w = 0; w < waves; ++w) {
      if (w == wave) at = count;
      count += wave_sum[0][w];
      base += wave_sum[1][w];
    }
#pragma unroll
    for (int u = 0; u < most; ++u)
      if (u < rounds) {
        const bool mine = begin + u * 64 < n && p[u].key % kBuckets == bucket;
        const uint64_t all = __ballot(mine);
        if (mine)
          held[at + lanes_below(all)] =
              p[u].key >> kBucketBits << kPlaceBits | (uint32_t)(begin + u * 64);
        at += __popcll(all);
      }
  }
  sort_held(held, next, wave_sum[0], count, a.bits, a.passes, [&](uint32_t at, uint32_t item) {
    const uint32_t i = item & (kFew - 1);
    a.to[base + at] = {item >> kPlaceBits << kBucketBits | bucket,
                       a.e.n_slots > 1 ? i / (uint32_t)a.e.n_slots : i};
  });
}

// More pairs, of slots with entries of their own and at most kFew rows: the slots' entries ascend, so a
// workgroup sorts each slot's pairs by their ids, in one pass (slots below 2^10 entries) or two.  Empty
// slots stand behind their slot's others.  Neighbouring slots, whose ids share cache lines, go to one XCD.
// Bound by the chain of steps within a workgroup, one a CU.  The whole gradient of 64 floats, this way / as
// all pairs: 16,384 rows x 100 slots 76 us / 90, 4000 x 100 35 / 57, 300 x 100 20 / 44; many slots of few
// rows leave most of a workgroup idle (40 x 4000 89 / 50).
__global__ __launch_bounds__(kFewThreads) void embed_slots_kernel(GradArgs a) {
  constexpr int waves = kFewThreads / 64, most = kFew / kFewThreads;
  __shared__ uint32_t held[kFew];  // id, row
  __shared__ uint32_t next[waves][1 << kFewDigit];
  __shared__ uint32_t wave_sum[waves];
  const int share = (a.e.n_slots + 7) / 8, block = blockIdx.x;  // slots of an XCD
  if (block >= share * 8) {
    fill_zeros(a, block - share * 8, kFewThreads);
    return;
  }
  const int slot = block % 8 * share + block / 8;
  if (slot >= a.e.n_slots) return;
  const int n = (int)a.e.n_rows, rounds = (n + kFewThreads - 1) / kFewThreads;
  const int first = threadIdx.x / 64 * rounds * 64 + (threadIdx.x & 63);
  int32_t id[most];
#pragma unroll
  for (int u = 0; u < most; ++u)
    if (u < rounds) {
      const int row = first + u * 64;
      id[u] = a.e.ids[(int64_t)(row < n ? row : n - 1) * a.e.ldi + slot];
    }
  const int64_t begin = a.e.offsets[slot], stop = a.e.offsets[slot + 1];
  const int64_t end = stop < a.e.n_entries ? stop : a.e.n_entries;
  const uint32_t size = begin >= 0 && begin < end ? (uint32_t)(end - begin) : 0;
#pragma unroll
  for (int u = 0; u < most; ++u)
    if (u < rounds && first + u * 64 < n)
      held[first + u * 64] = ((uint32_t)id[u] < size ? (uint32_t)id[u] : size) << kPlaceBits |
                             (uint32_t)(first + u * 64);
  const int bits = size ? 32 - __builtin_clz(size) : 1, passes = bits > kFewDigit ? 2 : 1;
  sort_held(held, next, wave_sum, n, (bits + passes - 1) / passes, passes,
            [&](uint32_t at, uint32_t item) {
              const uint32_t key = item >> kPlaceBits;
              a.to[(int64_t)slot * n + at] = {key < size ? (uint32_t)begin + key : (uint32_t)a.e.n_entries,
                                     item & (kFew - 1)};
            });
}

// More pairs: a pass counts every tile's digits, adds the counts up over the tiles, and moves the
// pairs.  1,638,400 pairs in two passes of 8 bits: 8, 5 and 15 us for the first, bound by the chain of steps
// within a tile (three or four tiles a CU, all at once).  How many of a tile's pairs have each digit:
__global__ __launch_bounds__(kThreads) void embed_count_kernel(GradArgs a) {
  __shared__ uint32_t count[1 << kMaxDigit];
  const int64_t block = a.first + blockIdx.x;
  if (block >= a.tiles) {
    fill_zeros(a, (int)(block - a.tiles), kThreads);
    return;
  }
  const int values = 1 << a.bits;
  for (int d = threadIdx.x; d < values; d += kThreads) count[d] = 0;
  __syncthreads();
  const int64_t begin = block * kTile;
  constexpr int rounds = kTile / kThreads;
  Pair p[rounds];
  load_pairs<rounds>(a, begin + threadIdx.x, kThreads, a.pairs, rounds, p);
#pragma unroll
  for (int u = 0; u < rounds; ++u)
    if (begin + u * kThreads + threadIdx.x < a.pairs)
      atomicAdd(&count[digit_of(p[u].key, a.shift, a.bits)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < values; d += kThreads) a.counts[d * a.tiles + block] = count[d];
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

// Moves a tile's pairs to their places: within the tile first, through LDS, so that what goes to one
// digit's place leaves in runs.
__global__ __launch_bounds__(kThreads) void embed_move_kernel(GradArgs a) {
  constexpr int waves = kThreads / 64, rounds = kTile / kThreads;
  __shared__ uint32_t next[waves][1 << kMaxDigit];
  __shared__ uint32_t wave_sum[waves];
  __shared__ Pair tile_pairs[kTile];
  __shared__ uint32_t shift_of[1 << kMaxDigit];  // from a pair's place in the tile to that in all
  const int values = 1 << a.bits, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int64_t tile = a.first + blockIdx.x, first = tile * kTile;
  const int begin = wave * (rounds * 64) + lane;
  const int n = (int)(a.pairs - first < kTile ? a.pairs - first : kTile);
  Pair p[rounds];
  load_pairs<rounds>(a, first + begin, 64, a.pairs, rounds, p);
  // where a digit's pairs of this tile begin among all
  {
    const int run = (values + kThreads - 1) / kThreads, d0 = threadIdx.x * run;
    uint32_t own = 0, all;
    for (int d = d0; d < d0 + run && d < values; ++d) own += a.totals[d];
    uint32_t before = lanes_before(own, &all);
    if (lane == 0) wave_sum[wave] = all;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before += wave_sum[w];
    for (int d = d0; d < d0 + run && d < values; ++d) {
      shift_of[d] = before + a.counts[d * a.tiles + tile];
      before += a.totals[d];
    }
  }
  for (int d = lane; d < values; d += 64) next[wave][d] = 0;
#pragma unroll
  for (int u = 0; u < rounds; ++u)
    if (begin + u * 64 < n) atomicAdd(&next[wave][digit_of(p[u].key, a.shift, a.bits)], 1u);
  __syncthreads();
  places<waves, 1 << kMaxDigit>(next, wave_sum, values);
  for (int d = threadIdx.x; d < values; d += kThreads) shift_of[d] -= next[0][d];
  __syncthreads();
#pragma unroll
  for (int u = 0; u < rounds; ++u) {
    const bool live = begin + u * 64 < n;
    const uint32_t at = take_place(next[wave], digit_of(p[u].key, a.shift, a.bits), a.bits, live);
    if (live) tile_pairs[at] = p[u];
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < rounds; ++u) {
    const int i = u * kThreads + threadIdx.x;
    if (i < n) {
      const Pair q = tile_pairs[i];
      a.to[shift_of[digit_of(q.key, a.shift, a.bits)] + i] = q;
    }
  }
}

// G lanes add the rows of a block of neighbouring pairs, whatever their entries, with U loads on
// their way, and hand on what they have where the entry changes: no entry's length decides a lane's work.
// 1,638,400 pairs of 64 floats 31 us (419 MB from the caches at 13 TB/s; 128 bytes a group 33, 64 bytes 50).
template <typename T, int G, int W>
__global__ __launch_bounds__(64) void embed_blocks_kernel(GradArgs a) {
  constexpr int U = G < 16 ? G : 16;
  const Place p = place_of<G, W>(a.e, a.first);
  const int lane = threadIdx.x % G;
  const int64_t block = p.block * (64 / G) + threadIdx.x / G;
  if (block >= a.blocks) return;
  const int64_t begin = block * a.length;
  const int64_t end = begin + a.length < a.pairs ? begin + a.length : a.pairs;
  const uint32_t none = 0xFFFFFFFFu;
  const uint32_t key_before = begin > 0 ? a.sorted[begin - 1].key : none;
  const uint32_t key_after = end < a.pairs ? a.sorted[end].key : none;
  const T *grad = (const T *)a.e.table + p.column;
  float sum[W];
  uint32_t key = key_before;
  bool goes_on = true;  // from the block before
  auto hand_on = [&](bool further) __attribute__((always_inline)) {
    if (key < (uint32_t)a.e.n_entries && p.inside) {
      if (goes_on || further) {
        __builtin_memcpy(
            a.partial + (2 * block + !goes_on) * (int64_t)a.e.n_features + p.column, sum,
            sizeof(sum));
      } else {
        float v[W];
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = sum[k] * a.e.scale;
        store_elements<T, W>((T *)a.e.out + (int64_t)key * a.e.ldo + p.column, v);
      }
    }
  };
  for (int64_t i0 = begin; i0 < end; i0 += U) {
    Pair mine = {none, 0};
    if (lane < U && i0 + lane < end) mine = a.sorted[i0 + lane];
    uint32_t keys[U];
    Elements<T, W> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      keys[u] = of_lane<G>(mine.key, u);
      const uint32_t row = of_lane<G>(mine.row, u);
      e[u].clear();
      if (keys[u] < (uint32_t)a.e.n_entries) e[u].load(grad + (int64_t)row * a.e.ldt);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u >= end) break;
      if (keys[u] != key || (i0 == begin && u == 0)) {
        if (i0 > begin || u > 0) hand_on(false);
        goes_on = keys[u] == key_before && i0 == begin && u == 0;
        key = keys[u];
#pragma unroll
        for (int k = 0; k < W; ++k) sum[k] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < W; ++k) sum[k] += e[u].at(k);
    }
  }
  hand_on(key == key_after);
}

// Entries of several blocks: the block where one begins has its first sum, the blocks after it one
// each.  A workgroup looks at kHeads blocks; a group of lanes adds the sums of a short entry, all
// groups together those of a long one.
constexpr int kHeads = 16, kShort = 32;
template <typename T, int G, int W>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(GradArgs a) {
  constexpr int groups = kThreads / G;
  __shared__ int32_t last[kHeads];  // blocks after the one where an entry begins; 0: none begins
  __shared__ uint32_t entry[kHeads];
  __shared__ float join[kThreads * W];
  const Place p = place_of<G, W>(a.e, a.first);
  const int group = threadIdx.x / G, width = a.e.n_features;
  const int64_t block0 = p.block * kHeads;
  {
    constexpr int lanes = kThreads / kHeads;  // of a block
    static_assert(lanes == 16, "a step's results are 16 bits of a ballot");
    const int h = threadIdx.x / lanes, r = threadIdx.x % lanes;
    const int64_t block = block0 + h, begin = block * a.length, end = begin + a.length;
    int32_t count = 0;
    uint32_t key = 0;
    if (end < a.pairs) {
      key = a.sorted[end - 1].key;
      const uint32_t after = a.sorted[end].key;
      const uint32_t before = begin > 0 ? a.sorted[begin - 1].key : ~key;
      if (key < (uint32_t)a.e.n_entries && after == key && before != key) {
        // the last block that begins with the entry: 16 probes a step, growing steps, then shrinking
        int64_t last_block = block + 1, step = 1;
        auto go = [&] {
          const int64_t probe = last_block + (r + 1) * step;
          const bool hit = probe < a.blocks && a.sorted[probe * a.length].key == key;
          const uint32_t hits = (uint32_t)(__ballot(hit) >> (threadIdx.x & 48)) & 0xFFFFu;
          const int n = __builtin_ctz(~hits);
          last_block += n * step;
          return n;
        };
        while (go() == lanes) step *= lanes;
        while (step > 1) {
          step /= lanes;
          go();
        }
        count = (int32_t)(last_block - block);
      }
    }
    if (r == 0) last[h] = count, entry[h] = key;
  }
  __syncthreads();
  // sum += those of blocks [c, end)
  auto add = [&](float(&sum)[W], int64_t c, int64_t end) {
    for (; c < end; c += kAhead) {
      float v[kAhead][W];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        __builtin_memcpy(v[u],
                         a.partial + 2 * (c + u < end ? c + u : c) * (int64_t)width + p.column,
                         sizeof(v[u]));
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int k = 0; k < W; ++k) sum[k] += c + u < end ? v[u][k] : 0.0f;
    }
  };
  auto finish = [&](float(&sum)[W], int h) {
    if (!p.inside) return;
#pragma unroll
    for (int k = 0; k < W; ++k) sum[k] *= a.e.scale;
    store_elements<T, W>((T *)a.e.out + (int64_t)entry[h] * a.e.ldo + p.column, sum);
  };
  for (int h = group; h < kHeads; h += groups) {
    if (last[h] == 0 || last[h] > kShort) continue;
    const int64_t block = block0 + h;
    float sum[W];
    __builtin_memcpy(sum, a.partial + (2 * block + 1) * (int64_t)width + p.column, sizeof(sum));
    add(sum, block + 1, block + 1 + last[h]);
    finish(sum, h);
  }
  for (int h = 0; h < kHeads; ++h) {
    if (last[h] <= kShort) continue;  // of the whole workgroup
    const int64_t block = block0 + h, share = (last[h] + groups - 1) / groups;
    const int64_t c = block + 1 + group * share, end = block + 1 + last[h];
    float sum[W];
#pragma unroll
    for (int k = 0; k < W; ++k) sum[k] = 0.0f;
    if (group == 0)
      __builtin_memcpy(sum, a.partial + (2 * block + 1) * (int64_t)width + p.column, sizeof(sum));
    add(sum, c, c + share < end ? c + share : end);
#pragma unroll
    for (int k = 0; k < W; ++k) join[k * kThreads + threadIdx.x] = sum[k];
    __syncthreads();
    if (group == 0) {
      for (int q = 1; q < groups; ++q)
#pragma unroll
        for (int k = 0; k < W; ++k) sum[k] += join[k * kThreads + threadIdx.x + q * G];
      finish(sum, h);
    }
    __syncthreads();
  }
}

// The workspace's parts, each from a multiple of 16 bytes.
struct Parts {
  int64_t pairs[2], counts, totals, partial, bytes;
};
static Parts parts_of(const SortPlan &p, int64_t width) {
  Parts w;
  int64_t at = 0;
  auto take = [&](int64_t words) {
    const int64_t begin = at;
    at += (words * 4 + 15) / 16 * 16;
    return begin;
  };
  w.pairs[0] = take(2 * p.pairs);
  w.pairs[1] = p.few ? w.pairs[0] : take(2 * p.pairs);
  w.counts = take(p.few ? 0 : p.tiles << p.bits);
  w.totals = take(p.few ? 0 : int64_t(1) << p.bits);
  w.partial = take(p.blocks * 2 * width);
  w.bytes = at;
  return w;
}

int64_t embed_backward_bytes(int64_t n_rows, int32_t n_slots, int32_t n_entries,
                             int32_t n_features) {
  const SortPlan p = plan_of(n_rows * n_slots, n_entries, n_features);
  return parts_of(p, n_features).bytes;
}

int launch_embed_backward(const EmbedArgs &args, int32_t dtype, void *stream) {
  const SortPlan plan = plan_of(args.n_rows * args.n_slots, args.n_entries, args.n_features);
  const Parts parts = parts_of(plan, args.n_features);
  char *ws = (char *)args.workspace;
  GradArgs a = {};
  a.e = args;
  a.pairs = plan.pairs;
  a.tiles = plan.tiles;
  a.counts = (uint32_t *)(ws + parts.counts);
  a.totals = (uint32_t *)(ws + parts.totals);
  a.partial = (float *)(ws + parts.partial);
  a.blocks = plan.blocks;
  a.length = plan.length;
  a.bits = plan.bits;
  a.passes = plan.passes;
  a.bytes = dtype == BRIDGER_F32 ? 4 : 2;
  const int64_t out_bytes = (int64_t)args.n_entries * args.n_features * a.bytes;
  auto fill_of = [&](int threads) {  // 64 bytes or more a lane
    const int64_t n = (out_bytes + threads * 64 - 1) / (threads * 64);
    const int64_t most = 2048 * 256 / threads;
    return (int)(n < most ? n : most);
  };
  int err = 0;
  if (plan.few) {
    a.fill = fill_of(kFewThreads);
    a.to = (Pair *)(ws + parts.pairs[0]);
    err = launch(embed_group_kernel, kBuckets + (int64_t)a.fill, kFewThreads, 0, a, stream);
    a.sorted = a.to;
  }
  const bool by_slot = !plan.few && args.offsets && args.n_rows <= kFew &&
                       args.n_slots <= kMostSlots && args.n_entries < 1 << (32 - kPlaceBits);
  if (by_slot) {
    a.fill = fill_of(kFewThreads);
    a.to = (Pair *)(ws + parts.pairs[0]);
    const int64_t slots = ((int64_t)args.n_slots + 7) / 8 * 8;
    err = launch(embed_slots_kernel, slots + a.fill, kFewThreads, 0, a, stream);
    a.sorted = a.to;
  }
  for (int pass = 0; pass < plan.passes && !plan.few && !by_slot; ++pass) {
    a.shift = pass * plan.bits;
    a.to = (Pair *)(ws + parts.pairs[pass & 1]);
    a.fill = pass == 0 ? fill_of(kThreads) : 0;
    err = launch_blocks(embed_count_kernel, a.tiles + a.fill, kThreads, a, stream);
    if (!err) {
      const int waves = kThreads / 64;
      err = launch(embed_scan_kernel, ((1 << a.bits) + waves - 1) / waves, kThreads, 0, a, stream);
    }
    if (!err) err = launch_blocks(embed_move_kernel, a.tiles, kThreads, a, stream);
    if (err) return err;
    a.sorted = a.to;
  }
  if (err || !plan.pairs) return err;
  return with_type(dtype, [&](auto t) {
    using T = decltype(t);
    return with_lanes<T>(args.n_features, [&](auto lanes, auto elements) {
      constexpr int G = decltype(lanes)::value, W = decltype(elements)::value;
      GradArgs g = a;
      g.e.tiles = tiles_of(g.e.n_features, G, W);
      const int64_t at_once = 64 / G;
      const int e = launch_blocks(embed_blocks_kernel<T, G, W>,
                                  (g.blocks + at_once - 1) / at_once * g.e.tiles, 64, g, stream);
      if (e || g.blocks == 1) return e;
      return launch_blocks(embed_join_kernel<T, G, W>, (g.blocks + kHeads - 1) / kHeads * g.e.tiles,
                           kThreads, g, stream);
    });
  });
}

}  // namespace bridger
