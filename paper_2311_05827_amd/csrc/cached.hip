// Attention of few tokens a sequence over its pages of keys and values: bound by reading those once.
#include "attention.hpp"

namespace accept {
namespace {

struct CacheArgs {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* parts_at;  // results of pieces of an item: see slot_at
  const int32_t* offsets;
  const int32_t* lengths;
  const int32_t* table;
  const uint64_t* tree;
  int64_t q_stride, o_stride;
  Pages pages;
  int sequences, tokens, each;
  int heads, group, head;
  int parts;       // of a key head's work
  int tree_words;
  int zeros;
  float scale;     // times log2(e)
};

// An item is 32 rows of a key head: its query heads for one token after the other.  Rows are columns of the products, as in attention_kernel.
constexpr int kItem = 32;

// What a wavefront goes through at a time is 32 keys; it keeps the next 32 coming, in shared memory of its own, and waits for nobody.  A
// unit of work is 32 keys for each wavefront of a workgroup.
template <typename T, int DB>
struct Shape {
  static constexpr int kTile = 32 * Head<T, DB>::kRowBytes;
  static constexpr int kWaves = 4 * kTile * 4 <= 131072 ? 4 : 131072 / (4 * kTile);
  static constexpr int kUnit = 32 * kWaves;
  static constexpr int kThreads = kWaves * kWave;
  static constexpr int kSum = DB * 32 * (kItem + 1);  // floats of a wavefront's results, transposed without meeting banks
  static_assert(kSum * 4 <= 4 * kTile, "results take the tiles' place");
};
// A sequence of the step.
struct Step {
  Span span;
  int length;  // cached tokens
  int keys;    // places that its tokens may see
  int64_t items, units;  // units of every item
};
__device__ __forceinline__ Step step_of(const CacheArgs& g, int seq, int unit) {
  Step s;
  s.span = span_of(g.offsets, seq, g.tokens, g.each);
  const int64_t capacity = g.pages.count > 0 ? int64_t(g.pages.table_pages) << g.pages.shift : 0;
  const int n = s.span.size(), given = g.lengths[seq];
  s.length = given < 0 ? 0 : given;
  const int64_t all = int64_t(s.length) + n;
  s.keys = int(all < capacity ? all : capacity);
  s.items = (int64_t(n) * g.group + kItem - 1) / kItem;
  const int64_t units = (int64_t(s.keys) + unit - 1) / unit;
  s.units = units > 0 ? units : 1;
  return s;
}
__device__ __forceinline__ Step uniform_step(const CacheArgs& g, int seq, int unit) {
  const Step s = step_of(g, seq, unit);
  return {{uniform(s.span.begin), uniform(s.span.end)}, uniform(s.length), uniform(s.keys), uniform(s.items), uniform(s.units)};
}
// Work of a key head, in units one behind the other, is dealt in equal parts.  A part has at most two pieces of items that are not whole: the end of one that
// began before it, and the beginning of one that goes on behind it.
__device__ __forceinline__ int64_t part_begin(int64_t all, int parts, int p) { return all * p / parts; }
__device__ __forceinline__ int used_parts(int64_t all, int parts) { return all < parts ? int(all) : parts; }
// Floats of a piece's results: 32 rows of sums, their maxima, their sums of weights.
__device__ __forceinline__ float* slot_at(const CacheArgs& g, int kv, int part, bool begins, int width) {
  return g.parts_at + (int64_t(kv) * g.parts + part) * 2 * kItem * (width + 2) + (begins ? kItem * (width + 2) : 0);
}

template <typename T, int DB>
__global__ __launch_bounds__((Shape<T, DB>::kThreads), 1) void cached_kernel(const CacheArgs g) {
  using S = Shape<T, DB>;
  using H = Head<T, DB>;
  constexpr int kWidth = DB * 32, kPad = kItem + 1;
  __shared__ __align__(kTileAlign) uint8_t tiles[S::kWaves][4 * S::kTile];
  __shared__ float peak[S::kWaves][kItem], total[S::kWaves][kItem];
  const int lane = threadIdx.x % kWave, wave = uniform(int(threadIdx.x / kWave));
  const int half = lane / 32, column = lane % 32;
  const int kv = blockIdx.y, part = blockIdx.x;
  const int parts_of_row = g.head * int(sizeof(T)) / 16;
  uint8_t* const mine = tiles[wave];

  const auto work = [&](int s) {
    const Step st = step_of(g, s, S::kUnit);
    return st.items * st.units;
  };
  const int64_t all = uniform(find_among(g.sequences, INT64_MAX, work).before);
  const int parts = used_parts(all, g.parts);
  if (part >= parts) return;
  int64_t at = part_begin(all, parts, part);
  const int64_t end = part_begin(all, parts, part + 1);
  const Found found = find_among(g.sequences, at, work);
  int seq = uniform(found.seq);
  int64_t before = uniform(found.before);
  if (g.head < kWidth) {
    for (int i = lane * 16; i < 4 * S::kTile; i += kWave * 16) *reinterpret_cast<uint4*>(mine + i) = make_uint4(0, 0, 0, 0);
  }

  while (at < end && seq < g.sequences) {
    const Step st = uniform_step(g, seq, S::kUnit);
    const int64_t in = at - before;
    if (in >= st.items * st.units) {
      before += st.items * st.units;
      ++seq;
      continue;
    }
    const int64_t item = in / st.units;
    const int unit0 = int(in - item * st.units);
    const int unit1 = int(st.units - unit0 < end - at ? st.units : unit0 + (end - at));
    at += unit1 - unit0;

    const int64_t rows = int64_t(st.span.size()) * g.group, row0 = item * kItem;
    const int count = int(rows - row0 < kItem ? rows - row0 : kItem);
    const int64_t row = row0 + (column < count ? column : count - 1);
    const int of_step = int(row / g.group), token = st.span.begin + of_step, head = kv * g.group + int(row % g.group);
    const int64_t sees = int64_t(st.length) + of_step + 1;
    const int limit = g.tree_words ? st.keys : int(sees < st.keys ? sees : st.keys);
    const int64_t first_sees = int64_t(st.length) + (g.tree_words ? 0 : row0 / g.group + 1);
    const int all_see = int(first_sees < st.keys ? first_sees : st.keys);       // every row sees keys before it
    const int64_t last_sees = int64_t(st.length) + (row0 + count - 1) / g.group + 1;
    const int some_see = g.tree_words || last_sees > st.keys ? st.keys : int(last_sees);
    RowParts<T, DB> q;
    q.load(static_cast<const T*>(g.q) + token * g.q_stride + int64_t(head) * g.head, half, parts_of_row);

    // 32 keys from key0 on, into buffer b; which of them exist
    typedef const __attribute__((address_space(4))) int32_t constant_int;
    const auto page_of = [&](int j) {
      return uniform(int(((constant_int*)(g.table))[int64_t(seq) * g.pages.table_pages + (j >> g.pages.shift)]));
    };
    const auto fetch = [&](int key0, int b) {
      constexpr int kPer = 1024 / H::kRowBytes, kLoads = 32 / kPer;
      const bool one_page = g.pages.shift >= 5;
      uint32_t there = 0;
      int page = 0;
      const uint32_t to = lds_offset(mine) + uint32_t(b) * 2u * S::kTile;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int j = key0 + i * kPer < st.keys ? key0 + i * kPer : st.keys - 1;
        if (i == 0 || !one_page) page = page_of(j);
        const bool is = is_page(g.pages, page);
        there |= is ? (kPer == 32 ? ~0u : ((1u << (kPer % 32)) - 1u)) << (i * kPer) : 0u;
        const int64_t first = cache_row(g.pages, is ? page : 0, j, kv) * g.head * int(sizeof(T));
        const int r = lane / H::kRowParts, p = lane % H::kRowParts ^ turn<H::kRowBytes>(i * kPer + r);
        const int left = st.keys - 1 - j;  // rows behind j
        const uint32_t offset = uint32_t(r < left ? r : left) * uint32_t(g.head * int(sizeof(T))) + uint32_t(p) * 16u;
        if (p < parts_of_row) {
          load_tile_part(static_cast<const uint8_t*>(g.k) + first, offset, to + i * 1024);
          load_tile_part(static_cast<const uint8_t*>(g.v) + first, offset, to + S::kTile + i * 1024);
        }
      }
      return there;
    };
    const auto seen_among = [&](int key0, uint32_t there) {
      uint32_t seen = bits_between(0, limit - key0) & there;
      if (g.tree_words && key0 + 32 > st.length) {
        const int first = key0 - st.length;  // the node that bit 0 is; below 0: cached
        const uint64_t* const words = g.tree + int64_t(token) * g.tree_words;
        const auto word = [&](int i) { return i < g.tree_words ? words[i] : 0; };
        uint32_t nodes;
        if (first < 0) {
          nodes = uint32_t(word(0)) << -first | ((1u << -first) - 1u);
        } else {
          const int by = first % 64;
          uint64_t w = word(first / 64) >> by;
          if (by > 32) w |= word(first / 64 + 1) << (64 - by);
          nodes = uint32_t(w);
        }
        seen &= nodes;
      }
      return seen;
    };

      const Reader<T, DB> lanes(lane);
    v16f_t acc[DB];
    float largest, sum;
    const int stop = some_see < unit1 * S::kUnit ? some_see : unit1 * S::kUnit;
    const auto run = [&](auto apart) {
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = v16f_t{};
      largest = -INFINITY;
      sum = 0.0f;
      int key0 = unit0 * S::kUnit + wave * 32, b = 0;
      uint32_t there = 0;
      if (key0 < stop) there = fetch(key0, 0);
      for (; key0 < stop; key0 += S::kUnit, b ^= 1) {
        __builtin_amdgcn_s_waitcnt(0);
        asm volatile("" : : : "memory");
        const uint32_t now_there = there;
        if (key0 + S::kUnit < stop) there = fetch(key0 + S::kUnit, b ^ 1);
        const uint8_t* const kt = mine + b * 2 * S::kTile;
        const uint8_t* const vt = kt + S::kTile;
        const Reader<T, DB> reader = lanes.fresh();
        v16f_t s = rows_product<T, DB>(lds_offset(kt), reader, 0, q);
        const bool masked = key0 + 32 > all_see || now_there != ~0u;
        uint32_t seen = ~0u;
        if (masked) {
          seen = seen_among(key0, now_there);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = seen >> result_row(r, half) & 1 ? s[r] : -INFINITY;
        }
        float most = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, s[r]);
        most = halves_max(most) * g.scale;
        if (__any(most > largest + 8.0f)) {  // (see kBehind of attention_kernel)
          const float now = fmaxf(largest, most);
          const float factor = largest == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(largest - now);
          largest = now;
          sum *= factor;
#pragma unroll
          for (int db = 0; db < DB; ++db) acc[db] *= factor;
        }
        const float base = largest == -INFINITY ? 0.0f : -largest;
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], g.scale, base));
          sum += p[r];
        }
        if (apart.value && masked) {
          weighted_rows_apart<T, DB>(acc, vt, 0, lane, p, seen);
        } else {
          Weights<T> w;
          set_weights(w, p);
          weighted_rows<T, DB>(acc, lds_offset(vt), reader, 0, w);
        }
      }
    };
    run(Flag<false>{});
    if (__any(column < count && !finite_column<DB>(acc))) run(Flag<true>{});
    sum = halves_sum(sum);

    // the wavefronts' results together, relative to the largest of their maxima
    if (half == 0) peak[wave][column] = largest;
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < S::kWaves; ++w) top = fmaxf(top, peak[w][column]);
    const float factor = largest == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(largest - top);
    if (half == 0) total[wave][column] = sum * factor;
    float* const out = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) out[(db * 32 + result_row(r, half)) * kPad + column] = largest == -INFINITY ? 0.0f : acc[db][r] * factor;
    __syncthreads();
    const bool begins = unit0 == 0, ends = unit1 == st.units;
    float* const slot = slot_at(g, kv, part, begins, kWidth);
    for (int i = threadIdx.x; i < count * kWidth; i += S::kThreads) {
      const int r = i / kWidth, d = i % kWidth;
      float v = 0.0f, l = 0.0f;
#pragma unroll
      for (int w = 0; w < S::kWaves; ++w) {
        v += reinterpret_cast<const float*>(tiles[w])[d * kPad + r];
        l += total[w][r];
      }
      if (begins && ends) {
        const int64_t flat = row0 + r;
        if (d < g.head)
          store_one(static_cast<T*>(g.o) + (st.span.begin + flat / g.group) * g.o_stride + (kv * g.group + flat % g.group) * g.head + d,
                    l == 0.0f ? 0.0f : v / l);
      } else {
        slot[r * kWidth + d] = v;
        if (d == 0) {
          float top_r = -INFINITY;
#pragma unroll
          for (int w = 0; w < S::kWaves; ++w) top_r = fmaxf(top_r, peak[w][r]);
          slot[kItem * kWidth + r] = top_r;
          slot[kItem * kWidth + kItem + r] = l;
        }
      }
    }
    __syncthreads();
    if (g.head < kWidth && at < end)  // the results went where the tiles have zeros
      for (int i = lane * 16; i < 4 * S::kTile; i += kWave * 16) *reinterpret_cast<uint4*>(mine + i) = make_uint4(0, 0, 0, 0);
  }
}

constexpr int kMaxParts = 256;  // of a key head's work
__device__ __forceinline__ int up_to_block(int v) { return (v + kBlock - 1) / kBlock * kBlock; }

// Items in several pieces: their results together; and zeros for tokens behind the last sequence.
template <typename T, int DB>
__global__ __launch_bounds__(kBlock) void cached_join_kernel(const CacheArgs g) {
  using S = Shape<T, DB>;
  constexpr int kWidth = DB * 32;
  __shared__ float factors[kMaxParts][kItem], sums[kMaxParts][kItem], total[kItem];
  __shared__ v4f_t halves[kBlock];
  const int kv = blockIdx.y;
  const Found f = find_among(g.sequences, blockIdx.x, [&](int s) { return step_of(g, s, S::kUnit).items; });
  const int seq = uniform(f.seq);
  const int64_t item = int64_t(blockIdx.x) - uniform(f.before);
  if (seq < 0) {
    if (!g.zeros) return;
    const int rest = rest_of(g.offsets, g.sequences, g.tokens);
    for (int i = threadIdx.x; i < kItem * g.head; i += kBlock) {
      const int64_t flat = item * kItem + i / g.head, token = rest + flat / g.group;
      if (token >= g.tokens) break;
      store_one(static_cast<T*>(g.o) + token * g.o_stride + (kv * g.group + flat % g.group) * g.head + i % g.head, 0.0f);
    }
    return;
  }
  const Step st = uniform_step(g, seq, S::kUnit);
  const auto work = [&](int s) {
    const Step each = step_of(g, s, S::kUnit);
    return each.items * each.units;
  };
  const int64_t all = uniform(find_among(g.sequences, INT64_MAX, work).before);
  const int64_t before = uniform(find_among(seq, INT64_MAX, work).before);
  const int parts = used_parts(all, g.parts);
  const int64_t first = before + item * st.units, last = first + st.units - 1;
  const auto part_of = [&](int64_t unit) {
    int p = int(unit * parts / all);
    while (p + 1 < parts && part_begin(all, parts, p + 1) <= unit) ++p;
    while (p > 0 && part_begin(all, parts, p) > unit) --p;
    return p;
  };
  const int p0 = part_of(first), p1 = part_of(last);
  if (p0 == p1) return;  // its part wrote the result
  const int64_t rows = int64_t(st.span.size()) * g.group, row0 = item * kItem;
  const int count = int(rows - row0 < kItem ? rows - row0 : kItem);
  const int pieces_of = p1 - p0 + 1;  // at most kBlock
  // what every piece counts for in every row
  for (int i = threadIdx.x; i < count * pieces_of; i += kBlock) {
    const int r = i % count, p = i / count;
    const float* const slot = slot_at(g, kv, p0 + p, p == 0, kWidth) + kItem * kWidth;
    factors[p][r] = slot[r];
    sums[p][r] = slot[kItem + r];
  }
  __syncthreads();
  if (int(threadIdx.x) < count) {
    const int r = threadIdx.x;
    float top = -INFINITY, l = 0.0f;
    for (int p = 0; p < pieces_of; ++p) top = fmaxf(top, factors[p][r]);
    for (int p = 0; p < pieces_of; ++p) {
      const float f = factors[p][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(factors[p][r] - top);
      factors[p][r] = f;
      l = fmaf(f, sums[p][r], l);
    }
    total[r] = l;
  }
  __syncthreads();
  // four values a thread; where there are few, several threads share the pieces
  constexpr int kFours = kWidth / 4;
  const int fours = count * kFours, shares = fours >= kBlock ? 1 : kBlock / fours;
  for (int i = threadIdx.x; i < up_to_block(fours); i += kBlock) {
    const int share = shares > 1 ? i / fours : 0, at = shares > 1 ? i % fours : i;
    const int r = at / kFours, d = at % kFours * 4;
    v4f_t v = {0, 0, 0, 0};
    if (at < fours && share < shares) {
#pragma unroll 4
      for (int p = share; p < pieces_of; p += shares) {
        const v4f_t x = *reinterpret_cast<const v4f_t*>(slot_at(g, kv, p0 + p, p == 0, kWidth) + r * kWidth + d);
        const float f = factors[p][r];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(f, x[j], v[j]);
      }
    }
    if (shares > 1) {
      halves[threadIdx.x] = v;
      __syncthreads();
      if (share == 0)
        for (int o = 1; o < shares; ++o) v += halves[threadIdx.x + o * fours];
    }
    if (share == 0 && at < fours && d < g.head) {
      const int64_t flat = row0 + r;
      T* const to = static_cast<T*>(g.o) + (st.span.begin + flat / g.group) * g.o_stride + (kv * g.group + flat % g.group) * g.head + d;
      const float inverse = total[r] == 0.0f ? 0.0f : 1.0f / total[r];
      const float f[4] = {v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse};
      if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
      else *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
    }
  }
}

template <typename T, int DB>
void launch_both(const CacheArgs& g, int64_t items, int kv_heads, hipStream_t s) {
  cached_kernel<T, DB><<<dim3(g.parts, kv_heads), Shape<T, DB>::kThreads, 0, s>>>(g);
  cached_join_kernel<T, DB><<<dim3(uint32_t(items), kv_heads), kBlock, 0, s>>>(g);
}
template <typename T>
hipError_t launch(const CacheArgs& g, int64_t items, int kv_heads, hipStream_t s) {
  if (g.head <= 32) launch_both<T, 1>(g, items, kv_heads, s);
  else if (g.head <= 64) launch_both<T, 2>(g, items, kv_heads, s);
  else if (g.head <= 96) launch_both<T, 3>(g, items, kv_heads, s);
  else if (g.head <= 128) launch_both<T, 4>(g, items, kv_heads, s);
  else launch_both<T, 8>(g, items, kv_heads, s);
  return hipGetLastError();
}

int blocks_of_head(int head) { return head <= 32 ? 1 : head <= 64 ? 2 : head <= 96 ? 3 : head <= 128 ? 4 : 8; }

}  // namespace

CachePlan make_cache_plan(const accept_cache_desc& d) {
  CachePlan p{};
  p.items = d.tokens * (d.heads / d.kv_heads) / kItem + d.sequences + 1;
  // as many workgroups as the chip has room for: one a compute unit, more where shared memory takes more
  constexpr int kUnits = 256;
  p.parts = int((kUnits + d.kv_heads - 1) / d.kv_heads);
  static_assert(kUnits <= kMaxParts, "what a row's pieces count for is in shared memory");
  const int width = blocks_of_head(d.head_size) * 32;
  p.bytes = size_t(up_to(int64_t(d.kv_heads) * p.parts * 2 * kItem * (width + 2) * 4, 256));
  return p;
}

hipError_t launch_cache_attention(const accept_cache_desc& d, const CachePlan& p, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* offsets, const int32_t* lengths, const int32_t* table, const uint64_t* tree, void* o,
                                  void* ws, hipStream_t s) {
  CacheArgs g{};
  const int64_t whole = int64_t(d.heads) * d.head_size;
  g.q = q, g.k = k_cache, g.v = v_cache, g.o = o;
  g.parts_at = static_cast<float*>(ws);
  g.offsets = offsets, g.lengths = lengths, g.table = table, g.tree = tree;
  g.q_stride = d.q_stride ? d.q_stride : whole;
  g.o_stride = d.o_stride ? d.o_stride : whole;
  g.pages = {int32_t(d.pages), int32_t(d.table_pages), __builtin_ctz(uint32_t(d.page_size)), d.kv_heads};
  g.sequences = int(d.sequences);
  g.tokens = int(d.tokens);
  g.each = offsets || d.sequences == 0 ? 0 : int(d.tokens / d.sequences);
  g.heads = d.heads;
  g.group = d.heads / d.kv_heads;
  g.head = d.head_size;
  g.parts = p.parts;
  g.tree_words = d.tree_words;
  g.zeros = d.rest == ACCEPT_REST_ZEROS;
  g.scale = float(d.scale * 1.4426950408889634074);
  return d.dtype == ACCEPT_F32 ? launch<float>(g, p.items, d.kv_heads, s) : launch<bf16_t>(g, p.items, d.kv_heads, s);
}

}  // namespace accept
