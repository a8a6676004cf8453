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
  const int64_t* item_sums;  // items in front of every sequence, and in all; units.  Null where a wavefront counts them
  const int64_t* unit_sums;
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

// Rows are columns of the products, as in attention_kernel: a key head's query heads for one token after the other.  An item is so many rows of a
// sequence as a workgroup has at a time, a unit of work so many keys for an item.
//
// Few rows (cached_keys_kernel): an item is 32 rows.  What a wavefront goes through at a time is 32 keys; it keeps the next 32 coming, in shared
// memory of its own, and waits for nobody; in the end the wavefronts' results are put together.
template <typename T, int DB>
struct KeysShape {
  static constexpr int kTile = 32 * Head<T, DB>::kRowBytes;
  static constexpr int kWaves = 4 * kTile * 4 <= 131072 ? 4 : 131072 / (4 * kTile);
  static constexpr int kItem = 32, kUnit = 32 * kWaves, kThreads = kWaves * kWave;
  static constexpr int kSum = DB * 32 * (kItem + 1);  // floats of a wavefront's results, transposed without meeting banks
  static_assert(kSum * 4 <= 4 * kTile, "results take the tiles' place");
};
// Many rows (cached_rows_kernel): an item is 32 rows of each wavefront, 256 where registers allow eight wavefronts, and all of them take the same
// keys, which come into shared memory once, several tiles ahead.
template <typename T, int DB>
struct RowsShape {
  static constexpr int kTile = 32 * Head<T, DB>::kRowBytes;
  static constexpr int kWaves = DB * int(sizeof(T)) <= 8 ? 8 : 4, kItem = 32 * kWaves, kUnit = 128, kThreads = kWaves * kWave;
  static constexpr int kRing = 65536 / kTile < 8 ? 65536 / kTile : 8;  // tiles of keys and of values that are there or on their way
};
// A sequence of the step.
struct Step {
  Span span;
  int length;  // cached tokens
  int keys;    // places that its tokens may see
  int64_t items, units;  // units of every item
};
__device__ __forceinline__ Step step_of(const CacheArgs& g, int seq, int item, int unit) {
  Step s;
  s.span = span_of(g.offsets, seq, g.tokens, g.each);
  const int64_t capacity = g.pages.count > 0 ? int64_t(g.pages.table_pages) << g.pages.shift : 0;
  const int n = s.span.size(), given = g.lengths[seq];
  s.length = given < 0 ? 0 : given;
  const int64_t all = int64_t(s.length) + n;
  s.keys = int(all < capacity ? all : capacity);
  s.items = (int64_t(n) * g.group + item - 1) / item;
  const int64_t units = (int64_t(s.keys) + unit - 1) / unit;
  s.units = units > 0 ? units : 1;
  return s;
}
template <typename S>
__device__ __forceinline__ Step step_of(const CacheArgs& g, int seq) {
  return step_of(g, seq, S::kItem, S::kUnit);
}
template <typename S>
__device__ __forceinline__ Step uniform_step(const CacheArgs& g, int seq) {
  const Step s = step_of<S>(g, seq);
  return {{uniform(s.span.begin), uniform(s.span.end)}, uniform(s.length), uniform(s.keys), uniform(s.items), uniform(s.units)};
}
// Work of a key head, in units one behind the other, is dealt in equal parts.  A part has at most two pieces of items that are not whole: the end of one that
// began before it, and the beginning of one that goes on behind it.
__device__ __forceinline__ int64_t part_begin(int64_t all, int parts, int p) { return quotient(all * p, parts); }
__device__ __forceinline__ int used_parts(int64_t all, int parts) { return all < parts ? int(all) : parts; }
// Floats of a piece's results: rows of sums, their maxima, their sums of weights.
template <typename S>
__device__ __forceinline__ float* slot_at(const CacheArgs& g, int kv, int part, bool begins, int width) {
  constexpr int kItem = S::kItem;
  return g.parts_at + (int64_t(kv) * g.parts + part) * 2 * kItem * (width + 2) + (begins ? kItem * (width + 2) : 0);
}

// Where a part of the work is: the pieces of items that it has, one after the other.
struct Walk {
  int64_t at, end, before;  // units; `before` the sequence's first
  int seq;
};
template <typename S>
__device__ __forceinline__ Walk begin_walk(const CacheArgs& g, int part) {
  const auto work = [&](int s) {
    const Step st = step_of<S>(g, s);
    return st.items * st.units;
  };
  const Index index(g.sequences, g.unit_sums, work);
  const int parts = used_parts(index.total, g.parts);
  if (part >= parts) return {0, 0, 0, 0};
  const int64_t at = part_begin(index.total, parts, part);
  const Found found = index.find(at);
  return {at, part_begin(index.total, parts, part + 1), found.before, found.seq};
}
struct Stretch {
  Step st;
  int64_t item;
  int unit0, unit1;
};
template <typename S>
__device__ __forceinline__ bool next_stretch(const CacheArgs& g, Walk& w, Stretch& s) {
  while (w.at < w.end && w.seq < g.sequences) {
    s.st = uniform_step<S>(g, w.seq);
    const int64_t in = w.at - w.before, all = s.st.items * s.st.units;
    if (in >= all) {
      w.before += all;
      ++w.seq;
      const int64_t* const sums = fresh_argument(&CacheArgs::unit_sums);
      if (sums && w.seq < g.sequences && uniform(sums[w.seq + 1]) <= w.at) {  // (not one by one over those without work)
        w.seq = last_up_to(g.sequences - 1, w.at, [&](int i) { return sums[i]; });
        w.before = uniform(sums[w.seq]);
      }
      continue;
    }
    s.item = quotient(in, s.st.units);
    s.unit0 = int(in - s.item * s.st.units);
    s.unit1 = int(s.st.units - s.unit0 < w.end - w.at ? s.st.units : s.unit0 + (w.end - w.at));
    w.at += s.unit1 - s.unit0;
    return true;
  }
  return false;
}

// What rows row0 .. row0 + count - 1 of a sequence see: a row its token's places, of which all see the first ones and none those from `some` on.
struct Sight {
  int all, some;
};
__device__ __forceinline__ Sight sight_of(const CacheArgs& g, const Step& st, int row0, int count) {
  const int64_t first = int64_t(st.length) + (g.tree_words ? 0 : row0 / g.group + 1);
  const int64_t last = int64_t(st.length) + (row0 + count - 1) / g.group + 1;
  return {uniform(int(first < st.keys ? first : st.keys)), uniform(g.tree_words || last > st.keys ? st.keys : int(last))};
}
// Which of the 32 places from key0 on a token sees: its number in its sequence's new ones, and in all.
__device__ __forceinline__ uint32_t seen_among(const CacheArgs& g, const Step& st, int of_step, int token, int key0) {
  const int64_t sees = int64_t(st.length) + of_step + 1;
  const int limit = g.tree_words ? st.keys : int(sees < st.keys ? sees : st.keys);
  uint32_t seen = bits_between(0, limit - key0);
  if (g.tree_words && st.length - key0 < 32) {
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
}

// The pages of a sequence, 128 of them at a time in two registers of the wavefront: a tile's page is then there at once, and not a trip to memory
// away.
struct Window {
  const int32_t* table;  // of the sequence
  int first, last;       // in the registers; of all
  int low, high;
  __device__ __forceinline__ Window(const CacheArgs& g, const Step& st, int seq)
      : table(g.table + int64_t(seq) * g.pages.table_pages), first(-kReach), last((st.keys - 1) >> g.pages.shift) {}
  static constexpr int kReach = 2 * kWave;
  __device__ __forceinline__ void load(int from) {
    first = from;
    const int lane = fresh_lane(), a = first + lane, b = a + kWave;
    low = table[a < last ? a : last];
    high = table[b < last ? b : last];
    asm volatile("" : "+v"(low), "+v"(high));  // they are waited for here, and not, with all tiles on their way, wherever they are used
  }
  __device__ __forceinline__ int at(int i) const {
    const int in = uniform(i - first);
    return in < kWave ? __builtin_amdgcn_readlane(low, in) : __builtin_amdgcn_readlane(high, in - kWave);
  }
};
// The pages of the 32 places from key0 (a multiple of 32) on, of which the first exists: two at most, a page has 16 places or more.
struct TwoPages {
  int page[2];
};
__device__ __forceinline__ TwoPages pages_of(const CacheArgs& g, const Step& st, Window& window, int key0) {
  const int i = key0 >> g.pages.shift, j = place_at(key0, 16, st.keys) >> g.pages.shift;
  if (j >= window.first + Window::kReach || i < window.first) window.load(i);
  return {window.at(i), window.at(j)};
}
// Those keys and values into tiles, by WAVES wavefronts; places behind the last one give that one again, places that do not exist some of page 0.  Returns which
// of them exist.
template <typename T, int DB, int WAVES, bool ONCE>
__device__ __forceinline__ uint32_t fetch_places(const CacheArgs& g, const Step& st, const TwoPages& two, int kv, int key0, int wave, uint32_t k_to,
                                                 uint32_t v_to) {
  using H = Head<T, DB>;
  constexpr int kPer = 1024 / H::kRowBytes, kAll = 32 / kPer, kLoads = (kAll + WAVES - 1) / WAVES;
  const int row_bytes = g.head * int(sizeof(T)), parts = row_bytes / 16;
  const auto place = [&](int half) { return place_at(key0, 16 * half, st.keys); };
  uint32_t there = 0;
  int64_t first[2];
  int more[2];  // places behind that
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int page = uniform(two.page[h]);
    const bool is = is_page(g.pages, page);
    there |= is ? 0xFFFFu << (16 * h) : 0u;
    first[h] = cache_row(g.pages, is ? page : 0, place(h), kv) * row_bytes;
    more[h] = st.keys - 1 - place(h);
  }
  const int lane = fresh_lane();
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int load = WAVES == 1 ? i : (i * WAVES + wave) % kAll, row = load * kPer, h = row >= 16;
    const int r = row + lane / H::kRowParts, p = lane % H::kRowParts ^ turn<H::kRowBytes>(r);
    const uint32_t offset = uint32_t(r % 16 < more[h] ? r % 16 : more[h]) * uint32_t(row_bytes) + uint32_t(p) * 16u;
    if (p < parts) {
      load_tile_part<ONCE>(static_cast<const uint8_t*>(g.k) + first[h], offset, k_to + load * 1024);
      load_tile_part<ONCE>(static_cast<const uint8_t*>(g.v) + first[h], offset, v_to + load * 1024);
    }
  }
  return there;
}

// The running softmax of 32 rows (a lane's column each) over one tile of 32 keys after the other.
template <typename T, int DB>
struct Rows {
  RowParts<T, DB> q;
  v16f_t acc[DB];
  float largest, sum;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = v16f_t{};
    largest = -INFINITY;
    sum = 0.0f;
  }
  // seen: for columns that do not see all of the tile (then `masked`)
  template <typename Seen>
  __device__ __forceinline__ void take(const uint8_t* kt, const uint8_t* vt, const Reader<T, DB>& reader, float scale, bool masked, const Seen& seen_of) {
    v16f_t s = rows_product<T, DB>(lds_offset(kt), reader, 0, q);
    if (masked) {
      const uint32_t here = seen_of() >> (fresh_lane() / 32 * 4);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = here >> result_row(r, 0) & 1 ? s[r] : -INFINITY;
    }
    float most = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) most = fmaxf(most, s[r]);
    most = halves_max(most) * scale;
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
      p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, base));
      sum += p[r];
    }
    Weights<T> w;
    set_weights(w, p);
    weighted_rows<T, DB>(acc, lds_offset(vt), reader, 0, w);
  }
  // Both halves' sum of weights.  A row that sees keys (of those that `mend` names), but no score above minus infinity, has no weights, as it is minus infinity less
  // itself: with a maximum of minus infinity its sum is 1, that of a row which sees nothing 0.
  template <typename RowOf>
  __device__ __forceinline__ float whole_sum(const Step& st, int seq, int count, const RowOf& row_of, int key, int by, int stop) const {
    float whole = halves_sum(sum);
    const int column = fresh_lane() % 32;
    uint64_t unsure = __ballot(column < count && whole == 0.0f);
    if (__builtin_expect(unsure != 0, false)) {
      const CacheArgs g = fresh_arguments<CacheArgs>();
      const int32_t* const table = g.table + int64_t(seq) * g.pages.table_pages;
      const int of_step = row_of(column) / g.group;
#pragma unroll 1
      for (int ahead = stop - key; ahead > 0 && unsure; ahead -= by) {
        const int key0 = stop - ahead;
        const uint32_t there = (is_page(g.pages, uniform(table[key0 >> g.pages.shift])) ? 0xFFFFu : 0u) |
                               (is_page(g.pages, uniform(table[place_at(key0, 16, st.keys) >> g.pages.shift])) ? 0xFFFF0000u : 0u);
        if (whole == 0.0f && (seen_among(g, st, of_step, st.span.begin + of_step, key0) & there)) whole = 1.0f;
        unsure &= __ballot(whole == 0.0f);
      }
    }
    return whole;
  }
  // Columns that masked rows spoiled (see of_both_halves): row row_of(c) of the sequence each, of which all see the first `all` places that exist.  Tiles as in
  // whole_sum; those with places that do not exist are masked ones too.
  template <typename RowOf>
  __device__ __forceinline__ void mend(const Step& st, int seq, int kv, bool bad, const RowOf& row_of, int all, int key, int by, int stop) {
    const CacheArgs g = fresh_arguments<CacheArgs>();
    const int lane = fresh_lane(), parts = g.head * int(sizeof(T)) / 16, row = row_of(lane % 32), of_step = row / g.group, token = st.span.begin + of_step;
    const T* const mine = static_cast<const T*>(g.q) + token * g.q_stride + int64_t(kv * g.group + row % g.group) * g.head;
    const float base = largest == -INFINITY ? 0.0f : -largest;
    const int32_t* const table = g.table + int64_t(seq) * g.pages.table_pages;
    int64_t first[2];  // the rows of a tile's two halves in the caches, as fetch_places takes them
    const auto look = [&](int key0) {
      uint32_t there = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = place_at(key0, 16 * h, st.keys), page = uniform(table[j >> g.pages.shift]);
        const bool is = is_page(g.pages, page);
        there |= is ? 0xFFFFu << (16 * h) : 0u;
        first[h] = cache_row(g.pages, is ? page : 0, j, kv);
      }
      return there;
    };
    const auto row_at = [&](const void* cache, int key0, int i) {  // of place key0 + i, or the last one
      const int j = place_at(key0, i, st.keys);
      return static_cast<const T*>(cache) + ((i < 16 ? first[0] : first[1]) + (j - place_at(key0, i < 16 ? 0 : 16, st.keys))) * g.head;
    };
    bool spoiled = false;
    for (int ahead = stop - key; ahead > 0; ahead -= by) {
      const int key0 = stop - ahead;
      if (look(key0) != ~0u || all - key0 < 32) spoiled |= !finite_row(row_at(g.v, key0, lane % 32), parts);
    }
    if (!__any(spoiled)) return;
    clear_columns<DB>(acc, bad);
#pragma unroll 1
    for (int ahead = stop - key; ahead > 0; ahead -= by) {
      const int key0 = stop - ahead;
      if (look(key0) != ~0u || all - key0 < 32) continue;
      const v16f_t s = rows_product_far<T, DB>(row_at(g.k, key0, lane % 32), mine, parts);
      float p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = bad ? __builtin_amdgcn_exp2f(fmaf(s[r], g.scale, base)) : 0.0f;
      Weights<T> w;
      set_weights(w, p);
      weighted_rows_far<T, DB>(acc, row_at(g.v, key0, 0), row_at(g.v, key0, 16), g.head, g.head, w);
    }
#pragma unroll 1
    for (int ahead = stop - key; ahead > 0; ahead -= by) {
      const int key0 = stop - ahead;
      const uint32_t there = look(key0);
      if (there == ~0u && all - key0 >= 32) continue;
      const uint32_t seen = seen_among(g, st, of_step, token, key0) & there;
#pragma unroll 1
      for (int i = 0; i < 32; ++i) {
        const bool takes = bad && (seen >> i & 1);
        if (!__any(takes)) continue;
        const float p = __builtin_amdgcn_exp2f(fmaf(dot_far<T, DB>(mine, row_at(g.k, key0, i), parts), g.scale, base));
        add_row<T, DB>(acc, row_at(g.v, key0, i), p, takes, g.head);
      }
    }
  }
};

// Bound by memory where there is enough of it to read: 240000 tokens in 48 sequences, 32 heads on 8 of 128, bfloat16, 160 to 166 us, 5.9 to 6.1 TB/s
// (a copy: 5.2).  With a single sequence of 4001 tokens it is trips to memory one behind the other (the lengths, the table, the tiles: 7.6 us).  Loads with
// the hint that a line is read once took 176 to 164 us off the former.
template <typename T, int DB>
__global__ __launch_bounds__((KeysShape<T, DB>::kThreads), 1) void cached_keys_kernel(const CacheArgs g) {
  using S = KeysShape<T, DB>;
  constexpr int kItem = S::kItem, kWidth = DB * 32, kPad = kItem + 1;
  __shared__ __align__(kTileAlign) uint8_t tiles[S::kWaves][4 * S::kTile];
  __shared__ float peak[S::kWaves][kItem], total[S::kWaves][kItem];
  const int wave = uniform(int(threadIdx.x / kWave));
  const int kv = blockIdx.y, part = blockIdx.x;
  uint8_t* const mine = tiles[wave];
  const auto clear_mine = [&] {
    for (int i = fresh_lane() * 16; i < 4 * S::kTile; i += kWave * 16) *reinterpret_cast<uint4*>(mine + i) = make_uint4(0, 0, 0, 0);
  };
  const Reader<T, DB> lanes(fresh_lane());
  Rows<T, DB> rows;
  Walk walk = begin_walk<S>(g, part);
  Stretch now;
  if (g.head < kWidth) clear_mine();
  while (next_stretch<S>(g, walk, now)) {
    const Step& st = now.st;
    // (rows of a sequence: fewer than 2^28, see the check of the descriptor)
    const int row0 = int(now.item) * kItem, left = st.span.size() * g.group - row0;
    const int count = left < kItem ? left : kItem;
    const auto row_of = [&](int c) { return row0 + (c < count ? c : count - 1); };
    const Sight sight = sight_of(g, st, row0, count);
    {
      const int row = row_of(fresh_lane() % 32), token = st.span.begin + row / g.group, head = kv * g.group + row % g.group;
      rows.q.load(static_cast<const T*>(g.q) + token * g.q_stride + int64_t(head) * g.head, fresh_lane() / 32, g.head * int(sizeof(T)) / 16);
    }
    const int stop = units_end(now.unit1, S::kUnit, sight.some);
    rows.clear();
    Window window(g, st, walk.seq);
    const auto fetch = [&](int key0, int b) {
      const uint32_t to = lds_offset(mine) + uint32_t(b) * 2u * S::kTile;
      return fetch_places<T, DB, 1, true>(g, st, pages_of(g, st, window, key0), kv, key0, 0, to, to + S::kTile);
    };
    int ahead = stop - (now.unit0 * S::kUnit + wave * 32), b = 0;  // places in front of `stop`
    uint32_t there = 0;
    if (ahead > 0) there = fetch(stop - ahead, 0);
    for (; ahead > 0; ahead -= S::kUnit, b ^= 1) {
      const int key0 = stop - ahead;
      wait_for_loads<0>();
      const uint32_t now_there = there;
      if (ahead > S::kUnit) there = fetch(key0 + S::kUnit, b ^ 1);
      const uint8_t* const kt = mine + b * 2 * S::kTile;
      rows.take(kt, kt + S::kTile, lanes.fresh(), g.scale, sight.all - key0 < 32 || now_there != ~0u,
                [&] {
                const int of_step = row_of(fresh_lane() % 32) / g.group;
                return seen_among(g, st, of_step, st.span.begin + of_step, key0) & now_there;
              });
    }
    const int first = now.unit0 * S::kUnit + wave * 32;
    const float sum = rows.whole_sum(st, walk.seq, count, row_of, first, S::kUnit, stop);
    const bool bad = of_both_halves(fresh_lane() % 32 < count && !finite_column<DB>(rows.acc)) && sum * 0.0f == 0.0f;
    if (__builtin_expect(__any(bad), false)) rows.mend(st, walk.seq, kv, bad, row_of, sight.all, first, S::kUnit, stop);

    // the wavefronts' results together, relative to the largest of their maxima (lanes anew: nothing of theirs is kept over the keys)
    const int half = fresh_lane() / 32, column = fresh_lane() % 32;
    if (half == 0) peak[wave][column] = rows.largest;
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < S::kWaves; ++w) top = fmaxf(top, peak[w][column]);
    const float factor = rows.largest == -INFINITY ? float(top == -INFINITY) : __builtin_amdgcn_exp2f(rows.largest - top);
    const bool begins = now.unit0 == 0, ends = now.unit1 == st.units;
    if (half == 0) total[wave][column] = begins && ends && top == -INFINITY && sum != 0.0f ? NAN : sum * factor;
    float* const out = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        out[(db * 32 + result_row(r, half)) * kPad + column] = rows.largest == -INFINITY ? 0.0f : rows.acc[db][r] * factor;
    __syncthreads();
    float* const slot = slot_at<S>(g, kv, part, begins, kWidth);
    for (int i = threadIdx.x; i < count * kWidth; i += S::kThreads) {
      const int r = i / kWidth, d = i % kWidth;
      float v = 0.0f, l = 0.0f;
#pragma unroll
      for (int w = 0; w < S::kWaves; ++w) {
        v += reinterpret_cast<const float*>(tiles[w])[d * kPad + r];
        l += total[w][r];
      }
      if (begins && ends) {
        const int flat = row0 + r;
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
    if (g.head < kWidth && walk.at < walk.end) clear_mine();  // the results went where the tiles have zeros
  }
}

// 55000 tokens in six sequences, trees of 40 with 4 query heads a key head, bfloat16: 109 us.  Bound by waiting: matrix and vector unit are busy 15 and 25 % of the
// time.  Five of a workgroup's eight wavefronts have rows, one SIMD those of two, and all meet at a barrier for every 32 keys, a chain of product, maximum,
// exponential and product apart.
template <typename T, int DB>
__global__ __launch_bounds__((RowsShape<T, DB>::kThreads), 1) void cached_rows_kernel(const CacheArgs g) {
  using S = RowsShape<T, DB>;
  constexpr int kItem = S::kItem, kWidth = DB * 32, kRing = S::kRing;
  __shared__ __align__(kTileAlign) uint8_t tiles[2 * kRing * S::kTile];
  const int wave = uniform(int(threadIdx.x / kWave));
  const int kv = blockIdx.y, part = blockIdx.x;
  const Reader<T, DB> lanes(fresh_lane());
  Rows<T, DB> rows;
  Walk walk = begin_walk<S>(g, part);
  Stretch now;
  if (g.head < kWidth) {
    clear_tiles<2 * kRing * S::kTile, S::kThreads>(tiles);
    __syncthreads();
  }
  while (next_stretch<S>(g, walk, now)) {
    const Step& st = now.st;
    const int item0 = int(now.item) * kItem, row0 = item0 + wave * 32, left = st.span.size() * g.group - row0;
    const int count = left < 0 ? 0 : left < 32 ? left : 32;
    const int item_rows = st.span.size() * g.group - item0, item_count = item_rows < kItem ? item_rows : kItem;
    // (a wavefront without rows of its own takes part with the item's last one)
    const auto row_of = [&](int c) { return count > 0 ? row0 + (c < count ? c : count - 1) : item0 + item_count - 1; };
    const Sight of_item = sight_of(g, st, item0, item_count);
    const Sight sight = count > 0 ? sight_of(g, st, row0, count) : Sight{0, 0};
    {
      const int row = row_of(fresh_lane() % 32), token = st.span.begin + row / g.group, head = kv * g.group + row % g.group;
      rows.q.load(static_cast<const T*>(g.q) + token * g.q_stride + int64_t(head) * g.head, fresh_lane() / 32, g.head * int(sizeof(T)) / 16);
    }
    const int begin = now.unit0 * S::kUnit, stop = units_end(now.unit1, S::kUnit, of_item.some);
    const int steps = begin < stop ? pieces(stop - begin, 32) : 0;
    constexpr int kLoads = 2 * ((32 * Head<T, DB>::kRowBytes / 1024 + S::kWaves - 1) / S::kWaves);  // of a wavefront and step
    rows.clear();
    uint32_t there[kRing];
    Window window(g, st, walk.seq);
    const auto fetch = [&](int step, uint32_t& exists) {
      exists = 0;
      if (step >= steps) return;
      const uint32_t to = lds_offset(tiles) + uint32_t(step % kRing) * 2u * S::kTile;
      const int key0 = begin + step * 32;
      exists = fetch_places<T, DB, S::kWaves, false>(g, st, pages_of(g, st, window, key0), kv, key0, wave, to, to + S::kTile);
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch(i, there[i]);
    for (int step = 0; step < steps; ++step) {
      if (step + kRing - 1 <= steps) wait_for_loads<(kRing - 2) * kLoads>();
      else wait_for_loads<0>();
      __syncthreads();
      fetch(step + kRing - 1, there[kRing - 1]);
      const int key0 = begin + step * 32;
      const uint32_t now_there = there[0];
#pragma unroll
      for (int i = 0; i + 1 < kRing; ++i) there[i] = there[i + 1];
      if (key0 >= sight.some) continue;
      const uint8_t* const kt = tiles + step % kRing * 2 * S::kTile;
      rows.take(kt, kt + S::kTile, lanes.fresh(), g.scale, sight.all - key0 < 32 || now_there != ~0u,
                [&] {
                  const int of_step = row_of(fresh_lane() % 32) / g.group;
                  return seen_among(g, st, of_step, st.span.begin + of_step, key0) & now_there;
                });
    }
    __syncthreads();  // the tiles are free for the next stretch
    const float sum = rows.whole_sum(st, walk.seq, count, row_of, begin, 32, stop);
    const bool bad = of_both_halves(fresh_lane() % 32 < count && !finite_column<DB>(rows.acc)) && sum * 0.0f == 0.0f;
    if (__builtin_expect(__any(bad), false)) rows.mend(st, walk.seq, kv, bad, row_of, sight.all, begin, 32, sight.some < stop ? sight.some : stop);
    const int half = fresh_lane() / 32, column = fresh_lane() % 32;  // (anew: nothing of theirs is kept over the keys)
    if (column >= count) continue;
    const int row = row0 + column, token = st.span.begin + row / g.group, head = kv * g.group + row % g.group;
    const bool begins = now.unit0 == 0, ends = now.unit1 == st.units;
    if (begins && ends) {
      store_column<T, DB>(static_cast<T*>(g.o) + token * g.o_stride + int64_t(head) * g.head, rows.acc, half, g.head,
                         sum == 0.0f ? 0.0f : rows.largest == -INFINITY ? NAN : 1.0f / sum);
    } else {
      float* const slot = slot_at<S>(g, kv, part, begins, kWidth);
      const int r = wave * 32 + column;
      store_column<float, DB>(slot + r * kWidth, rows.acc, half, kWidth, 1.0f);
      if (half == 0) {
        slot[kItem * kWidth + r] = rows.largest;
        slot[kItem * kWidth + kItem + r] = sum;
      }
    }
  }
}

// Items and units in front of every sequence, and in all, for Index: in one workgroup, where there are more than 64 sequences.  (8192 of 5 tokens, one
// new token each, 32 heads on 8 of 128, bfloat16: 1795 us, and 23700 with every wavefront counting all of them, which grows with the square of their number; 65 of 700
// tokens 53 and 56.)
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void cached_sums_kernel(const CacheArgs g, int64_t* item_sums, int64_t* unit_sums, int item, int unit) {
  __shared__ int64_t of_waves[2][kSumThreads / kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int64_t before[2] = {0, 0};
  for (int base = 0; base < g.sequences; base += kSumThreads) {
    const int seq = base + int(threadIdx.x);
    int64_t n[2] = {0, 0}, incl[2];
    if (seq < g.sequences) {
      const Step st = step_of(g, seq, item, unit);
      n[0] = st.items;
      n[1] = st.items * st.units;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      incl[i] = n[i];
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const int64_t up = __shfl_up(incl[i], d, kWave);
        if (lane >= d) incl[i] += up;
      }
      if (lane == kWave - 1) of_waves[i][wave] = incl[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int64_t front = before[i];
      for (int w = 0; w < kSumThreads / kWave; ++w) {
        if (w < wave) front += of_waves[i][w];
        before[i] += of_waves[i][w];
      }
      if (seq < g.sequences) (i ? unit_sums : item_sums)[seq] = front + incl[i] - n[i];
    }
    __syncthreads();
  }
  if (threadIdx.x < 2) (threadIdx.x ? unit_sums : item_sums)[g.sequences] = before[threadIdx.x];
}

constexpr int kMaxParts = 256;  // of a key head's work
__device__ __forceinline__ int up_to_block(int v) { return (v + kBlock - 1) / kBlock * kBlock; }

// Items in several pieces: their results together; and zeros for tokens behind the last sequence.  All of the pieces' maxima first, then a thread
// four values of some pieces, so that their loads are on their way at once (one sequence of 4001 tokens: 6.7 us; piece after piece 30).
template <typename T, int DB, typename S>
__global__ __launch_bounds__(kBlock) void cached_join_kernel(const CacheArgs g) {
  constexpr int kWidth = DB * 32, kItem = S::kItem, kRows = 32;
  __shared__ float factors[kMaxParts][kRows], sums[kMaxParts][kRows], total[kRows];
  __shared__ v4f_t halves[kBlock];
  const int kv = blockIdx.y, row_in = int(blockIdx.z) * kRows;  // of the item
  const auto items = [&](int s) { return step_of<S>(g, s).items; };
  const Found f = Index(g.sequences, g.item_sums, items).find(blockIdx.x);
  const int seq = f.seq;
  const int64_t item = int64_t(blockIdx.x) - f.before;
  if (seq < 0) {
    if (!g.zeros) return;
    const int rest = rest_of(g.offsets, g.sequences, g.tokens);
    for (int i = threadIdx.x; i < kRows * g.head; i += kBlock) {
      const int64_t flat = item * kItem + row_in + i / g.head, token = rest + flat / g.group;
      if (token >= g.tokens) break;
      store_one(static_cast<T*>(g.o) + token * g.o_stride + (kv * g.group + flat % g.group) * g.head + i % g.head, 0.0f);
    }
    return;
  }
  const Step st = uniform_step<S>(g, seq);
  const auto work = [&](int s) {
    const Step each = step_of<S>(g, s);
    return each.items * each.units;
  };
  const Index index(g.sequences, g.unit_sums, work);
  const int64_t all = index.total, before = index.before(seq);
  const int parts = used_parts(all, g.parts);
  const int64_t first = before + item * st.units, last = first + st.units - 1;
  const auto part_of = [&](int64_t unit) {
    int p = int(quotient(unit * parts, all));
    while (p + 1 < parts && part_begin(all, parts, p + 1) <= unit) ++p;
    while (p > 0 && part_begin(all, parts, p) > unit) --p;
    return p;
  };
  const int p0 = part_of(first), p1 = part_of(last);
  if (p0 == p1) return;  // its part wrote the result
  const int row0 = int(item) * kItem + row_in, left = st.span.size() * g.group - row0;
  const int count = left < kRows ? left : kRows;
  if (count <= 0) return;
  const int pieces_of = p1 - p0 + 1;  // at most kBlock
  // what every piece counts for in every row
  for (int i = threadIdx.x; i < count * pieces_of; i += kBlock) {
    const int r = i % count, p = i / count;
    const float* const slot = slot_at<S>(g, kv, p0 + p, p == 0, kWidth) + kItem * kWidth + row_in;
    factors[p][r] = slot[r];
    sums[p][r] = slot[kItem + r];
  }
  __syncthreads();
  if (int(threadIdx.x) < count) {
    const int r = threadIdx.x;
    float top = -INFINITY, l = 0.0f;
    for (int p = 0; p < pieces_of; ++p) top = fmaxf(top, factors[p][r]);
    for (int p = 0; p < pieces_of; ++p) {
      const float f = factors[p][r] == -INFINITY ? float(top == -INFINITY) : __builtin_amdgcn_exp2f(factors[p][r] - top);
      factors[p][r] = f;
      l = fmaf(f, sums[p][r], l);
    }
    total[r] = l != 0.0f && top == -INFINITY ? NAN : l;
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
        const v4f_t x = *reinterpret_cast<const v4f_t*>(slot_at<S>(g, kv, p0 + p, p == 0, kWidth) + (row_in + r) * kWidth + d);
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
      const int flat = row0 + r;
      T* const to = static_cast<T*>(g.o) + (st.span.begin + flat / g.group) * g.o_stride + (kv * g.group + flat % g.group) * g.head + d;
      const float inverse = total[r] == 0.0f ? 0.0f : 1.0f / total[r];
      const float f[4] = {v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse};
      if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
      else *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
    }
  }
}

template <typename T, int DB>
void launch_both(const CacheArgs& g, const CachePlan& p, int kv_heads, hipStream_t s) {
  const dim3 grid(uint32_t(g.parts), uint32_t(kv_heads));
  if (g.item_sums)
    cached_sums_kernel<<<dim3(1), kSumThreads, 0, s>>>(g, const_cast<int64_t*>(g.item_sums), const_cast<int64_t*>(g.unit_sums),
                                                       p.rows ? RowsShape<T, DB>::kItem : KeysShape<T, DB>::kItem,
                                                       p.rows ? RowsShape<T, DB>::kUnit : KeysShape<T, DB>::kUnit);
  if (p.rows) {
    using S = RowsShape<T, DB>;
    cached_rows_kernel<T, DB><<<grid, S::kThreads, 0, s>>>(g);
    cached_join_kernel<T, DB, S><<<dim3(uint32_t(p.items), kv_heads, S::kItem / 32), kBlock, 0, s>>>(g);
  } else {
    using S = KeysShape<T, DB>;
    cached_keys_kernel<T, DB><<<grid, S::kThreads, 0, s>>>(g);
    cached_join_kernel<T, DB, S><<<dim3(uint32_t(p.items), kv_heads), kBlock, 0, s>>>(g);
  }
}
template <typename T>
hipError_t launch(const CacheArgs& g, const CachePlan& p, int kv_heads, hipStream_t s) {
  if (g.head <= 32) launch_both<T, 1>(g, p, kv_heads, s);
  else if (g.head <= 64) launch_both<T, 2>(g, p, kv_heads, s);
  else if (g.head <= 96) launch_both<T, 3>(g, p, kv_heads, s);
  else if (g.head <= 128) launch_both<T, 4>(g, p, kv_heads, s);
  else launch_both<T, 8>(g, p, kv_heads, s);
  return hipGetLastError();
}

int blocks_of_head(int head) { return head <= 32 ? 1 : head <= 64 ? 2 : head <= 96 ? 3 : head <= 128 ? 4 : 8; }

}  // namespace

CachePlan make_cache_plan(const accept_cache_desc& d) {
  CachePlan p{};
  const int64_t rows = d.tokens * (d.heads / d.kv_heads);
  // More than one wavefront's, of a sequence on average: for all of a step's sequences, whatever each has.  (Contexts of 8000, 32 heads on 8 of 128, bfloat16: a chunk of
  // 512 takes 150 us so by itself, 47 single tokens 245 the other way, and both in one step 755 the other way, 127 with the chunk 960.)
  p.rows = rows > 32 * d.sequences;
  const int blocks = blocks_of_head(d.head_size), width = blocks * 32;
  const int item = !p.rows ? 32 : blocks * (d.dtype == ACCEPT_F32 ? 4 : 2) <= 8 ? 256 : 128;  // (as in RowsShape)
  p.items = rows / item + d.sequences + 1;
  // as many workgroups as the chip has room for: one a compute unit, two where few rows of short heads leave room in shared memory
  const int64_t groups = !p.rows && d.dtype == ACCEPT_BF16 && d.head_size <= 64 ? 512 : 256;
  p.parts = int(blocks_of(groups, d.kv_heads) < kMaxParts ? blocks_of(groups, d.kv_heads) : kMaxParts);
  p.sums = size_t(up_to(int64_t(d.kv_heads) * p.parts * 2 * item * (width + 2) * 4, 256));
  p.bytes = p.sums + (d.sequences > kWave ? size_t(up_to(16 * (d.sequences + 1), 256)) : 0);
  return p;
}

hipError_t launch_cache_attention(const accept_cache_desc& d, const CachePlan& p, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* offsets, const int32_t* lengths, const int32_t* table, const uint64_t* tree, void* o,
                                  void* ws, hipStream_t s) {
  CacheArgs g{};
  const int64_t whole = int64_t(d.heads) * d.head_size;
  g.q = q, g.k = k_cache, g.v = v_cache, g.o = o;
  g.parts_at = static_cast<float*>(ws);
  if (d.sequences > kWave) {
    g.item_sums = reinterpret_cast<const int64_t*>(static_cast<const uint8_t*>(ws) + p.sums);
    g.unit_sums = g.item_sums + d.sequences + 1;
  }
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
  return d.dtype == ACCEPT_F32 ? launch<float>(g, p, d.kv_heads, s) : launch<bf16_t>(g, p, d.kv_heads, s);
}

}  // namespace accept
