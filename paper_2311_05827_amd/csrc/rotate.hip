// Rotation of queries and keys by their position, and the way of new keys and values into a cache of pages.
#include "attention.hpp"

namespace accept {
namespace {

// cos and sin of a position's angle.  In turns, as sums of two numbers of 64 bits: the product and what its rounding left, times 1 / (2 pi) and what that one's
// left.  The part of a turn that is left is then off by 2^-53, and by 2^-100 of the whole angle, so by nothing that 32 bits hold, which do from there.
// (In 64 bits alone the angle was off by up to 2^-52 of itself: by 14 steps of 2^-24 at position 2^32 and frequency 1, more at higher ones.)
__device__ __forceinline__ void turn_of(double position, float frequency, float* c, float* s) {
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;
  const double angle = position * double(frequency), angle_rest = fma(position, double(frequency), -angle);
  const double whole = rint(angle * kTurn);
  const double turns = fma(angle, kTurn, -whole) + fma(angle, kTurnRest, angle_rest * kTurn);
  sincospif(float(2.0 * turns), s, c);
}

struct RotateArgs {
  const void* q;      // of append: queries, may be null; of a rotation: the tensor
  const void* k;
  const void* v;
  void* qo;
  void* k_cache;
  void* v_cache;
  const float* frequencies;
  const int32_t* offsets;
  const int32_t* lengths;
  const int32_t* positions;
  const int32_t* table;
  int64_t q_stride, k_stride, v_stride, qo_stride;
  Pages pages;
  int sequences, tokens, each;
  int heads, kv_heads, head;  // heads of q: 0 where there are none
  int half;                   // pairs that turn
  float sign;                 // of the angle
  int zeros;                  // what becomes of tokens without a sequence
  int lanes;                  // items of a head: vectors of pairs, then vectors that are copied
  int pair_lanes;
  int per;                    // heads of a thread: some times kBatch, or 1 where that leaves too few threads
  int turning_chunks, chunks; // groups of heads that turn, and all
};

template <int N>
struct Number {
  static constexpr int value = N;
};

template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, float (&f)[N]) {
  if constexpr (N == 1) {
    f[0] = load_one(p);
  } else {
    const uint4 w = load16(p);
    Raw<T, N> r;
    r.w[0] = w.x, r.w[1] = w.y, r.w[2] = w.z, r.w[3] = w.w;
    widened(r, f);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&f)[N]) {
  if constexpr (N == 1) store_some<T, 1>(p, f);
  else *reinterpret_cast<uint4*>(p) = narrow(f);
}

constexpr int kBatch = 4;
// A thread has the same part of some heads of one token: N pairs (their sines once for all of those heads, whose loads go out together), or 16 bytes that are copied.  Pairs come in
// vectors of 16 bytes (halves: one of each half; neighbours: two behind each other) where those are whole, else one at a time.
// Bound by memory: 20000 tokens, 40 heads of 128 in float32, 64 of them turned by far positions, 159 us at least as a copy's rate goes, and 148 to 159 here.
// (Before heads shared their sines a far position's remainder and its sine were a good part: 161 us there, and 113 instead of 91 for an append of 27000 tokens.)
// CACHE: heads are those of q (if there are any), then of k, into their places; then v's, copied.
template <typename T, int N, bool NEIGHBOURS, bool CACHE>
__global__ __launch_bounds__(kBlock) void rotate_kernel(const RotateArgs g) {
  constexpr int VEC = 16 / int(sizeof(T));
  const int64_t at = (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * kBlock + threadIdx.x;
  const uint32_t per_token = uint32_t(g.lanes) * uint32_t(g.chunks);
  const int64_t all = int64_t(per_token) * g.tokens;
  const bool mine = at < all;
  const int token = !mine ? g.tokens - 1 : all >> 32 == 0 ? int(uint32_t(at) / per_token) : int(at / per_token);
  // the token's sequence, searched for (a wavefront's tokens lie next to each other, so its lanes look at the same offsets)
  int seq = 0, place = token;
  bool outside = false;
  if (!g.offsets) {
    if (g.each > 0) seq = token / g.each, place = token - seq * g.each;
  } else if (CACHE || !g.positions || !g.zeros) {
    int lo = 0, hi = g.sequences;  // the first sequence that ends behind the token
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (g.offsets[mid + 1] > token) hi = mid;
      else lo = mid + 1;
    }
    seq = lo;
    outside = seq >= g.sequences;
    if (!outside) place = token - span_of(g.offsets, seq, g.tokens, 0).begin;
    if (place < 0) outside = true;
  } else {
    outside = token >= rest_of(g.offsets, g.sequences, g.tokens);
  }
  if (!mine) return;
  const uint32_t in_token = uint32_t(at - int64_t(token) * per_token);
  const int chunk = int(in_token / uint32_t(g.lanes)), item = int(in_token) - chunk * g.lanes;
  int length = 0;
  int64_t row = -1;  // of key head 0 in the caches
  if (CACHE && !outside) {
    length = g.lengths[seq] < 0 ? 0 : g.lengths[seq];
    const int64_t j = int64_t(length) + place;
    if (has_place(g.pages, j)) {
      const int page = g.table[int64_t(seq) * g.pages.table_pages + (j >> g.pages.shift)];
      if (is_page(g.pages, page)) row = cache_row(g.pages, page, j, 0);
    }
  }
  const int64_t head_rows = int64_t(1) << g.pages.shift;
  if (outside && (!g.zeros || (CACHE && g.heads == 0))) return;

  if (chunk >= g.turning_chunks) {  // v's heads: CACHE only
    if (outside || row < 0) return;
    const int first = (chunk - g.turning_chunks) * g.per, end = first + g.per < g.kv_heads ? first + g.per : g.kv_heads;
    const T* const v = static_cast<const T*>(g.v) + token * g.v_stride;
    T* const to = static_cast<T*>(g.v_cache);
    for (int h = first; h < end; h += kBatch)
      for (int c = item; c < g.head / VEC; c += g.lanes) {
        uint4 part[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (h + i < end) part[i] = load16(v + (h + i) * g.head + c * VEC);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (h + i < end) *reinterpret_cast<uint4*>(to + (row + (h + i) * head_rows) * g.head + c * VEC) = part[i];
      }
    return;
  }
  const int turning = g.heads + (CACHE ? g.kv_heads : 0);
  const int first = chunk * g.per, end = first + g.per < turning ? first + g.per : turning;
  const bool pair = item < g.pair_lanes;
  float c[N], s[N];
  if (pair && !outside) {
    // (a place may be one that 32 bits do not count: no key goes there, but its query turns)
    const double position = g.positions ? double(g.positions[token]) : double(length) + double(place);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      turn_of(position, g.frequencies[item * N + i], &c[i], &s[i]);
      s[i] *= g.sign;
    }
  }
  // BATCH heads at a time: what they read is asked for before any of it is used
  const auto go = [&](auto batch, int first) {
    constexpr int kHeads = decltype(batch)::value;
    const T* from[kHeads];
    T* to[kHeads];
    bool here[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int h = first + i;
      if (!CACHE || h < g.heads) {
        from[i] = static_cast<const T*>(g.q) + token * g.q_stride + h * g.head;
        to[i] = static_cast<T*>(g.qo) + token * g.qo_stride + h * g.head;
        here[i] = h < end;
      } else {
        from[i] = static_cast<const T*>(g.k) + token * g.k_stride + (h - g.heads) * g.head;
        to[i] = static_cast<T*>(g.k_cache) + (row + (h - g.heads) * head_rows) * g.head;
        here[i] = h < end && row >= 0;
      }
    }
    if (!pair) {
      const int copied = 2 * g.half + (item - g.pair_lanes) * (N == 1 ? 1 : VEC);
      uint4 v[kHeads];
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if constexpr (N == 1) v[i].x = here[i] && !outside ? f32_as_u32(load_one(from[i] + copied)) : 0u;
        else v[i] = here[i] && !outside ? load16(from[i] + copied) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (!here[i]) continue;
        if constexpr (N == 1) store_one(to[i] + copied, u32_as_f32(v[i].x));
        else *reinterpret_cast<uint4*>(to[i] + copied) = v[i];
      }
      return;
    }
    // a pair's first values and its second ones: of halves, or neighbours (N = 1: one pair; else a vector's N / 2, and the next one's)
    const int at_a = NEIGHBOURS ? item * 2 * N : item * N, at_b = NEIGHBOURS ? at_a + N : g.half + item * N;
    float a[kHeads][N], b[kHeads][N];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (!here[i]) continue;
      load_n<T, N>(from[i] + at_a, a[i]);
      load_n<T, N>(from[i] + at_b, b[i]);
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (!here[i]) continue;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        // values j of the two vectors; neighbours: pairs lie inside a vector, and the second vector has the second half of them
        float& x = !NEIGHBOURS || N == 1 ? a[i][j] : j < N / 2 ? a[i][2 * j] : b[i][2 * j - N];
        float& y = !NEIGHBOURS || N == 1 ? b[i][j] : j < N / 2 ? a[i][2 * j + 1] : b[i][2 * j - N + 1];
        const float p = x, q = y;
        x = outside ? 0.0f : fmaf(p, c[j], -(q * s[j]));
        y = outside ? 0.0f : fmaf(p, s[j], q * c[j]);
      }
      store_n<T, N>(to[i] + at_a, a[i]);
      store_n<T, N>(to[i] + at_b, b[i]);
    }
  };
  if (g.per == 1) go(Number<1>{}, first);
  else
    for (int h = first; h < end; h += kBatch) go(Number<kBatch>{}, h);
}

template <typename T, bool CACHE>
hipError_t launch(RotateArgs g, int pairs, hipStream_t s) {
  constexpr int VEC = 16 / int(sizeof(T));
  const bool vectors = g.half % VEC == 0;  // then every vector of a head (a multiple of 8) is whole
  const int n = vectors ? VEC : 1;
  g.pair_lanes = g.half / n;
  g.lanes = g.pair_lanes + (g.head - 2 * g.half) / n;
  const int turning = g.heads + (CACHE ? g.kv_heads : 0);
  // As many threads as keep every compute unit busy, and beyond that kBatch heads each, twice that for a cache, where a thread begins with a trip
  // to memory each for its sequence, its length and its page: 8144 tokens x 16 heads x 64 in bfloat16 10.9 us with a head a thread, 7.2 with four;
  // 16332 tokens x 48 heads x 128 into pages 114 with one, 97 with four, 92 with eight (tensors without a cache: 159 and 162 us for 819 MB).
  const int64_t threads = int64_t(g.tokens) * g.lanes * turning;
  g.per = threads < 65536 * kBatch ? 1 : CACHE && threads >= 8 * 65536 * kBatch ? 2 * kBatch : kBatch;
  g.turning_chunks = int(blocks_of(turning, g.per));
  g.chunks = g.turning_chunks + (CACHE ? int(blocks_of(g.kv_heads, g.per)) : 0);
  const int64_t groups = blocks_of(int64_t(g.tokens) * g.lanes * g.chunks, kBlock);
  const dim3 grid(grid_x(groups), grid_rest(groups));
  if (pairs == ACCEPT_ROTATE_NEIGHBOURS) {
    if (vectors) rotate_kernel<T, VEC, true, CACHE><<<grid, kBlock, 0, s>>>(g);
    else rotate_kernel<T, 1, true, CACHE><<<grid, kBlock, 0, s>>>(g);
  } else {
    if (vectors) rotate_kernel<T, VEC, false, CACHE><<<grid, kBlock, 0, s>>>(g);
    else rotate_kernel<T, 1, false, CACHE><<<grid, kBlock, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const accept_rotate_desc& d, const void* x, const float* frequencies, const int32_t* offsets,
                         const int32_t* positions, void* y, hipStream_t s) {
  RotateArgs g{};
  const int64_t whole = int64_t(d.heads) * d.head_size;
  g.q = x;
  g.qo = y;
  g.frequencies = frequencies;
  g.offsets = offsets;
  g.positions = positions;
  g.q_stride = d.x_stride ? d.x_stride : whole;
  g.qo_stride = d.y_stride ? d.y_stride : whole;
  g.sequences = int(d.sequences);
  g.tokens = int(d.tokens);
  g.each = !offsets && !positions && d.sequences > 0 ? int(d.tokens / d.sequences) : 0;
  g.heads = d.heads;
  g.head = d.head_size;
  g.half = d.rotated / 2;
  g.sign = d.inverse ? -1.0f : 1.0f;
  g.zeros = d.rest == ACCEPT_REST_ZEROS;
  return d.dtype == ACCEPT_F32 ? launch<float, false>(g, d.pairs, s) : launch<bf16_t, false>(g, d.pairs, s);
}

hipError_t launch_cache_append(const accept_cache_desc& d, const void* q, const void* k, const void* v, const float* frequencies,
                               const int32_t* offsets, const int32_t* lengths, const int32_t* positions, const int32_t* table,
                               void* qo, void* k_cache, void* v_cache, hipStream_t s) {
  RotateArgs g{};
  const int64_t whole = int64_t(d.heads) * d.head_size, kv_whole = int64_t(d.kv_heads) * d.head_size;
  g.q = q;
  g.k = k;
  g.v = v;
  g.qo = qo;
  g.k_cache = k_cache;
  g.v_cache = v_cache;
  g.frequencies = frequencies;
  g.offsets = offsets;
  g.lengths = lengths;
  g.positions = positions;
  g.table = table;
  g.q_stride = d.q_stride ? d.q_stride : whole;
  g.k_stride = d.k_stride ? d.k_stride : kv_whole;
  g.v_stride = d.v_stride ? d.v_stride : kv_whole;
  g.qo_stride = d.qo_stride ? d.qo_stride : whole;
  g.pages = {int32_t(d.pages), int32_t(d.table_pages), __builtin_ctz(uint32_t(d.page_size)), d.kv_heads};
  g.sequences = int(d.sequences);
  g.tokens = int(d.tokens);
  g.each = offsets || d.sequences == 0 ? 0 : int(d.tokens / d.sequences);
  g.heads = q ? d.heads : 0;
  g.kv_heads = d.kv_heads;
  g.head = d.head_size;
  g.half = d.rotated / 2;
  g.sign = 1.0f;
  g.zeros = d.rest == ACCEPT_REST_ZEROS;
  return d.dtype == ACCEPT_F32 ? launch<float, true>(g, d.pairs, s) : launch<bf16_t, true>(g, d.pairs, s);
}

}  // namespace accept
