// Gradients of attention.  The weights are computed again from the scores and the logarithms of the rows' sums; one kernel goes over the
// keys of its queries (dq, and the sums of do * o), a second one over the queries of its keys (dk and dv).  That is seven products
// of tiles where a single kernel would do with five, but each gradient is one workgroup's own sum, in a fixed order: no atomics.
#include "attention.hpp"

#include <type_traits>

namespace accept {
namespace {

struct BackArgs {
  const void* dout;
  const void* q;
  const void* k;
  const void* v;
  const void* o;
  const float* lse;
  float* stats;  // heads x q_tokens: sums of do * o; and then as many lse, times log2(e)
  float* shares; // [share][dk, dv][k_tokens][kv_heads][head], where a key head's queries are shared out
  int split;     // in so many
  float* q_shares;  // [share][q_tokens][heads][head]: dq, where a query's keys are shared out
  int q_split;
  void* dq;
  void* dk;
  void* dv;
  const int32_t* q_offsets;
  const int32_t* k_offsets;
  int64_t q_stride, k_stride, v_stride, o_stride, dq_stride, dk_stride, dv_stride;
  int sequences, q_tokens, k_tokens, q_each, k_each;
  int heads, kv_heads, group, head;
  int causal, zeros;
  float scale, scale2;  // as it is, and times log2(e)
};

constexpr int kRows = 128;  // of a workgroup, 32 of a wavefront
constexpr int kWaves = 4;

// Zeros for this piece of the tokens behind the last sequence.
template <typename T>
__device__ __forceinline__ void clear_rest(T* to, int64_t stride, int head, int first, int tile, int tokens) {
  const int parts = head * int(sizeof(T)) / 16;
  for (int i = threadIdx.x; i < kRows * parts; i += kWaves * kWave) {
    const int row = first + tile * kRows + i / parts;
    if (row >= tokens) break;
    reinterpret_cast<uint4*>(to + row * stride)[i % parts] = make_uint4(0, 0, 0, 0);
  }
}

// dq: 128 queries of a head, a lane has a query of its own as in the forward pass; the sums of do * o, which both kernels need, are made on the way.
// Bound as the forward pass is, with three products of tiles for its two.  12288 tokens in 7 sequences, 32 heads on 8 of 128, bfloat16: 380 to
// 400 us, 860 TFLOP/s of these products.
template <typename T, int DB>
__global__ __launch_bounds__(kWaves * kWave, groups_a_unit(DB, sizeof(T))) void back_queries_kernel(const BackArgs g) {
  constexpr int BN = 32 * (sizeof(T) == 2 && DB <= 4 ? 2 : 1);
  constexpr int kTile = BN * Head<T, DB>::kRowBytes;
  __shared__ __align__(kTileAlign) uint8_t tiles[4 * kTile];
  const int lane = threadIdx.x % kWave, wave = uniform(int(threadIdx.x / kWave));
  const int half = lane / 32, column = lane % 32;
  const HeadPiece hp = deal(blockIdx.x, g.heads * g.q_split);
  const int head = hp.head / g.q_split, share = hp.head % g.q_split;
  const Piece piece = find_piece(g.q_offsets, g.sequences, g.q_tokens, g.q_each, kRows, hp.index);
  T* const dq = static_cast<T*>(g.dq) + int64_t(head) * g.head;
  if (piece.seq < 0) {
    if (g.zeros && share == 0) clear_rest(dq, g.dq_stride, g.head, rest_of(g.q_offsets, g.sequences, g.q_tokens), piece.tile, g.q_tokens);
    return;
  }
  const Span qs = uniform_span(g.q_offsets, piece.seq, g.q_tokens, g.q_each), ks = uniform_span(g.k_offsets, piece.seq, g.k_tokens, g.k_each);
  const int rows = qs.size(), keys = ks.size(), more = keys - rows, last = rows - 1;
  const int row0 = piece.tile * kRows + wave * 32, row = row0 + column;
  const bool is_row = row < rows;
  const auto seen_by = [&](int i) { return !g.causal ? keys : i + 1 + more < 0 ? 0 : i + 1 + more; };
  const auto limit = [&] {
    const int i = row0 + fresh_lane() % 32;
    return seen_by(i < rows ? i : last);
  };
  const int first_limit = row0 < rows ? seen_by(row0) : 0;
  const int wave_limit = row0 < rows ? seen_by(row0 + 31 < last ? row0 + 31 : last) : 0;
  const int end = piece.tile * kRows + kRows - 1;
  const int all_steps = pieces(seen_by(end < last ? end : last), BN);
  const int step0 = int(int64_t(all_steps) * share / g.q_split), steps = int(int64_t(all_steps) * (share + 1) / g.q_split);

  const int parts = g.head * int(sizeof(T)) / 16;
  const int64_t token = qs.begin + (is_row ? row : last);
  RowParts<T, DB> q, dout;
  float along = 0.0f;
  {
    RowParts<T, DB> o;
    dout.load(static_cast<const T*>(g.dout) + token * g.o_stride + int64_t(head) * g.head, half, parts);
    o.load(static_cast<const T*>(g.o) + token * g.o_stride + int64_t(head) * g.head, half, parts);
#pragma unroll
    for (int i = 0; i < Head<T, DB>::kPairs; ++i) {
      constexpr int VEC = 16 / int(sizeof(T));
      float a[VEC], b[VEC];
      widened(Raw<T, VEC>{dout.p[i].x, dout.p[i].y, dout.p[i].z, dout.p[i].w}, a);
      widened(Raw<T, VEC>{o.p[i].x, o.p[i].y, o.p[i].z, o.p[i].w}, b);
#pragma unroll
      for (int j = 0; j < VEC; ++j) along = fmaf(a[j], b[j], along);
    }
    along = halves_sum(along);
  }
  const float lse = g.lse[int64_t(head) * g.q_tokens + token] * kLog2e;
  if (is_row && share == 0) g.stats[(int64_t(half) * g.heads + head) * g.q_tokens + token] = half ? lse : along;
  q.load(static_cast<const T*>(g.q) + token * g.q_stride + int64_t(head) * g.head, half, parts);

  const T* const k0 = uniform(static_cast<const T*>(g.k) + ks.begin * g.k_stride + int64_t(head / g.group) * g.head);
  const T* const v0 = uniform(static_cast<const T*>(g.v) + ks.begin * g.v_stride + int64_t(head / g.group) * g.head);
  const TileRows<T, DB, BN, kWaves> k_rows(wave, g.k_stride, parts), v_rows(wave, g.v_stride, parts);
  const auto fetch = [&](int step) {
    uint8_t* const to = tiles + step % 2 * 2 * kTile;
    k_rows.fetch(k0 + int64_t(step) * BN * g.k_stride, keys - step * BN, to);
    v_rows.fetch(v0 + int64_t(step) * BN * g.v_stride, keys - step * BN, to + kTile);
  };
  if (g.head < DB * 32) {
    clear_tiles<4 * kTile, kWaves * kWave>(tiles);
    __syncthreads();
  }
  const Reader<T, DB> lanes(lane);
  v16f_t acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = v16f_t{};
  if (step0 < steps) fetch(step0);
  for (int step = step0; step < steps; ++step) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (step + 1 < steps) fetch(step + 1);
    const int key0 = step * BN;
    if (key0 >= wave_limit) continue;
    const uint8_t* const kt = tiles + step % 2 * 2 * kTile;
    const uint8_t* const vt = kt + kTile;
    const Reader<T, DB> reader = lanes.fresh();
    const bool masked = key0 + BN > first_limit;
#pragma unroll
    for (int n = 0; n < BN; n += 32) {
      const v16f_t s = rows_product<T, DB>(lds_offset(kt), reader, n, q);
      const v16f_t dp = rows_product<T, DB>(lds_offset(vt), reader, n, dout);
      float ds[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], g.scale2, -lse)) * (dp[r] - along);
      if (masked) {
        const int left = limit() - key0 - n - fresh_lane() / 32 * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = result_row(r, 0) < left ? ds[r] : 0.0f;
      }
      Weights<T> w;
      set_weights(w, ds);
      weighted_rows<T, DB>(acc, lds_offset(kt), reader, n, w);
    }
  }
  const bool bad = of_both_halves(is_row && !finite_column<DB>(acc)) && lse == lse;  // (as in attention_kernel)
  if (__builtin_expect(__any(bad), false)) {
    const BackArgs f = fresh_arguments<BackArgs>();
    const int lane_now = fresh_lane();
    const Masked masked = masked_keys(first_limit, keys, step0 * BN, steps * BN, BN);
    bool spoiled = false;
    for (int j = masked.unseen + lane_now; j < masked.end; j += kWave) spoiled |= !finite_row(k0 + j * f.k_stride, parts);
    if (__any(spoiled)) {
      const int64_t at = qs.begin + (is_row ? row : last);
      const T* const q_row = static_cast<const T*>(f.q) + at * f.q_stride + int64_t(head) * f.head;
      const T* const do_row = static_cast<const T*>(f.dout) + at * f.o_stride + int64_t(head) * f.head;
      clear_columns<DB>(acc, bad);
#pragma unroll 1
      for (int key0 = step0 * BN; key0 < masked.first; key0 += 32) {
        const int j = key0 + lane_now % 32;
        const v16f_t s = rows_product_far<T, DB>(k0 + j * f.k_stride, q_row, parts);
        const v16f_t dp = rows_product_far<T, DB>(v0 + j * f.v_stride, do_row, parts);
        float ds[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = bad ? __builtin_amdgcn_exp2f(fmaf(s[r], f.scale2, -lse)) * (dp[r] - along) : 0.0f;
        Weights<T> w;
        set_weights(w, ds);
        weighted_rows_far<T, DB>(acc, k0 + key0 * f.k_stride, k0 + (key0 + 16) * f.k_stride, f.k_stride, f.head, w);
      }
      const int stop = wave_limit < masked.end ? wave_limit : masked.end;
#pragma unroll 1
      for (int j = masked.first; j < stop; ++j) {
        const float p = __builtin_amdgcn_exp2f(fmaf(dot_far<T, DB>(q_row, k0 + j * f.k_stride, parts), f.scale2, -lse));
        const float ds = p * (dot_far<T, DB>(do_row, v0 + j * f.v_stride, parts) - along);
        add_row<T, DB>(acc, k0 + j * f.k_stride, ds, bad && j < limit(), f.head);
      }
    }
  }
  if (!is_row) return;
  if (g.q_split > 1)
    store_column<float, DB>(g.q_shares + ((int64_t(share) * g.q_tokens + token) * g.heads + head) * g.head, acc, half, g.head, g.scale);
  else
    store_column<T, DB>(dq + token * g.dq_stride, acc, half, g.head, g.scale);
}

// dk and dv: 128 keys of a key head, a lane has a key of its own; tiles of 32 queries and their do come through shared memory, head after
// head of those that share the key head.  Wide heads in bfloat16 leave their values in shared memory: with both gradients' sums and the
// keys in registers there are two wavefronts a SIMD then, one of which multiplies while the other one exponentiates.  (12288 tokens in 7 sequences, 32
// heads on 8 of 128, bfloat16: 490 to 520 us, four products of tiles at 800 to 900 TFLOP/s; with the values in registers and one wavefront a SIMD
// 875.  All of a tile's parts asked for before its first product, instead of each before its own: all gradients 993 us, 972 so.)
// Heads of 256 have registers for one of the two gradients (K: dk, V: dv), and a launch for each.
template <typename T, int DB, bool K, bool V>
__global__ __launch_bounds__(kWaves * kWave, sizeof(T) == 2 && DB <= 4 ? 2 : 1) void back_keys_kernel(const BackArgs g) {
  constexpr int BM = 32;
  constexpr int kTile = BM * Head<T, DB>::kRowBytes;
  constexpr bool kValuesInLds = sizeof(T) == 2 && (DB == 3 || DB == 4);
  __shared__ __align__(kTileAlign) uint8_t tiles[4 * kTile + (kValuesInLds ? kRows * Head<T, DB>::kRowBytes : 0)];
  __shared__ __align__(16) float stats[2][2][BM];
  const int lane = threadIdx.x % kWave, wave = uniform(int(threadIdx.x / kWave));
  const int half = lane / 32, column = lane % 32;
  const HeadPiece hp = deal(blockIdx.x, g.kv_heads * g.split);
  const int head = hp.head / g.split, share = hp.head % g.split;
  Piece piece = find_piece(g.k_offsets, g.sequences, g.k_tokens, g.k_each, kRows, hp.index);
  if (piece.seq >= 0)  // the first keys have most queries
    piece.tile = pieces(uniform_span(g.k_offsets, piece.seq, g.k_tokens, g.k_each).size(), kRows) - 1 - piece.tile;
  T* const dk = static_cast<T*>(g.dk) + int64_t(head) * g.head;
  T* const dv = static_cast<T*>(g.dv) + int64_t(head) * g.head;
  if (piece.seq < 0) {
    if (g.zeros && share == 0) {
      const int rest = rest_of(g.k_offsets, g.sequences, g.k_tokens);
      if constexpr (K) clear_rest(dk, g.dk_stride, g.head, rest, piece.tile, g.k_tokens);
      if constexpr (V) clear_rest(dv, g.dv_stride, g.head, rest, piece.tile, g.k_tokens);
    }
    return;
  }
  const Span qs = uniform_span(g.q_offsets, piece.seq, g.q_tokens, g.q_each), ks = uniform_span(g.k_offsets, piece.seq, g.k_tokens, g.k_each);
  const int rows = qs.size(), keys = ks.size(), more = keys - rows, last = keys - 1;
  const int key0 = piece.tile * kRows + wave * 32, key = key0 + column;
  // the first query that sees a key
  const auto seen_from = [&](int j) { return !g.causal || j - more < 0 ? 0 : j - more; };
  const int wave_from = seen_from(key0), wave_all = seen_from(key0 + 31);
  const int first = seen_from(piece.tile * kRows) / BM;  // tile of queries
  const int each = pieces(rows, BM) - first > 0 ? pieces(rows, BM) - first : 0;
  const int steps = each * g.group, step = int(int64_t(steps) * share / g.split), step_end = int(int64_t(steps) * (share + 1) / g.split);

  const int parts = g.head * int(sizeof(T)) / 16;
  const int64_t token = ks.begin + (key < keys ? key : last);
  if (g.head < DB * 32) {
    clear_tiles<int(sizeof(tiles)), kWaves * kWave>(tiles);
    __syncthreads();
  }
  uint8_t* const values = tiles + 4 * kTile;
  RowParts<T, DB> k, v;
  if constexpr (kValuesInLds) {
    const TileRows<T, DB, kRows, kWaves> v_rows(wave, g.v_stride, parts);
    v_rows.fetch(static_cast<const T*>(g.v) + (ks.begin + int64_t(piece.tile) * kRows) * g.v_stride + int64_t(head) * g.head,
                 keys - piece.tile * kRows, values);
  } else if constexpr (K) {
    v.load(static_cast<const T*>(g.v) + token * g.v_stride + int64_t(head) * g.head, half, parts);
  }
  k.load(static_cast<const T*>(g.k) + token * g.k_stride + int64_t(head) * g.head, half, parts);
  const TileRows<T, DB, BM, kWaves> q_rows(wave, g.q_stride, parts), o_rows(wave, g.o_stride, parts);
  const auto fetch = [&](int h, int tile, int b) {
    uint8_t* const to = tiles + b * 2 * kTile;
    const int row = tile * BM;
    const int64_t at = qs.begin + row;
    q_rows.fetch(static_cast<const T*>(g.q) + at * g.q_stride + int64_t(h) * g.head, rows - row, to);
    o_rows.fetch(static_cast<const T*>(g.dout) + at * g.o_stride + int64_t(h) * g.head, rows - row, to + kTile);
    const int lane_now = fresh_lane();
    if (wave < 2 && lane_now < BM)  // the rows' sums of do * o, and their logarithms
      load_tile_word(g.stats + (int64_t(wave) * g.heads + h) * g.q_tokens + at, uint32_t(lane_now < rows - row ? lane_now : rows - row - 1) * 4u,
                     lds_offset(stats[b][wave]));
  };
  const Reader<T, DB> lanes(lane);
  v16f_t sum_k[DB], sum_v[DB];
  const auto add_up = [&] {
#pragma unroll
    for (int db = 0; db < DB; ++db) sum_k[db] = v16f_t{}, sum_v[db] = v16f_t{};
    if (step == step_end) return;
    // from the last queries down: the workgroups of a sequence, which have different first ones, are at the same ones then
    const int tile_last = first + each - 1;
    int h = head * g.group + step / each, tile = tile_last - step % each, left = step_end - step, b = 0;
    fetch(h, tile, 0);
    while (left > 0) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      const int row0 = tile * BM;
      const uint8_t* const qt = tiles + b * 2 * kTile;
      const uint8_t* const ot = qt + kTile;
      const float* const stat = stats[b][0] + fresh_lane() / 32 * 4;
      if (--tile < first) tile = tile_last, ++h;
      b ^= 1;
      if (--left > 0) fetch(h, tile, b);
      if (row0 + 31 < wave_from || key0 >= keys) continue;
      const bool masked = row0 < wave_all || row0 + 32 > rows || key0 + 32 > keys;
      const Reader<T, DB> reader = lanes.fresh();
      v16f_t s;
      if constexpr (sizeof(T) == 2 && DB <= 4) {  // all of a tile's parts are asked for before the first product
        RowParts<T, DB> a;
        load_parts<T, DB>(a, lds_offset(qt), reader, 0);
        __builtin_amdgcn_sched_barrier(0);
        s = rows_product<T, DB>(a, k);
      } else {
        s = rows_product<T, DB>(lds_offset(qt), reader, 0, k);
      }
      v16f_t dp = {};
      if constexpr (kValuesInLds) dp = rows_product<T, DB>(lds_offset(ot), reader, lds_offset(values) + uint32_t(wave * 32 * Head<T, DB>::kRowBytes));
      else if constexpr (K) dp = rows_product<T, DB>(lds_offset(ot), reader, 0, v);
      float p[16], ds[16];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 sums = *reinterpret_cast<const float4*>(stat + q * 8), logs = *reinterpret_cast<const float4*>(stat + BM + q * 8);
        const float l[4] = {logs.x, logs.y, logs.z, logs.w}, e[4] = {sums.x, sums.y, sums.z, sums.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = 4 * q + j;
          p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], g.scale2, -l[j]));
          ds[r] = p[r] * (dp[r] - e[j]);
        }
      }
      uint32_t seen = ~0u;
      if (masked) {
        const int lane_now = fresh_lane(), j = key0 + lane_now % 32;
        seen = bits_between(seen_from(j < keys ? j : last) - row0, rows - row0);
        const uint32_t here = seen >> (lane_now / 32 * 4);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool sees = here >> result_row(r, 0) & 1;
          p[r] = sees ? p[r] : 0.0f;
          ds[r] = sees ? ds[r] : 0.0f;
        }
      }
      Weights<T> wp, ws;
      set_weights(wp, p);
      set_weights(ws, ds);
      if constexpr (V) weighted_rows<T, DB>(sum_v, lds_offset(ot), reader, 0, wp);
      if constexpr (K) weighted_rows<T, DB>(sum_k, lds_offset(qt), reader, 0, ws);
    }
  };
  add_up();
  // (as in attention_kernel; here masked tiles are of queries: those that some keys are not seen by, and where there are fewer than 32 left)
  const int lane_now = fresh_lane(), key_now = key0 + lane_now % 32;  // (anew: nothing of theirs is kept over the queries)
  const bool bad = of_both_halves(key_now < keys && !((!K || finite_column<DB>(sum_k)) && (!V || finite_column<DB>(sum_v))));
  if (__builtin_expect(__any(bad), false)) {
    const BackArgs f = fresh_arguments<BackArgs>();
    const int j = key_now < keys ? key_now : last, from = seen_from(j);
    const auto tile_of = [&](int i) { return (first + each - 1 - i % each) * BM; };  // its first query
    const auto row_of = [&](const void* x, int64_t stride, int i, int row) {
      return static_cast<const T*>(x) + (qs.begin + row) * stride + int64_t(head * f.group + i / each) * f.head;
    };
    const auto is_masked = [&](int row0) { return row0 < wave_all || row0 + BM > rows; };
    bool spoiled = false;
    for (int i = step; i < step_end; ++i) {  // (a lane for a row of q, one for a row of do)
      const int row0 = tile_of(i), row = row0 + lane_now % 32 < rows ? row0 + lane_now % 32 : rows - 1;
      if (row0 + BM - 1 < wave_from || !is_masked(row0)) continue;
      if (row < wave_all || (row == rows - 1 && row0 + BM > rows))
        spoiled |= !finite_row(lane_now < 32 ? row_of(f.q, f.q_stride, i, row) : row_of(f.dout, f.o_stride, i, row), parts);
    }
    if (__any(spoiled)) {
      const T* const k_row = static_cast<const T*>(f.k) + (ks.begin + j) * f.k_stride + int64_t(head) * f.head;
      const T* const v_row = static_cast<const T*>(f.v) + (ks.begin + j) * f.v_stride + int64_t(head) * f.head;
      const auto again = [&](v16f_t (&sum)[DB], auto of_k) {  // (one gradient after the other: both at a time have no registers)
        constexpr bool kOfK = decltype(of_k)::value;
        clear_columns<DB>(sum, bad);
#pragma unroll 1
        for (int i = step; i < step_end; ++i) {
          const int row0 = tile_of(i);
          if (row0 + BM - 1 < wave_from || is_masked(row0)) continue;
          const int row = row0 + lane_now % 32;
          const float* const e = f.stats + int64_t(head * f.group + i / each) * f.q_tokens + qs.begin + row0 + lane_now / 32 * 4;
          const float* const l = e + int64_t(f.heads) * f.q_tokens;
          const v16f_t s = rows_product_far<T, DB>(row_of(f.q, f.q_stride, i, row), k_row, parts);
          float p[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) p[r] = bad ? __builtin_amdgcn_exp2f(fmaf(s[r], f.scale2, -l[result_row(r, 0)])) : 0.0f;
          if constexpr (kOfK) {
            const v16f_t dp = rows_product_far<T, DB>(row_of(f.dout, f.o_stride, i, row), v_row, parts);
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = bad ? p[r] * (dp[r] - e[result_row(r, 0)]) : 0.0f;
          }
          Weights<T> w;
          set_weights(w, p);
          const void* const x = kOfK ? f.q : f.dout;
          const int64_t stride = kOfK ? f.q_stride : f.o_stride;
          weighted_rows_far<T, DB>(sum, row_of(x, stride, i, row0), row_of(x, stride, i, row0 + 16), stride, f.head, w);
        }
#pragma unroll 1
        for (int i = step; i < step_end; ++i) {
          const int row0 = tile_of(i);
          if (row0 + BM - 1 < wave_from || !is_masked(row0)) continue;
          const float* const e = f.stats + int64_t(head * f.group + i / each) * f.q_tokens + qs.begin;
#pragma unroll 1
          for (int row = row0; row < row0 + BM && row < rows; ++row) {
            const T* const q_row = row_of(f.q, f.q_stride, i, row);
            const T* const do_row = row_of(f.dout, f.o_stride, i, row);
            float w = __builtin_amdgcn_exp2f(fmaf(dot_far<T, DB>(k_row, q_row, parts), f.scale2, -e[int64_t(f.heads) * f.q_tokens + row]));
            if constexpr (kOfK) w *= dot_far<T, DB>(v_row, do_row, parts) - e[row];
            add_row<T, DB>(sum, kOfK ? q_row : do_row, w, bad && row >= from, f.head);
          }
        }
      };
      if constexpr (V) again(sum_v, std::false_type{});
      if constexpr (K) again(sum_k, std::true_type{});
    }
  }
  if (key_now >= keys) return;
  const int64_t token_now = ks.begin + key_now;
  if (g.split > 1) {
    const int64_t whole = int64_t(g.k_tokens) * g.kv_heads * g.head;
    float* const to = g.shares + 2 * share * whole + (token_now * g.kv_heads + head) * g.head;
    if constexpr (K) store_column<float, DB>(to, sum_k, lane_now / 32, g.head, g.scale);
    if constexpr (V) store_column<float, DB>(to + whole, sum_v, lane_now / 32, g.head, 1.0f);
    return;
  }
  if constexpr (K) store_column<T, DB>(dk + token_now * g.dk_stride, sum_k, lane_now / 32, g.head, g.scale);
  if constexpr (V) store_column<T, DB>(dv + token_now * g.dv_stride, sum_v, lane_now / 32, g.head, 1.0f);
}

// The shares' sums, four values a thread, of `tokens` (those of a sequence) of `row_values` each.
template <typename T>
__device__ __forceinline__ void join(const float* shares, int split, int64_t apart, int64_t at, int row_values, T* to, int64_t stride) {
  v4f_t v = {0, 0, 0, 0};
  for (int p = 0; p < split; ++p) v += *reinterpret_cast<const v4f_t*>(shares + p * apart + at);
  to += at / row_values * stride + at % row_values;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<v4f_t*>(to) = v;
  else *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}
template <typename T>
__global__ __launch_bounds__(kBlock) void back_join_kernel(const BackArgs g) {
  const int row_values = g.kv_heads * g.head;
  const int64_t whole = int64_t(g.k_tokens) * row_values, at = (int64_t(blockIdx.x) * kBlock + threadIdx.x) * 4;
  if (at >= whole || at / row_values >= rest_of(g.k_offsets, g.sequences, g.k_tokens)) return;
  join(g.shares, g.split, 2 * whole, at, row_values, static_cast<T*>(g.dk), g.dk_stride);
  join(g.shares + whole, g.split, 2 * whole, at, row_values, static_cast<T*>(g.dv), g.dv_stride);
}
template <typename T>
__global__ __launch_bounds__(kBlock) void back_join_queries_kernel(const BackArgs g) {
  const int row_values = g.heads * g.head;
  const int64_t whole = int64_t(g.q_tokens) * row_values, at = (int64_t(blockIdx.x) * kBlock + threadIdx.x) * 4;
  if (at >= whole || at / row_values >= rest_of(g.q_offsets, g.sequences, g.q_tokens)) return;
  join(g.q_shares, g.q_split, whole, at, row_values, static_cast<T*>(g.dq), g.dq_stride);
}

template <typename T, int DB>
void launch_both(BackArgs g, int q_tiles, int k_tiles, hipStream_t s) {
  constexpr int kThreads = kWaves * kWave;
  if (q_tiles > 0) {
    back_queries_kernel<T, DB><<<dim3(uint32_t(q_tiles) * g.heads * g.q_split), kThreads, 0, s>>>(g);
    if (g.q_split > 1) {
      const int64_t fours = int64_t(g.q_tokens) * g.heads * g.head / 4;
      back_join_queries_kernel<T><<<dim3(uint32_t(blocks_of(fours, kBlock))), kBlock, 0, s>>>(g);
    }
  }
  if (k_tiles > 0) {
    const dim3 grid(uint32_t(k_tiles) * g.kv_heads * g.split);
    if constexpr (DB == 8) {
      back_keys_kernel<T, DB, true, false><<<grid, kThreads, 0, s>>>(g);
      back_keys_kernel<T, DB, false, true><<<grid, kThreads, 0, s>>>(g);
    } else {
      back_keys_kernel<T, DB, true, true><<<grid, kThreads, 0, s>>>(g);
    }
    if (g.split > 1) {
      const int64_t fours = int64_t(g.k_tokens) * g.kv_heads * g.head / 4;
      back_join_kernel<T><<<dim3(uint32_t(blocks_of(fours, kBlock))), kBlock, 0, s>>>(g);
    }
  }
}
template <typename T>
hipError_t launch(const BackArgs& g, int q_tiles, int k_tiles, hipStream_t s) {
  if (g.head <= 32) launch_both<T, 1>(g, q_tiles, k_tiles, s);
  else if (g.head <= 64) launch_both<T, 2>(g, q_tiles, k_tiles, s);
  else if (g.head <= 96) launch_both<T, 3>(g, q_tiles, k_tiles, s);
  else if (g.head <= 128) launch_both<T, 4>(g, q_tiles, k_tiles, s);
  else launch_both<T, 8>(g, q_tiles, k_tiles, s);
  return hipGetLastError();
}

}  // namespace

AttentionBackPlan make_attention_back_plan(const accept_attention_desc& d) {
  AttentionBackPlan p{};
  p.stats = size_t(up_to(8 * int64_t(d.heads) * d.q_tokens, 256));
  // A key tile's queries are one workgroup's work, one after the other, and there are two workgroups a compute unit: below four rounds of
  // those the last ones' queries are shared out.  (12288 tokens in seven sequences, 32 heads on 8: 824 workgroups, the longest with 3.6
  // times the average's work: 718 us; in two shares 521 and 39 for their sums, in four 471 and 76.)
  constexpr int64_t kEnough = 1024, kMost = 16;
  const int64_t groups = (blocks_of(d.k_tokens, kRows) + d.sequences) * d.kv_heads;
  const int64_t queries = d.sequences > 0 ? blocks_of(d.q_tokens, d.sequences) * (d.heads / d.kv_heads) : 0;  // of a key tile
  p.split = 1;
  while (p.split < kMost && groups * p.split < kEnough && queries >= 512 * p.split) p.split *= 2;
  p.bytes = p.stats;
  if (p.split > 1) p.bytes += size_t(up_to(8 * p.split * d.k_tokens * d.kv_heads * d.head_size, 256));
  // The same for the queries' gradients and their keys, below one round of workgroups.  (One sequence of 4096 tokens, 4 heads, all gradients
  // 181 us, and 122 so; a query over 8192 keys, 8 heads, 223 and 44.)
  const int64_t q_groups = blocks_of(d.q_tokens, kRows) * d.heads, keys = d.sequences > 0 ? blocks_of(d.k_tokens, d.sequences) : 0;
  p.q_split = 1;
  while (p.q_split < kMost && q_groups * p.q_split * 2 <= kEnough / 2 && keys >= 1024 * p.q_split) p.q_split *= 2;
  p.q_shares = p.bytes;
  if (p.q_split > 1) p.bytes += size_t(up_to(4 * p.q_split * d.q_tokens * d.heads * d.head_size, 256));
  return p;
}

hipError_t launch_attention_backward(const accept_attention_desc& d, const AttentionBackPlan& p, const void* dout, const void* q,
                                     const void* k, const void* v, const void* o, const float* lse, const int32_t* q_offsets,
                                     const int32_t* k_offsets, void* dq, void* dk, void* dv, void* ws, hipStream_t s) {
  BackArgs g{};
  const int64_t whole = int64_t(d.heads) * d.head_size, kv_whole = int64_t(d.kv_heads) * d.head_size;
  const auto stride = [](int64_t given, int64_t otherwise) { return given ? given : otherwise; };
  g.dout = dout, g.q = q, g.k = k, g.v = v, g.o = o, g.lse = lse;
  g.stats = static_cast<float*>(ws);
  g.shares = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.stats);
  g.split = p.split;
  g.q_shares = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.q_shares);
  g.q_split = p.q_split;
  g.dq = dq, g.dk = dk, g.dv = dv;
  g.q_offsets = q_offsets, g.k_offsets = k_offsets;
  g.q_stride = stride(d.q_stride, whole), g.o_stride = stride(d.o_stride, whole), g.dq_stride = stride(d.dq_stride, whole);
  g.k_stride = stride(d.k_stride, kv_whole), g.v_stride = stride(d.v_stride, kv_whole);
  g.dk_stride = stride(d.dk_stride, kv_whole), g.dv_stride = stride(d.dv_stride, kv_whole);
  g.sequences = int(d.sequences);
  g.q_tokens = int(d.q_tokens);
  g.k_tokens = int(d.k_tokens);
  g.q_each = q_offsets || d.sequences == 0 ? 0 : int(d.q_tokens / d.sequences);
  g.k_each = k_offsets || d.sequences == 0 ? 0 : int(d.k_tokens / d.sequences);
  g.heads = d.heads;
  g.kv_heads = d.kv_heads;
  g.group = d.heads / d.kv_heads;
  g.head = d.head_size;
  g.causal = d.causal;
  g.zeros = d.rest == ACCEPT_REST_ZEROS;
  g.scale = float(d.scale);
  g.scale2 = float(d.scale * 1.4426950408889634074);
  const auto tiles = [&](const int32_t* offsets, int64_t tokens, int64_t each) {
    return int(tokens == 0 ? 0 : offsets ? blocks_of(tokens, kRows) + d.sequences : d.sequences * blocks_of(each, kRows));
  };
  const int q_tiles = tiles(q_offsets, d.q_tokens, g.q_each), k_tiles = tiles(k_offsets, d.k_tokens, g.k_each);
  return d.dtype == ACCEPT_F32 ? launch<float>(g, q_tiles, k_tiles, s) : launch<bf16_t>(g, q_tiles, k_tiles, s);
}

}  // namespace accept
