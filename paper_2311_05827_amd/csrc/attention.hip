// Attention over sequences: one pass over the keys with the running maximum and sum of a softmax.
#include "attention.hpp"

namespace accept {
namespace {

struct AttentionArgs {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  const int32_t* q_offsets;
  const int32_t* k_offsets;
  int64_t q_stride, k_stride, v_stride, o_stride;
  int sequences, q_tokens, k_tokens, q_each, k_each;
  int heads, group, head;
  float* shares;  // [share][heads][q_tokens][width + 2]: sums of values, maximum, sum of weights, where a row's keys are shared out
  int split;      // in so many
  int causal, zeros;
  float scale;    // times log2(e)
};

constexpr int kRows = 128;     // queries of a workgroup, 32 of a wavefront
constexpr int kWaves = 4;
// Sums are taken relative to a maximum that may be this much (in powers of two) behind the true one: results are put to a new
// one only where it grows by more, once or twice a row instead of with every tile.  Sums stay below 2^8 times the
// number of keys, and p has the same relative precision at any size.
constexpr float kBehind = 8.0f;

// A workgroup has 128 queries of a head, a wavefront 32 of them: as columns, so that a lane has a query of its own (its
// maximum, sum and factor are the lane's, two lanes' together) and the weights come out of the first product in the registers that the second one
// takes them from.  Tiles of keys and values come into shared memory one ahead.
//
// Bound by what a SIMD issues: for 64 keys its wavefronts have 32 products of 32 x 32 x 16 (heads of 128) and, beside them, 1024 exponentials with
// scale, sum and rounding, and matrix and vector unit are busy 58 and 59 % of the time, one after the other more than side by side.  16384
// tokens, 16 heads on 2 of 128 in bfloat16: 1.00 to 1.09 ms, 1050 TFLOP/s (the library's 8192^3 product: 1150 to 1390); 8144 tokens in 16 sequences,
// 12 heads of 64: 16 to 18 us, twice what its
// tensors take to go through memory: a workgroup has 8 tiles at most, and its start and end are a good part.  Tried, and slower
// at the first of these: 32 keys at a time with the next scores' products among the exponentials 1160 to 1208 us; 64 queries a wavefront, whose
// registers leave one of them a SIMD, 1733; priority for the wavefront that multiplies 1130; eight wavefronts in two halves that take turns at products and exponentials 1079 to 1116.  All of the keys' parts
// asked for before the first product, instead of each before its own: 1095 us, 1072 so.  In float32 the products are 2 deep and
// are the bound: 4096 tokens, 32 heads of 64, 610 us, 112 TFLOP/s of the 153 that the library's product reaches.
template <typename T, int DB, bool SPLIT>
__global__ __launch_bounds__(kWaves * kWave, groups_a_unit(DB, sizeof(T))) void attention_kernel(const AttentionArgs g) {
  constexpr int NB = sizeof(T) == 2 ? 2 : 1, BN = 32 * NB;
  constexpr int kTile = BN * Head<T, DB>::kRowBytes;
  __shared__ __align__(kTileAlign) uint8_t tiles[4 * kTile];  // keys, values; and the next ones
  const int lane = threadIdx.x % kWave, wave = uniform(int(threadIdx.x / kWave));
  const int half = lane / 32, column = lane % 32;
  const int split = SPLIT ? g.split : 1;
  const HeadPiece hp = deal(blockIdx.x, g.heads * split);
  const int head = SPLIT ? hp.head / split : hp.head, share = SPLIT ? hp.head % split : 0;
  const Piece piece = find_piece(g.q_offsets, g.sequences, g.q_tokens, g.q_each, kRows, hp.index);
  const int seq = piece.seq, tile = piece.tile;
  if (seq < 0) {  // pieces that no sequence has: the tokens behind the last one
    if (!g.zeros || share > 0) return;
    const int rest = rest_of(g.q_offsets, g.sequences, g.q_tokens);
    const int parts = g.head * int(sizeof(T)) / 16;
    for (int i = threadIdx.x; i < kRows * parts; i += kWaves * kWave) {
      const int row = rest + tile * kRows + i / parts;
      if (row >= g.q_tokens) break;
      T* const to = static_cast<T*>(g.o) + row * g.o_stride + int64_t(head) * g.head;
      reinterpret_cast<uint4*>(to)[i % parts] = make_uint4(0, 0, 0, 0);
      if (g.lse && i % parts == 0) g.lse[int64_t(head) * g.q_tokens + row] = -INFINITY;
    }
    return;
  }
  const Span qs = uniform_span(g.q_offsets, seq, g.q_tokens, g.q_each), ks = uniform_span(g.k_offsets, seq, g.k_tokens, g.k_each);
  const int rows = qs.size(), keys = ks.size();
  const int more = keys - rows;  // query i sees keys up to i + more

  const int row0 = tile * kRows + wave * 32, row = row0 + column;
  const bool is_row = row < rows;
  const auto seen_by = [&](int i) { return !g.causal ? keys : i + 1 + more < 0 ? 0 : i + 1 + more; };
  const int last = rows - 1;
  // this lane's query sees keys before it
  const auto limit = [&] {
    const int i = row0 + fresh_lane() % 32;
    return seen_by(i < rows ? i : last);
  };
  const int first_limit = row0 < rows ? seen_by(row0) : 0;    // all of the wavefront's queries do
  const int wave_limit = row0 < rows ? seen_by(row0 + 31 < last ? row0 + 31 : last) : 0;
  const int end = tile * kRows + kRows - 1;
  const int all_steps = pieces(seen_by(end < last ? end : last), BN);
  const int step0 = SPLIT ? int(int64_t(all_steps) * share / split) : 0, steps = SPLIT ? int(int64_t(all_steps) * (share + 1) / split) : all_steps;

  const int parts = g.head * int(sizeof(T)) / 16;
  RowParts<T, DB> q;
  q.load(static_cast<const T*>(g.q) + (qs.begin + (is_row ? row : last)) * g.q_stride + int64_t(head) * g.head, half, parts);
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
  float largest, sum;
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = v16f_t{};
  largest = -INFINITY;
  sum = 0.0f;
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
    v16f_t s[NB];
    float most = -INFINITY;
    const bool masked = key0 + BN > first_limit;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if constexpr (sizeof(T) == 2 && DB <= 4) {  // all of the parts are asked for before the first product
        RowParts<T, DB> parts_of_keys;
        load_parts<T, DB>(parts_of_keys, lds_offset(kt), reader, nb * 32);
        __builtin_amdgcn_sched_barrier(0);
        s[nb] = rows_product<T, DB>(parts_of_keys, q);
      } else {
        s[nb] = rows_product<T, DB>(lds_offset(kt), reader, nb * 32, q);
      }
      if (masked) {
        const int left = limit() - key0 - nb * 32 - fresh_lane() / 32 * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[nb][r] = result_row(r, 0) < left ? s[nb][r] : -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) most = fmaxf(most, s[nb][r]);
    }
    most = halves_max(most) * g.scale;
    if (__any(most > largest + kBehind)) {
      const float now = fmaxf(largest, most);
      const float factor = largest == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(largest - now);
      largest = now;
      sum *= factor;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] *= factor;
    }
    const float base = largest == -INFINITY ? 0.0f : -largest;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(s[nb][r], g.scale, base));
        sum += p[r];
      }
      Weights<T> w;
      set_weights(w, p);
      weighted_rows<T, DB>(acc, lds_offset(vt), reader, nb * 32, w);
    }
  }
  sum = halves_sum(sum);
  // (see of_both_halves; a row whose sum is not finite is NaN whatever its values are)
  const bool bad = of_both_halves(is_row && !finite_column<DB>(acc)) && sum * 0.0f == 0.0f;
  if (__builtin_expect(__any(bad), false)) {
    const AttentionArgs f = fresh_arguments<AttentionArgs>();
    const int lane_now = fresh_lane();
    const Masked masked = masked_keys(first_limit, keys, step0 * BN, steps * BN, BN);
    bool spoiled = false;
    for (int j = masked.unseen + lane_now; j < masked.end; j += kWave) spoiled |= !finite_row(v0 + j * f.v_stride, parts);
    if (__any(spoiled)) {
      const T* const mine = static_cast<const T*>(f.q) + (qs.begin + (is_row ? row : last)) * f.q_stride + int64_t(head) * f.head;
      const float base = largest == -INFINITY ? 0.0f : -largest;
      clear_columns<DB>(acc, bad);
#pragma unroll 1
      for (int key0 = step0 * BN; key0 < masked.first; key0 += 32) {
        const v16f_t s = rows_product_far<T, DB>(k0 + (key0 + lane_now % 32) * f.k_stride, mine, parts);
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = bad ? __builtin_amdgcn_exp2f(fmaf(s[r], f.scale, base)) : 0.0f;
        Weights<T> w;
        set_weights(w, p);
        weighted_rows_far<T, DB>(acc, v0 + key0 * f.v_stride, v0 + (key0 + 16) * f.v_stride, f.v_stride, f.head, w);
      }
      const int stop = wave_limit < masked.end ? wave_limit : masked.end;
#pragma unroll 1
      for (int j = masked.first; j < stop; ++j) {
        const float p = __builtin_amdgcn_exp2f(fmaf(dot_far<T, DB>(mine, k0 + j * f.k_stride, parts), f.scale, base));
        add_row<T, DB>(acc, v0 + j * f.v_stride, p, bad && j < limit(), f.head);
      }
    }
  }
  if (!is_row) return;
  // A row that sees keys, but no score above minus infinity, has no weights: minus infinity less itself.
  const int sees = seen_by(row), stop = sees < steps * BN ? sees : steps * BN;
  const bool lost = sum == 0.0f && stop > step0 * BN;
  const int64_t token = qs.begin + row;
  if constexpr (SPLIT) {
    float* const to = g.shares + ((int64_t(share) * g.heads + head) * g.q_tokens + token) * (DB * 32 + 2);
    store_pairs<DB>(to, acc, half);
    if (half == 0) *reinterpret_cast<float2*>(to + DB * 32) = make_float2(largest, lost ? 1.0f : sum);
    return;
  }
  store_column<T, DB>(static_cast<T*>(g.o) + token * g.o_stride + int64_t(head) * g.head, acc, half, g.head,
                      lost ? NAN : sum == 0.0f ? 0.0f : 1.0f / sum);
  if (g.lse && half == 0)
    g.lse[int64_t(head) * g.q_tokens + token] = sum == 0.0f ? -INFINITY : (largest + __builtin_amdgcn_logf(sum)) * kLn2;
}

// A row's shares together, relative to the largest of their maxima: four values a thread.  (Maximum minus infinity and a sum: a share that sees keys, and
// nothing above that.)
template <typename T, int DB>
__global__ __launch_bounds__(kBlock) void attention_join_kernel(const AttentionArgs g) {
  constexpr int kWidth = DB * 32, kFours = kWidth / 4;
  const int64_t at = int64_t(blockIdx.x) * kBlock + threadIdx.x, row = at / kFours;  // head, token
  const int d = int(at % kFours) * 4;
  if (row >= int64_t(g.heads) * g.q_tokens) return;
  const int head = int(row / g.q_tokens), token = int(row % g.q_tokens);
  if (token >= rest_of(g.q_offsets, g.sequences, g.q_tokens)) return;
  const int64_t apart = int64_t(g.heads) * g.q_tokens * (kWidth + 2);
  const float* const from = g.shares + row * (kWidth + 2);
  float top = -INFINITY;
  for (int p = 0; p < g.split; ++p) top = fmaxf(top, from[p * apart + kWidth]);
  float v[4] = {0, 0, 0, 0}, sum = 0.0f;
  for (int p = 0; p < g.split; ++p) {
    const float peak = from[p * apart + kWidth], factor = peak == -INFINITY ? float(top == -INFINITY) : __builtin_amdgcn_exp2f(peak - top);
    sum = fmaf(factor, from[p * apart + kWidth + 1], sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = fmaf(factor, from[p * apart + d + j], v[j]);
  }
  if (g.lse && d == 0) g.lse[row] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
  if (d >= g.head) return;
  const float inverse = sum == 0.0f ? 0.0f : top == -INFINITY ? NAN : 1.0f / sum;
  T* const to = static_cast<T*>(g.o) + token * g.o_stride + int64_t(head) * g.head + d;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = make_float4(v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse);
  else *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(v[0] * inverse, v[1] * inverse), bf16_pair(v[2] * inverse, v[3] * inverse));
}

template <typename T, int DB>
void launch_head(const AttentionArgs& g, uint32_t groups, hipStream_t s) {
  if (g.split == 1) return attention_kernel<T, DB, false><<<dim3(groups), kWaves * kWave, 0, s>>>(g);
  attention_kernel<T, DB, true><<<dim3(groups * uint32_t(g.split)), kWaves * kWave, 0, s>>>(g);
  attention_join_kernel<T, DB><<<dim3(uint32_t(blocks_of(int64_t(g.heads) * g.q_tokens * DB * 8, kBlock))), kBlock, 0, s>>>(g);
}
template <typename T>
hipError_t launch(const AttentionArgs& g, int64_t tiles, hipStream_t s) {
  const uint32_t groups = uint32_t(g.heads * tiles);
  if (g.head <= 32) launch_head<T, 1>(g, groups, s);
  else if (g.head <= 64) launch_head<T, 2>(g, groups, s);
  else if (g.head <= 96) launch_head<T, 3>(g, groups, s);
  else if (g.head <= 128) launch_head<T, 4>(g, groups, s);
  else launch_head<T, 8>(g, groups, s);
  return hipGetLastError();
}

int64_t tiles_of(const accept_attention_desc& d) { return blocks_of(d.q_tokens, kRows) + d.sequences; }  // of a head: at most so many

}  // namespace

AttentionPlan make_attention_plan(const accept_attention_desc& d) {
  AttentionPlan p{1, 0};
  // A piece's keys are one workgroup's work, one tile after the other, and there are two workgroups a compute unit: where there are fewer, the
  // keys are shared out, as long as a share has some.  (One query over 8192 keys, 8 heads of 128 in bfloat16, 156 us, and 24 so; 4096 tokens,
  // 4 heads, 84 and 40; 1024 tokens, 8 heads, 26 and 23.)
  constexpr int64_t kEnough = 512, kMost = 16, kKeys = 512;
  const int64_t groups = (tiles_of(d) - (d.sequences > 0)) * d.heads, keys = d.sequences > 0 ? blocks_of(d.k_tokens, d.sequences) : 0;
  while (p.split < kMost && groups * p.split * 2 <= kEnough && keys >= kKeys * 2 * p.split) p.split *= 2;
  const int64_t width = d.head_size <= 32 ? 32 : d.head_size <= 64 ? 64 : d.head_size <= 96 ? 96 : d.head_size <= 128 ? 128 : 256;
  if (p.split > 1) p.bytes = size_t(up_to(4 * int64_t(p.split) * d.heads * d.q_tokens * (width + 2), 256));
  return p;
}

hipError_t launch_attention(const accept_attention_desc& d, const AttentionPlan& p, const void* q, const void* k, const void* v,
                            const int32_t* q_offsets, const int32_t* k_offsets, void* o, float* lse, void* ws, hipStream_t s) {
  AttentionArgs g{};
  const int64_t whole = int64_t(d.heads) * d.head_size, kv_whole = int64_t(d.kv_heads) * d.head_size;
  g.q = q;
  g.k = k;
  g.v = v;
  g.o = o;
  g.lse = lse;
  g.shares = static_cast<float*>(ws);
  g.split = p.split;
  g.q_offsets = q_offsets;
  g.k_offsets = k_offsets;
  g.q_stride = d.q_stride ? d.q_stride : whole;
  g.k_stride = d.k_stride ? d.k_stride : kv_whole;
  g.v_stride = d.v_stride ? d.v_stride : kv_whole;
  g.o_stride = d.o_stride ? d.o_stride : whole;
  g.sequences = int(d.sequences);
  g.q_tokens = int(d.q_tokens);
  g.k_tokens = int(d.k_tokens);
  g.q_each = q_offsets || d.sequences == 0 ? 0 : int(d.q_tokens / d.sequences);
  g.k_each = k_offsets || d.sequences == 0 ? 0 : int(d.k_tokens / d.sequences);
  g.heads = d.heads;
  g.group = d.heads / d.kv_heads;
  g.head = d.head_size;
  const int64_t tiles = q_offsets ? tiles_of(d) : d.sequences * blocks_of(g.q_each, kRows);
  g.causal = d.causal;
  g.zeros = d.rest == ACCEPT_REST_ZEROS;
  g.scale = float(d.scale * 1.4426950408889634074);
  return d.dtype == ACCEPT_F32 ? launch<float>(g, tiles, s) : launch<bf16_t>(g, tiles, s);
}

}  // namespace accept
