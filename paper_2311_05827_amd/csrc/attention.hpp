// Internal declarations of the attention operators: rotation, attention with its gradients, the cache of pages.
#pragma once

#include "accept_attention.h"
#include "pages.hpp"
#include "stage.hpp"

namespace accept {

constexpr int64_t kMaxTokenStride = int64_t(1) << 22;  // elements: a tile's rows are told apart by 32 bits

hipError_t launch_rotate(const accept_rotate_desc& d, const void* x, const float* frequencies, const int32_t* offsets,
                         const int32_t* positions, void* y, hipStream_t s);
hipError_t launch_cache_append(const accept_cache_desc& d, const void* q, const void* k, const void* v, const float* frequencies,
                               const int32_t* offsets, const int32_t* lengths, const int32_t* positions, const int32_t* table,
                               void* qo, void* k_cache, void* v_cache, hipStream_t s);
struct AttentionPlan {
  int split;     // shares of a row's keys
  size_t bytes;  // workspace: the shares' results
};
AttentionPlan make_attention_plan(const accept_attention_desc& d);
hipError_t launch_attention(const accept_attention_desc& d, const AttentionPlan& p, const void* q, const void* k, const void* v,
                            const int32_t* q_offsets, const int32_t* k_offsets, void* o, float* lse, void* ws, hipStream_t s);
struct AttentionBackPlan {
  int split;        // shares of a key tile's queries
  int q_split;      // shares of a query tile's keys
  size_t stats;     // bytes of the rows' statistics, in front of the shares' sums
  size_t q_shares;  // where those of the queries are
  size_t bytes;
};
AttentionBackPlan make_attention_back_plan(const accept_attention_desc& d);
hipError_t launch_attention_backward(const accept_attention_desc& d, const AttentionBackPlan& p, const void* dout, const void* q,
                                     const void* k, const void* v, const void* o, const float* lse, const int32_t* q_offsets,
                                     const int32_t* k_offsets, void* dq, void* dk, void* dv, void* ws, hipStream_t s);

struct CachePlan {
  bool rows;      // many rows a sequence: items of 128 (see cached_rows_kernel), else of 32
  int64_t items;  // at most so many
  int parts;      // of the work of a key head
  size_t sums;    // in the workspace, behind the parts' results: sums over more sequences than a wavefront counts
  size_t bytes;   // workspace
};
CachePlan make_cache_plan(const accept_cache_desc& d);
hipError_t launch_cache_attention(const accept_cache_desc& d, const CachePlan& p, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* offsets, const int32_t* lengths, const int32_t* table, const uint64_t* tree, void* o,
                                  void* ws, hipStream_t s);

#if defined(__HIPCC__)

__device__ __forceinline__ int pieces(int v, int of) { return (v + of - 1) / of; }

// A value that is the same for all lanes, in a scalar register, and with it what is computed from it.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  return int64_t(uint64_t(uint32_t(uniform(int(v >> 32)))) << 32 | uint32_t(uniform(int(v))));
}

template <typename P>
__device__ __forceinline__ P* uniform(P* p) {
  return reinterpret_cast<P*>(uniform(int64_t(reinterpret_cast<uintptr_t>(p))));
}

// The lane's number, made anew: what is computed from it in a loop takes no register through the loop.  (Loops here fill the registers, and a value
// that does not fit and is loaded from memory waits for all loads in front of it, the next tiles' among them.)
__device__ __forceinline__ int fresh_lane() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// A kernel's argument (its only one) from memory again: for code that is rarely reached, so that nothing of it takes a scalar register through the loops before.
template <typename A>
__device__ __forceinline__ A fresh_arguments() {
  auto at = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  A a;
  __builtin_memcpy(&a, (const void*)at, sizeof(A));
  return a;
}
template <typename A, typename F>
__device__ __forceinline__ F fresh_argument(F A::*field) {  // one of its members
  auto at = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return ((const A*)(const void*)at)->*field;
}

// ---- sequences ---------------------------------------------------------------------------------
// First token and end of a sequence; whatever the offsets hold, inside 0 .. tokens.
struct Span {
  int begin, end;
  __device__ __forceinline__ int size() const { return end - begin; }
};
__device__ __forceinline__ Span span_of(const int32_t* offsets, int s, int tokens, int each) {
  if (!offsets) return {s * each, s * each + each};
  int b = offsets[s], e = offsets[s + 1];
  b = b < 0 ? 0 : b > tokens ? tokens : b;
  e = e < b ? b : e > tokens ? tokens : e;
  return {b, e};
}
__device__ __forceinline__ Span uniform_span(const int32_t* offsets, int s, int tokens, int each) {
  const Span span = span_of(offsets, s, tokens, each);
  return {uniform(span.begin), uniform(span.end)};
}
// The tokens behind the last sequence begin here.
__device__ __forceinline__ int rest_of(const int32_t* offsets, int sequences, int tokens) {
  if (!offsets || sequences == 0) return offsets ? 0 : tokens;
  const int e = offsets[sequences];
  return e < 0 ? 0 : e > tokens ? tokens : e;
}

// The last s of 0 .. count for which value(s) <= at, where value does not fall from one s to the next (0 if there is none); 64 of them at a time.
template <typename F>
__device__ __forceinline__ int last_up_to(int count, int64_t at, const F& value) {
  const int lane = threadIdx.x % kWave;
  int lo = 0, left = count;  // it is one of lo .. lo + left
  while (left > 0) {
    const int step = (left + kWave - 1) / kWave, mine = step * (lane + 1) < left ? step * (lane + 1) : left;
    const int n = __builtin_popcountll(__ballot(value(lo + mine) <= at));
    const int below = step * n < left ? step * n : left, above = step * (n + 1) < left ? step * (n + 1) : left;
    left = n == kWave || above == below ? 0 : above - 1 - below;
    lo += below;
  }
  return uniform(lo);
}
// Where a number is when the sequences have size(s) numbers each, one behind the other: the sequence, and its first number; seq = -1 where there
// are fewer, `before` being how many there are then.  A wavefront counts them together, up to 64 sequences; where there are more, `sums` has what lies in front of each
// and in all.  The same for all lanes.
struct Found {
  int seq;
  int64_t before;
};
struct Index {
  int sequences;
  const int64_t* sums;
  int64_t incl, total;
  template <typename F>
  __device__ __forceinline__ Index(int sequences_, const int64_t* sums_, const F& size) : sequences(sequences_), sums(sums_), incl(0) {
    if (sums) {
      total = uniform(sums[sequences]);
      return;
    }
    const int lane = threadIdx.x % kWave;
    incl = lane < sequences ? int64_t(size(lane)) : 0;
    if (sequences > 1) {
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const int64_t up = __shfl_up(incl, d, kWave);
        if (lane >= d) incl += up;
      }
      total = uniform(__shfl(incl, kWave - 1, kWave));
    } else {
      total = uniform(incl);  // lane 0's
    }
  }
  // what lies in front of a sequence
  __device__ __forceinline__ int64_t before(int seq) const {
    if (sums) return uniform(sums[seq]);
    return seq == 0 ? 0 : uniform(__shfl(incl, seq - 1, kWave));
  }
  __device__ __forceinline__ Found find(int64_t at) const {
    if (at >= total) return {-1, total};
    int seq = 0;
    if (sums) seq = last_up_to(sequences - 1, at, [&](int s) { return sums[s]; });
    else if (sequences > 1) seq = __builtin_ctzll(__ballot(incl > at));
    return {seq, before(seq)};
  }
};
// a / b for a >= 0, b > 0, the same for all lanes; most often short ones
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return int64_t(uniform(int(uint32_t(a) / uint32_t(b))));
  return uniform(a / b);
}

// The same of up to 64 sequences with the longest ones first, so that a launch ends with short pieces of work: 12288 tokens in seven sequences,
// 32 heads, the gradients of keys and values in 793 us in their own order, 718 so; 16 x 509 tokens, 12 heads of 64, forward 28.4 and 22.2.
template <typename F, typename L>
__device__ __forceinline__ Found find_longest_first(int sequences, int64_t at, const F& size, const L& length) {
  const int lane = threadIdx.x % kWave;
  const int n = lane < sequences ? int(size(lane)) : 0, key = lane < sequences ? int(length(lane)) : -1;
  int64_t mine = 0, all = 0;
  for (int j = 0; j < sequences; ++j) {
    const int n_j = __builtin_amdgcn_readlane(n, j), key_j = __builtin_amdgcn_readlane(key, j);
    if (key_j > key || (key_j == key && j < lane)) mine += n_j;
    all += n_j;
  }
  const uint64_t it = __ballot(lane < sequences && mine <= at && at < mine + n);
  if (!it) return {-1, all};
  const int first = __builtin_ctzll(it);
  return {first, __shfl(mine, first, kWave)};
}
// Piece number `index`, heaviest ones first, of sequences that are cut in pieces of `rows` tokens: its sequence, and its place in it with the
// last piece first (seq -1: number `tile` of the pieces of the tokens behind the last sequence, or behind those).
struct Piece {
  int seq, tile;
};
__device__ __forceinline__ Piece find_piece(const int32_t* offsets, int sequences, int tokens, int each, int rows, int index) {
  if (!offsets) {
    const int per = pieces(each, rows);
    return {index % sequences, per - 1 - index / sequences};
  }
  if (sequences > kWave) {
    // More than a look at all of them: sequence s has the numbers from first(s) on, of which there are as many as it has pieces at least (some
    // are nobody's).  1024 sequences of 16 tokens, 32 heads on 8 of 128, forward: 320 us, and 5060 by counting the pieces of those in front, which grows with the
    // square of their number; 65 of 250 122, where counting 64 of 256 takes 178 and gives the order of lengths.
    const auto first = [&](int s) { return span_of(offsets, s, tokens, 0).begin / rows + s; };
    const int rest = rest_of(offsets, sequences, tokens), behind = index - (rest / rows + sequences);
    if (behind >= 0) return {-1, uniform(behind)};
    const int seq = last_up_to(sequences - 1, index, first);
    const Span span = uniform_span(offsets, seq, tokens, 0);
    const int in = index - (span.begin / rows + seq), of = pieces(span.size(), rows);
    if (in < 0 || in >= of) return {-1, tokens / rows + 1};
    return {seq, of - 1 - in};
  }
  const Found f = find_longest_first(sequences, index, [&](int s) { return pieces(span_of(offsets, s, tokens, 0).size(), rows); },
                                     [&](int s) { return span_of(offsets, s, tokens, 0).size(); });
  const int seq = uniform(f.seq), in = int(index - uniform(f.before));
  if (seq < 0) return {-1, in};
  const Span span = uniform_span(offsets, seq, tokens, 0);
  return {seq, pieces(span.size(), rows) - 1 - in};
}

// ---- tiles in shared memory, and products of 32 x 32 ---------------------------------------------
// A tile is rows of ROWB bytes, head_size up to a power of two; a row's 16-byte parts lie in an order of their own, part ^ turn(row), so that
// 16 rows' parts of one number, and four rows' 64 neighbouring bytes (which a transposing read takes), meet no bank twice.
template <int ROWB>
__device__ __forceinline__ int turn(int row) {
  if constexpr (ROWB >= 256) return (row & 3) << 2 | (row >> 2 & 3);
  else if constexpr (ROWB == 128) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
  else return row >> 2 & 3;
}
template <int ROWB>
__device__ __forceinline__ int part_at(int row, int part) { return row * ROWB + ((part ^ turn<ROWB>(row)) << 4); }

typedef float v16f_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// The sum of products over one part of 16 bytes of each operand's rows: lanes 0-31 give row lane of a and column lane of b in the first part
// of a pair, lanes 32-63 in the second.  A lane gets column lane%32 of the result, rows result_row(r): 32 values are as a
// right operand of the next product what they were as a result of this one, as long as its left operand takes the same order.
__device__ __forceinline__ int result_row(int r, int half) { return r / 4 * 8 + half * 4 + r % 4; }
template <typename T>
__device__ __forceinline__ v16f_t multiply_parts(uint4 a, uint4 b, v16f_t c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
  } else {
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(u32_as_f32(a.x), u32_as_f32(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(u32_as_f32(a.y), u32_as_f32(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(u32_as_f32(a.z), u32_as_f32(b.z), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x2f32(u32_as_f32(a.w), u32_as_f32(b.w), c, 0, 0, 0);
  }
}

// Workgroups of four wavefronts that a compute unit has to have room for, where a wavefront goes over keys for its queries: two of heads up to 128, whose sums,
// queries and scores take 199 registers; three of those up to 64 (114 registers, so four; 4096 tokens, 32 heads of 64, forward: two 117 us, more 100).
constexpr int groups_a_unit(int blocks, int bytes) { return bytes == 4 || blocks > 4 ? 1 : blocks <= 2 ? 3 : 2; }

// DB blocks of 32 values of a head (the last ones zeros where head_size is less).
template <typename T, int DB>
struct Head {
  static constexpr int kParts = DB * 32 * int(sizeof(T)) / 16;  // of 16 bytes
  static constexpr int kRowBytes = (DB <= 1 ? 32 : DB <= 2 ? 64 : DB <= 4 ? 128 : 256) * int(sizeof(T));
  static constexpr int kRowParts = kRowBytes / 16;
  static constexpr int kPairs = kParts / 2;
};

// A lane's half of a row: parts 2i + lane/32, from memory (zeros behind head_size, and where there is no row).
template <typename T, int DB>
struct RowParts {
  uint4 p[Head<T, DB>::kPairs];
  __device__ __forceinline__ void load(const T* row, int half, int parts) {
#pragma unroll
    for (int i = 0; i < Head<T, DB>::kPairs; ++i) {
      const int part = 2 * i + half;
      p[i] = part < parts ? load16(row + part * (16 / int(sizeof(T)))) : make_uint4(0, 0, 0, 0);
    }
  }
};

// Where a lane reads in a tile: every other address of a product is this one with some bits turned over, and a constant added.
// Tiles begin at multiples of kTileAlign.
constexpr int kTileAlign = 1024;
typedef const __attribute__((address_space(3))) v4u_t lds_v4u_t;
typedef const __attribute__((address_space(3))) float lds_float_t;
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;
__device__ __forceinline__ uint4 lds_load16(uint32_t at) {
  const v4u_t v = *reinterpret_cast<lds_v4u_t*>(at);
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <typename T, int DB>
struct Reader {
  static constexpr int ROWB = Head<T, DB>::kRowBytes;
  uint32_t row;      // part lane/32 of row lane%32
  uint32_t columns;  // of weighted_rows
  __device__ __forceinline__ explicit Reader(int lane) {
    const int half = lane / 32, column = lane % 32;
    row = uint32_t(part_at<ROWB>(column, half));
    if constexpr (sizeof(T) == 2) columns = uint32_t(part_at<ROWB>(4 * half + lane % 16 / 4, column / 16 * 2 + lane % 4 / 2) + lane % 2 * 8);
    else columns = uint32_t(part_at<ROWB>(4 * half, column / 4) + lane % 4 * 4);
  }
  // Kept as these two: the compiler would keep all of a product's addresses in registers through the loop instead of making them anew.
  __device__ __forceinline__ Reader fresh() const {
    Reader r = *this;
    asm volatile("" : "+v"(r.row), "+v"(r.columns));
    return r;
  }
};

// A tile's 32 rows from its row n on as a left operand.
template <typename T, int DB>
__device__ __forceinline__ void load_parts(RowParts<T, DB>& a, uint32_t tile, const Reader<T, DB>& reader, int n) {
  const uint32_t at = tile + reader.row;
#pragma unroll
  for (int i = 0; i < Head<T, DB>::kPairs; ++i) a.p[i] = lds_load16((at ^ uint32_t(i << 5)) + n * Head<T, DB>::kRowBytes);
}
template <typename T, int DB>
__device__ __forceinline__ v16f_t rows_product(const RowParts<T, DB>& a, const RowParts<T, DB>& b) {
  v16f_t c = {};
#pragma unroll
  for (int i = 0; i < Head<T, DB>::kPairs; ++i) c = multiply_parts<T>(a.p[i], b.p[i], c);
  return c;
}
// 32 rows of a tile (from its row n on, a multiple of 32) times 32 rows in registers: result[row of the tile][row of the registers].
template <typename T, int DB>
__device__ __forceinline__ v16f_t rows_product(uint32_t tile, const Reader<T, DB>& reader, int n, const RowParts<T, DB>& b) {
  v16f_t c = {};
  const uint32_t at = tile + reader.row;
#pragma unroll
  for (int i = 0; i < Head<T, DB>::kPairs; ++i) {
    c = multiply_parts<T>(lds_load16((at ^ uint32_t(i << 5)) + n * Head<T, DB>::kRowBytes), b.p[i], c);
    if (Head<T, DB>::kPairs >= 32 && i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // no more loads ahead: they have no registers
  }
  return c;
}
// The same with the other operand's 32 rows in shared memory too.
template <typename T, int DB>
__device__ __forceinline__ v16f_t rows_product(uint32_t tile, const Reader<T, DB>& reader, uint32_t other) {
  v16f_t c = {};
  const uint32_t at = tile + reader.row, other_at = other + reader.row;
#pragma unroll
  for (int i = 0; i < Head<T, DB>::kPairs; ++i)
    c = multiply_parts<T>(lds_load16(at ^ uint32_t(i << 5)), lds_load16(other_at ^ uint32_t(i << 5)), c);
  return c;
}

// 16 columns (of 32 that this lane's half has 16 of) of a result, as right operand of the next product.
template <typename T>
struct Weights;
template <>
struct Weights<float> {
  float w[16];
};
template <>
struct Weights<bf16_t> {
  bf16x8_t w[2];
};
__device__ __forceinline__ void set_weights(Weights<float>& o, const float (&f)[16]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) o.w[r] = f[r];
}
__device__ __forceinline__ void set_weights(Weights<bf16_t>& o, const float (&f)[16]) {
#pragma unroll
  for (int s = 0; s < 2; ++s)
    o.w[s] = __builtin_bit_cast(bf16x8_t, make_uint4(bf16_pair(f[8 * s], f[8 * s + 1]), bf16_pair(f[8 * s + 2], f[8 * s + 3]),
                                                     bf16_pair(f[8 * s + 4], f[8 * s + 5]), bf16_pair(f[8 * s + 6], f[8 * s + 7])));
}

// 4 rows x 16 columns of 16 bits, transposed: each lane of 16 gives the address of four neighbours, lane i of row i/4 and columns 4*(i%4), and
// gets column i of the four rows.
__device__ __forceinline__ short4_t transposed(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_short4_t*>(at));
}

// acc[value of a head][lane's column] += sum over 32 rows of a tile, from row n (a multiple of 32) on, of x[row][value] * w[row][column].
template <typename T, int DB>
__device__ __forceinline__ void weighted_rows(v16f_t (&acc)[DB], uint32_t tile, const Reader<T, DB>& reader, int n, const Weights<T>& w) {
  constexpr int ROWB = Head<T, DB>::kRowBytes;
  const uint32_t at = tile + reader.columns;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const uint32_t from = at ^ uint32_t(db << 6);
        const short4_t lo = transposed(from + (n + 16 * s) * ROWB), hi = transposed((from ^ 32u) + (n + 16 * s + 8) * ROWB);
        typedef short short8_t __attribute__((ext_vector_type(8)));
        const short8_t a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), w.w[s], acc[db], 0, 0, 0);
      }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t flips = uint32_t(turn<ROWB>(result_row(r, 0))) << 4;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const float a = *reinterpret_cast<lds_float_t*>((at ^ flips ^ uint32_t(db << 7)) + (n + result_row(r, 0)) * ROWB);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.w[r], acc[db], 0, 0, 0);
      }
      if (DB > 4) __builtin_amdgcn_sched_barrier(0);
    }
  }
}
// The lane's column: values result_row of block db, as elements of T in a row, times `factor`.
template <typename T, int DB>
__device__ __forceinline__ void store_column(T* row, const v16f_t (&acc)[DB], int half, int head, float factor) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int value = db * 32 + q * 8 + half * 4;
      if (value >= head) continue;  // (head is a multiple of 8)
      const float f[4] = {acc[db][4 * q] * factor, acc[db][4 * q + 1] * factor, acc[db][4 * q + 2] * factor, acc[db][4 * q + 3] * factor};
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(row + value) = make_float4(f[0], f[1], f[2], f[3]);
      } else {
        *reinterpret_cast<uint2*>(row + value) = make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]));
      }
    }
}
// The same as floats, from an address that is a multiple of 8 bytes.
template <int DB>
__device__ __forceinline__ void store_pairs(float* row, const v16f_t (&acc)[DB], int half) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; r += 2) *reinterpret_cast<float2*>(row + db * 32 + result_row(r, half)) = make_float2(acc[db][r], acc[db][r + 1]);
}
// Not finite anywhere in the values that are stored?
template <int DB>
__device__ __forceinline__ bool finite_column(const v16f_t (&acc)[DB]) {
  float zero = 0.0f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) zero = fmaf(acc[db][r], 0.0f, zero);
  return zero == 0.0f;
}

// Of the two halves of a column (lanes l and l + 32): the larger, the sum.
__device__ __forceinline__ float halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(f32_as_u32(v), f32_as_u32(v), false, false);
  return fmaxf(u32_as_f32(r[0]), u32_as_f32(r[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(f32_as_u32(v), f32_as_u32(v), false, false);
  return u32_as_f32(r[0]) + u32_as_f32(r[1]);
}

// ---- columns that masked rows spoiled ---------------------------------------------------------------
// A masked row has weight zero, and zero times an infinity or NaN of its is NaN.  So where a wavefront's sums are not all finite, and its masked tiles (the few that some of
// its columns do not see all of) hold a row that is not, these columns are made again: over the other tiles by products as before,
// then from the masked tiles' rows one by one, where a lane has its own column's weight and adds its values of a row that the column sees, times that.  Operands come from memory
// here: nothing is kept for it in the registers of the loops, and no other wavefront has to wait.  16384 tokens, 16 heads on 2 of 128, bfloat16: with NaN
// in one token's values, or in one row of do, 1.0 and 3.4 ms, as with none; in all values 6.5 ms forward, in all of do 28 backward.  (Going over the masked tiles
// first, so that only their rows are left to make again, took 1 to 7 % of the time of calls that have no such value.)
__device__ __forceinline__ bool of_both_halves(bool is) {
  const uint64_t lanes = __ballot(is);
  return (uint32_t(lanes) | uint32_t(lanes >> 32)) >> (fresh_lane() % 32) & 1;
}
template <int DB>
__device__ __forceinline__ void clear_columns(v16f_t (&acc)[DB], bool is) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[db][r] = is ? 0.0f : acc[db][r];
}
// Of a wavefront's keys, which are those from `begin` to `end` (both whole tiles of `tile`; places from `keys` on give the last key again): the first one of its masked
// tiles, the first one that some column does not see (the last key, if it is taken for places that no column sees), and the end.
struct Masked {
  int first, unseen, end;
};
__device__ __forceinline__ Masked masked_keys(int all_see, int keys, int begin, int end, int tile) {
  int first = all_see / tile * tile;
  first = first < begin ? begin : first > end ? end : first;
  const int unseen = all_see < first ? first : all_see;
  return {first, end > keys && unseen > keys - 1 ? keys - 1 : unseen, end < keys ? end : keys};
}
// Is a row of `parts` parts finite everywhere?  A row a lane.
template <typename T>
__device__ __forceinline__ bool finite_row(const T* row, int parts) {
  constexpr int VEC = 16 / int(sizeof(T));
  float zero = 0.0f;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    float x[VEC];
    load_vec(row + i * VEC, x);
#pragma unroll
    for (int j = 0; j < VEC; ++j) zero = fmaf(x[j], 0.0f, zero);
  }
  return zero == 0.0f;
}
// rows_product with a lane's row of either operand in memory.
template <typename T, int DB>
__device__ __forceinline__ v16f_t rows_product_far(const T* a, const T* b, int parts) {
  constexpr int VEC = 16 / int(sizeof(T));
  const int half = fresh_lane() / 32;
  v16f_t c = {};
#pragma unroll
  for (int i = 0; i < Head<T, DB>::kPairs; ++i) {
    const int part = 2 * i + half;
    const bool is = part < parts;
    const int at = (is ? part : 0) * VEC;
    const uint4 x = load16(a + at), y = load16(b + at), none = make_uint4(0, 0, 0, 0);
    c = multiply_parts<T>(is ? x : none, is ? y : none, c);
    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // no more loads at a time: they have no registers
  }
  return c;
}
// weighted_rows with the 32 rows in memory: 16 from `low` and 16 from `high` on (the same for all lanes), `stride` elements apart.
template <typename T, int DB>
__device__ __forceinline__ void weighted_rows_far(v16f_t (&acc)[DB], const T* low, const T* high, int64_t stride, int head, const Weights<T>& w) {
  const int lane = fresh_lane(), column = lane % 32;
  const uint32_t mine = uint32_t(lane / 32 * 4) * uint32_t(stride);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const T* const from = uniform(s ? high : low);
    const auto value = [&](int e, int db) {  // (what is behind head_size is not stored: the last value again)
      return load_one(from + result_row(e, 0) * stride + (mine + uint32_t(db * 32 + column < head ? db * 32 + column : head - 1)));
    };
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = value(e, db);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, narrow(f)), w.w[s], acc[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(e, db), w.w[8 * s + e], acc[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
}
// The product of this lane's column and a row that is the same for all lanes; both in memory.
template <typename T, int DB>
__device__ __forceinline__ float dot_far(const T* mine, const T* row, int parts) {
  constexpr int VEC = 16 / int(sizeof(T));
  const int half = fresh_lane() / 32;
  float sum = 0.0f;
#pragma unroll 4
  for (int part = half; part < parts; part += 2) {
    float x[VEC], y[VEC];
    load_vec(mine + part * VEC, x);
    load_vec(row + part * VEC, y);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum = fmaf(x[j], y[j], sum);
  }
  return halves_sum(sum);
}
// Columns that take it: their sums and weight * row.
template <typename T, int DB>
__device__ __forceinline__ void add_row(v16f_t (&acc)[DB], const T* row, float weight, bool takes, int head) {
  const int half = fresh_lane() / 32;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (db * 32 + q * 8 >= head) continue;
      float x[4];
      load_quad(row + db * 32 + q * 8 + half * 4, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[db][4 * q + j] = takes ? fmaf(weight, x[j], acc[db][4 * q + j]) : acc[db][4 * q + j];
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Bits first .. end-1 of 32.
__device__ __forceinline__ uint32_t bits_between(int first, int end) {
  const uint32_t below_end = end >= 32 ? ~0u : end <= 0 ? 0u : (1u << end) - 1u;
  const uint32_t below_first = first >= 32 ? ~0u : first <= 0 ? 0u : (1u << first) - 1u;
  return below_end & ~below_first;
}

// ---- loads straight into shared memory -------------------------------------------------------------
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p));
}
// 16 bytes a lane from base + offset to shared memory, `to` on, lane by lane; lanes that are off load and write nothing.  Nothing waits for it but an
// explicit wait for all loads (the compiler would wait before every read of shared memory).
// ONCE: what no other workgroup reads; it does not stay in the caches.
template <bool ONCE = false>
__device__ __forceinline__ void load_tile_part(const void* base, uint32_t offset, uint32_t to) {
  base = uniform(base);  // (the same for all lanes, whatever register it is in)
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(uniform(int(to))), "v"(offset), "s"(base) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(uniform(int(to))), "v"(offset), "s"(base) : "memory");
}
// The same with 4 bytes a lane.
__device__ __forceinline__ void load_tile_word(const void* base, uint32_t offset, uint32_t to) {
  base = uniform(base);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(uniform(int(to))), "v"(offset), "s"(base) : "memory");
}

// Rows of a tensor into a tile, ROWS of them by WAVES wavefronts: 1024 bytes a wavefront and load.  Rows from `end` on give the last one
// again; they are not used.  Parts behind head_size are not loaded.
template <typename T, int DB, int ROWS, int WAVES>
struct TileRows {
  static constexpr int kRowBytes = Head<T, DB>::kRowBytes, kRowParts = Head<T, DB>::kRowParts;
  static constexpr int kRowsPer = 1024 / kRowBytes, kAll = ROWS / kRowsPer, kLoads = (kAll + WAVES - 1) / WAVES;
  static_assert(kRowsPer >= 1 && ROWS % kRowsPer == 0 && (kAll % WAVES == 0 || kAll < WAVES), "whole loads");
  static constexpr int kStep = kRowsPer * WAVES;      // rows from a load to the next
  static constexpr bool kAlike = kStep % 16 == 0;     // whose parts then lie in the same order
  uint32_t stride;  // bytes
  int wave, parts;
  // (where there are fewer loads than wavefronts some load the same, so that all wait for the same number)
  __device__ __forceinline__ TileRows(int wave_, int64_t stride_elements, int parts_)
      : stride(uint32_t(stride_elements) * uint32_t(sizeof(T))), wave(kAll < WAVES ? wave_ % kAll : wave_), parts(parts_) {}
  __device__ __forceinline__ int row(int i, int lane) const { return (i * WAVES + wave) * kRowsPer + lane / kRowParts; }
  __device__ __forceinline__ int part(int i, int lane) const { return lane % kRowParts ^ turn<kRowBytes>(row(kAlike ? 0 : i, lane)); }
  // rows first .. first + ROWS - 1 behind `base`, of which there are `left`, at least one
  __device__ __forceinline__ void fetch(const void* base, int left, const uint8_t* tile) const {
    const uint32_t to = lds_offset(tile) + uint32_t(wave) * 1024u;
    const int lane = fresh_lane();
    if (kAlike && left >= ROWS && parts == kRowParts) {
      const uint32_t from = uint32_t(row(0, lane)) * stride + uint32_t(part(0, lane)) * 16u;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        load_tile_part(static_cast<const uint8_t*>(base) + uint32_t(i * kStep) * uint64_t(stride), from, to + uint32_t(i * WAVES) * 1024u);
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row(i, lane);
      if (part(i, lane) < parts)
        load_tile_part(base, uint32_t(r < left ? r : left - 1) * stride + uint32_t(part(i, lane)) * 16u, to + uint32_t(i * WAVES) * 1024u);
    }
  }
};
// Waits until no more than N of this wavefront's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_for_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x70 | 0xF00);
  asm volatile("" : : : "memory");
}
// Tiles' parts that no load fills are zeros.
template <int BYTES, int THREADS>
__device__ __forceinline__ void clear_tiles(uint8_t* tiles) {
  for (int i = threadIdx.x * 16; i < BYTES; i += THREADS * 16) *reinterpret_cast<uint4*>(tiles + i) = make_uint4(0, 0, 0, 0);
}

// Workgroups are dealt to the chip's eight dies in turn; a die gets neighbouring heads, all of their pieces, so that the keys and values
// its workgroups read at a time are in its cache.
struct HeadPiece {
  int head, index;
};
__device__ __forceinline__ HeadPiece deal(int id, int heads) {
  constexpr int kDies = 8;
  if (heads % kDies == 0) {
    const int each = heads / kDies, in = id / kDies;
    return {id % kDies * each + in % each, in / each};
  }
  return {id % heads, id / heads};
}

#endif  // __HIPCC__

}  // namespace accept
