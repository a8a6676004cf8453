// The product of two matrices of 8-bit codes with a power-of-two scale for each block of 128 along the contracted axis.
#include "stage.hpp"

namespace accept {
namespace {

typedef int v8i_t __attribute__((ext_vector_type(8)));

struct MatmulArgs {
  const uint8_t* a;
  const uint8_t* b;
  const uint8_t* sa;
  const uint8_t* sb;
  void* y;           // the result, or float32 parts [split][m][n]
  int64_t a_stride, b_stride, y_stride;
  int64_t sa_rows, sb_rows;  // bytes of scales to a block of the contracted axis
  int m, n, k;
  int blocks;        // of the contracted axis
  int splits;
  int sa_shift, sb_shift;    // rows that share a scale: 1 << shift
};

// A block of 128 of the contracted axis for 16 x 16 results.  A lane gives 32 codes of row lane%16 of each operand and gets the results of
// four rows of the first operand, 4*(lane/16) on, in column lane%16.  Which of the 128 columns its 32 codes are does not
// matter as long as it is the same in both operands.  b goes first: a lane's four results then lie next to each other in y.
//
// Results in bfloat16 (EXACT false): one 8-bit matrix instruction, which applies both operands' scales (a byte each per row, one
// of the four in a register).  It adds products in eights, with the bits down to 2^-13 of the largest's leading one, and cuts
// off what is below: at most 2^-10 of the sum of the terms' magnitudes, 1.3e-5 of the result for normally distributed operands and
// 6e-5 for heavy tails (measured), where rounding to bfloat16 is 1.7e-3.
//
// Results in float32 (EXACT true): that would be 100 times a float32's rounding.  The codes are converted to bfloat16, scale
// and all, which is exact (4 bits and a power of two; two values an instruction), and go through four 16-bit matrix
// instructions, which add in float32: 5e-9 and 5e-8 on the same operands, at half the instructions' rate.
typedef __bf16 v8b_t __attribute__((ext_vector_type(8)));
typedef __bf16 v2b_t __attribute__((ext_vector_type(2)));

template <int I>
struct Int {
  static constexpr int value = I;
};
template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(const F& f) {
  if constexpr (I < N) {
    f(Int<I>{});
    unrolled<I + 1, N>(f);
  }
}

template <bool EXACT>
struct Fragment;
template <>
struct Fragment<false> {
  v8i_t codes;
};
template <>
struct Fragment<true> {
  v8b_t values[4];
};

template <int CODE>
__device__ __forceinline__ Fragment<false> fragment_of(v8i_t codes, int, Int<0>) { return {codes}; }
// scale: the byte of an E8M0, which is a float32's exponent field
template <int CODE>
__device__ __forceinline__ Fragment<true> fragment_of(v8i_t codes, int scale, Int<1>) {
  const float f = u32_as_f32(uint32_t(scale) << 23);
  Fragment<true> r;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v2b_t lo, hi;
      if constexpr (CODE == ACCEPT_E4M3) {
        lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * q + h], f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * q + h], f, true);
      } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes[2 * q + h], f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(codes[2 * q + h], f, true);
      }
      r.values[q][4 * h + 0] = lo[0], r.values[q][4 * h + 1] = lo[1];
      r.values[q][4 * h + 2] = hi[0], r.values[q][4 * h + 3] = hi[1];
    }
  }
  return r;
}

template <int ACODE, int BCODE, int SUB_A, int SUB_B>
__device__ __forceinline__ v4f_t multiply(const Fragment<false>& b, const Fragment<false>& a, v4f_t sum, int scale_b, int scale_a) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.codes, a.codes, sum, BCODE, ACODE, SUB_B, scale_b, SUB_A, scale_a);
}
template <int ACODE, int BCODE, int SUB_A, int SUB_B>
__device__ __forceinline__ v4f_t multiply(const Fragment<true>& b, const Fragment<true>& a, v4f_t sum, int, int) {
#pragma unroll
  for (int q = 0; q < 4; ++q) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.values[q], a.values[q], sum, 0, 0, 0);
  return sum;
}

// 16 codes with those from `left` on put to zero, whatever they are.
__device__ __forceinline__ uint4 first_codes(uint4 v, int left) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int here = left - 4 * i;
    w[i] = here >= 4 ? w[i] : here <= 0 ? 0u : w[i] & ((1u << (8 * here)) - 1u);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Four results next to each other.
template <typename TO>
__device__ __forceinline__ void put_four(TO* y, int64_t at, v4f_t v, int left) {
  const float f[4] = {v[0], v[1], v[2], v[3]};
  store_values(y + at, f, left);
}

// ---- many rows: tiles -------------------------------------------------------------------------
// A workgroup has a tile of BM x BN results, its WM x WN wavefronts a part of it each, in registers.  Per block of 128 columns the
// tile's rows of both operands come into shared memory directly from memory (16 bytes a lane, no registers), one block ahead
// of the one that is multiplied; one barrier a block.  A row is 128 bytes there, half of the banks, so its eight
// 16-byte parts lie in an order of their own, part ^ (row % 8), and eight rows' reads meet no bank twice.
template <int BM, int BN, int WM, int WN, int ACODE, int BCODE, typename TO, bool EXACT>
__global__ __launch_bounds__(WM* WN* kWave, 2) void matmul_tile_kernel(const MatmulArgs args) {
  constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
  constexpr int MI = BM / WM / 16, NI = BN / WN / 16;  // 16 x 16 results of a wavefront
  static_assert(MI % 4 == 0 && NI % 4 == 0, "a register holds the scales of four");
  constexpr int kLoads = (BM + BN) / 8 / kWaves;  // of a wavefront and block: 8 rows each
  static_assert(BM / 8 % kWaves == 0 && BN / 8 % kWaves == 0, "a load is of one operand");
  __shared__ __align__(16) uint8_t tile0[(BM + BN) * kQBlock];
  __shared__ __align__(16) uint8_t tile1[(BM + BN) * kQBlock];
  __shared__ uint32_t scales[2][(BM + BN) / 4];

  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  // Workgroups are dealt to the chip's eight dies in turn; a die gets neighbouring tiles, in groups of kGroup rows of tiles, so
  // that what its workgroups read at a time is in its cache.
  constexpr int kDies = 8, kGroup = 8;
  const int tiles_m = (args.m + BM - 1) / BM, tiles_n = (args.n + BN - 1) / BN, tiles = tiles_m * tiles_n;
  const int split = blockIdx.x / tiles;
  int id = blockIdx.x % tiles;
  const int die = id % kDies, each = tiles / kDies, more = tiles % kDies;
  id = die * each + (die < more ? die : more) + id / kDies;
  const int group = id / (kGroup * tiles_n), in_group = id % (kGroup * tiles_n);
  const int group_rows = tiles_m - group * kGroup < kGroup ? tiles_m - group * kGroup : kGroup;
  const int m0 = (group * kGroup + in_group % group_rows) * BM, n0 = in_group / group_rows * BN;
  const int first = int(int64_t(args.blocks) * split / args.splits), last = int(int64_t(args.blocks) * (split + 1) / args.splits);

  // where this lane's loads come from: rows behind the last one give that one again, and are not used
  const int part = (lane % 8) ^ (lane / 8);
  const uint8_t* from[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (i * kWaves + wave) * 8 + lane / 8;
    if (i < BM / 8 / kWaves) {
      const int r = m0 + row < args.m ? m0 + row : args.m - 1;
      from[i] = args.a + r * args.a_stride + part * 16;
    } else {
      const int r = n0 + row - BM < args.n ? n0 + row - BM : args.n - 1;
      from[i] = args.b + r * args.b_stride + part * 16;
    }
  }
  static_assert(BM + BN <= kThreads || (BM + BN) % kThreads == 0, "scales of a block: one byte per thread and turn");
  constexpr int kScaleTurns = (BM + BN + kThreads - 1) / kThreads;
  const uint8_t* scale_from[kScaleTurns];
  int64_t scale_step[kScaleTurns];
  int scale_to[kScaleTurns];
#pragma unroll
  for (int i = 0; i < kScaleTurns; ++i) {
    const int row = i * kThreads + t;
    if (row < BM) {
      const int r = m0 + row < args.m ? m0 + row : args.m - 1;
      scale_from[i] = args.sa + (r >> args.sa_shift);
      scale_step[i] = args.sa_rows;
    } else {
      const int r = n0 + row - BM < args.n ? n0 + row - BM : args.n - 1;
      scale_from[i] = args.sb + (r >> args.sb_shift);
      scale_step[i] = args.sb_rows;
    }
    scale_to[i] = (row / 64 * 16 + row % 16) * 4 + row / 16 % 4;
  }

  uint8_t scale_byte[kScaleTurns];
  auto fetch = [&](int block, uint8_t* tile) {
#pragma unroll
    for (int i = 0; i < kScaleTurns; ++i) scale_byte[i] = scale_from[i][block * scale_step[i]];
    const int64_t col = int64_t(block) * kQBlock;
    if (args.k - col >= kQBlock) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void*)(from[i] + col),
            (__attribute__((address_space(3))) void*)(tile + (i * kWaves + wave) * 8 * kQBlock), 16, 0, 0);
    } else {  // the last, incomplete one goes through registers, where what is behind column k is put to zero
      const int left = int(args.k - col) - part * 16;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (left > 0) v = first_codes(load16(from[i] + col), left);
        *reinterpret_cast<uint4*>(tile + (i * kWaves + wave) * 8 * kQBlock + lane * 16) = v;
      }
    }
  };
  auto put_scales = [&](int slot) {
#pragma unroll
    for (int i = 0; i < kScaleTurns; ++i)
      if (BM + BN >= kThreads || t < BM + BN) reinterpret_cast<uint8_t*>(scales[slot])[scale_to[i]] = scale_byte[i];
  };

  const int wm = wave / WN, wn = wave % WN;
  v4f_t sum[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) sum[i][j] = v4f_t{0, 0, 0, 0};

  const int swap = lane % 8;
  const int at0 = (lane % 16) * kQBlock + ((lane / 16 * 2) ^ swap) * 16, at1 = (lane % 16) * kQBlock + ((lane / 16 * 2 + 1) ^ swap) * 16;
  auto codes_of = [&](const uint8_t* rows) {
    const uint4 lo = *reinterpret_cast<const uint4*>(rows + at0), hi = *reinterpret_cast<const uint4*>(rows + at1);
    return v8i_t{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  auto work = [&](const uint8_t* tile, int slot) {
    const uint8_t* const ta = tile + wm * (BM / WM) * kQBlock;
    const uint8_t* const tb = tile + (BM + wn * (BN / WN)) * kQBlock;
    int sa[MI / 4], sb[NI / 4];
#pragma unroll
    for (int i = 0; i < MI / 4; ++i) sa[i] = int(scales[slot][(wm * (MI / 4) + i) * 16 + lane % 16]);
#pragma unroll
    for (int i = 0; i < NI / 4; ++i) sb[i] = int(scales[slot][BM / 4 + (wn * (NI / 4) + i) * 16 + lane % 16]);
    Fragment<EXACT> fb[NI];
    unrolled<0, NI>([&](auto j) {
      fb[j.value] = fragment_of<BCODE>(codes_of(tb + j.value * 16 * kQBlock), sb[j.value / 4] >> (8 * (j.value % 4)) & 255, Int<EXACT>{});
    });
    unrolled<0, MI>([&](auto i) {
      const Fragment<EXACT> fa =
          fragment_of<ACODE>(codes_of(ta + i.value * 16 * kQBlock), sa[i.value / 4] >> (8 * (i.value % 4)) & 255, Int<EXACT>{});
      unrolled<0, NI>([&](auto j) {
        sum[i.value][j.value] = multiply<ACODE, BCODE, i.value % 4, j.value % 4>(fb[j.value], fa, sum[i.value][j.value],
                                                                                 sb[j.value / 4], sa[i.value / 4]);
      });
    });
  };
  // what was fetched last is in shared memory, for all
  auto arrive = [&](int slot) {
    put_scales(slot);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  };

  if (first < last) {
    fetch(first, tile0);
    arrive(0);
    for (int block = first; block < last; block += 2) {
      if (block + 1 < last) fetch(block + 1, tile1);
      work(tile0, 0);
      if (block + 1 >= last) break;
      arrive(1);
      if (block + 2 < last) fetch(block + 2, tile0);
      work(tile1, 1);
      if (block + 2 < last) arrive(0);
    }
  }

  TO* const y = static_cast<TO*>(args.y) + int64_t(split) * args.m * args.n;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int row = m0 + wm * (BM / WM) + i * 16 + lane % 16;
    if (row < args.m)
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int col = n0 + wn * (BN / WN) + j * 16 + lane / 16 * 4;
        put_four(y, row * args.y_stride + col, sum[i][j], args.n - col);
      }
  }
}

// ---- few rows ---------------------------------------------------------------------------------
// Bound by reading b.  A workgroup has 16 rows of b and all (at most 16*MT) rows of a; its wavefronts take the blocks of the
// contracted axis in turn, straight from memory into registers, and their sums are added up in shared memory, in order.
constexpr int kFewWaves = 8;
template <int MT, int ACODE, int BCODE, typename TO, bool EXACT>
__global__ __launch_bounds__(kFewWaves* kWave) void matmul_few_kernel(const MatmulArgs args) {
  __shared__ v4f_t parts[kFewWaves - 1][MT][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int n0 = blockIdx.x * 16;
  const int split = blockIdx.y;
  const int first = int(int64_t(args.blocks) * split / args.splits), last = int(int64_t(args.blocks) * (split + 1) / args.splits);
  const int rb = n0 + lane % 16 < args.n ? n0 + lane % 16 : args.n - 1;
  const uint8_t* const b = args.b + rb * args.b_stride + lane / 16 * 32;
  const uint8_t* const sb = args.sb + (rb >> args.sb_shift);
  const uint8_t* a[MT];
  const uint8_t* sa[MT];
  v4f_t sum[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int ra = i * 16 + lane % 16 < args.m ? i * 16 + lane % 16 : args.m - 1;
    a[i] = args.a + ra * args.a_stride + lane / 16 * 32;
    sa[i] = args.sa + (ra >> args.sa_shift);
    sum[i] = v4f_t{0, 0, 0, 0};
  }
  auto load = [&](const uint8_t* p, int64_t col) {
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    const int left = int(args.k - col) - lane / 16 * 32;
    if (left >= 32) {
      lo = load16(p + col);
      hi = load16(p + col + 16);
    } else {
      if (left > 0) lo = first_codes(load16(p + col), left);
      if (left > 16) hi = first_codes(load16(p + col + 16), left - 16);
    }
    return v8i_t{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  for (int block = first + wave; block < last; block += kFewWaves) {
    const int64_t col = int64_t(block) * kQBlock;
    const int scale_b = sb[block * args.sb_rows];
    const Fragment<EXACT> fb = fragment_of<BCODE>(load(b, col), scale_b, Int<EXACT>{});
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int scale_a = sa[i][block * args.sa_rows];
      sum[i] = multiply<ACODE, BCODE, 0, 0>(fb, fragment_of<ACODE>(load(a[i], col), scale_a, Int<EXACT>{}), sum[i], scale_b, scale_a);
    }
  }
  if (wave) {
#pragma unroll
    for (int i = 0; i < MT; ++i) parts[wave - 1][i][lane] = sum[i];
  }
  __syncthreads();
  if (wave) return;
  TO* const y = static_cast<TO*>(args.y) + int64_t(split) * args.m * args.n;
  const int col = n0 + lane / 16 * 4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    v4f_t v = sum[i];
#pragma unroll
    for (int w = 0; w < kFewWaves - 1; ++w) v += parts[w][i][lane];
    const int row = i * 16 + lane % 16;
    if (row < args.m) put_four(y, row * args.y_stride + col, v, args.n - col);
  }
}

// Sum of the parts of the contracted axis, in order; zeros where there are none.
template <typename TO>
__global__ __launch_bounds__(256) void matmul_join_kernel(const float* parts, int splits, int64_t m, int64_t n, TO* y, int64_t y_stride) {
  const int64_t total = m * n;
  for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; at < total; at += int64_t(gridDim.x) * 1024) {
    float sum[4] = {0, 0, 0, 0};
    for (int s = 0; s < splits; ++s) {
      float f[4];
      load_short(parts + s * total, at, total, f);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += f[j];
    }
    const int64_t row = at / n, col = at % n;
    if (col + 4 <= n) {
      store_values(y + row * y_stride + col, sum, 4);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (at + j < total) {
          const int64_t r = (at + j) / n, c = (at + j) % n;
          if constexpr (sizeof(TO) == 4) y[r * y_stride + c] = sum[j];
          else y[r * y_stride + c].bits = uint16_t(bf16_pair(sum[j], 0.0f));
        }
    }
  }
}

enum { kFew1, kFew2, kFew4, kTile128 };

template <int ACODE, int BCODE, typename TO, bool EXACT>
hipError_t run(const MatmulArgs& a, const MatmulPlan& p, hipStream_t s) {
  const auto tiles = [&](int size) { return uint32_t(blocks_of(a.m, size) * blocks_of(a.n, size) * a.splits); };
  const dim3 few(uint32_t(blocks_of(a.n, 16)), uint32_t(a.splits));
  switch (p.tile) {
    case kFew1: matmul_few_kernel<1, ACODE, BCODE, TO, EXACT><<<few, kFewWaves * kWave, 0, s>>>(a); break;
    case kFew2: matmul_few_kernel<2, ACODE, BCODE, TO, EXACT><<<few, kFewWaves * kWave, 0, s>>>(a); break;
    case kFew4: matmul_few_kernel<4, ACODE, BCODE, TO, EXACT><<<few, kFewWaves * kWave, 0, s>>>(a); break;
    default: matmul_tile_kernel<128, 128, 2, 2, ACODE, BCODE, TO, EXACT><<<tiles(128), 256, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

template <typename TO, bool EXACT>
hipError_t by_code(int a_code, int b_code, const MatmulArgs& a, const MatmulPlan& p, hipStream_t s) {
  if (a_code == ACCEPT_E4M3) return b_code == ACCEPT_E4M3 ? run<0, 0, TO, EXACT>(a, p, s) : run<0, 1, TO, EXACT>(a, p, s);
  return b_code == ACCEPT_E4M3 ? run<1, 0, TO, EXACT>(a, p, s) : run<1, 1, TO, EXACT>(a, p, s);
}

template <typename TO>
hipError_t join(const MatmulArgs& a, const void* parts, int splits, void* y, hipStream_t s) {
  const int64_t want = blocks_of(int64_t(a.m) * a.n, 1024);
  matmul_join_kernel<TO><<<uint32_t(want < 4096 ? want : 4096), 256, 0, s>>>(static_cast<const float*>(parts), splits, a.m, a.n,
                                                                            static_cast<TO*>(y), a.y_stride);
  return hipGetLastError();
}

}  // namespace

MatmulPlan make_matmul_plan(const accept_matmul_desc& d) {
  MatmulPlan p{};
  p.splits = 1;
  const int64_t blocks = blocks_of(d.k, kQBlock);
  int64_t groups;  // workgroups without splits
  int64_t least;   // blocks that a split is worth
  if (d.m <= 64) {
    p.tile = d.m <= 16 ? kFew1 : d.m <= 32 ? kFew2 : kFew4;
    groups = blocks_of(d.n, 16);
    least = kFewWaves;
  } else {
    p.tile = kTile128;
    groups = blocks_of(d.m, 128) * blocks_of(d.n, 128);
    least = 4;
  }
  if (groups < 256 && d.m > 0 && d.n > 0) {
    const int64_t most = blocks / least, want = 512 / (groups < 1 ? 1 : groups);
    const int64_t s = want < most ? want : most;
    p.splits = int(s < 1 ? 1 : s > 64 ? 64 : s);
  }
  p.bytes = p.splits > 1 ? size_t(up_to(int64_t(p.splits) * d.m * d.n * 4, 256)) : 0;
  return p;
}

hipError_t launch_matmul(const accept_matmul_desc& d, const MatmulPlan& p, const void* a, const void* a_scales, const void* b,
                         const void* b_scales, void* y, void* ws, hipStream_t s) {
  if (d.m == 0 || d.n == 0) return hipSuccess;
  MatmulArgs g{};
  g.a = static_cast<const uint8_t*>(a);
  g.b = static_cast<const uint8_t*>(b);
  g.sa = static_cast<const uint8_t*>(a_scales);
  g.sb = static_cast<const uint8_t*>(b_scales);
  g.m = int(d.m);
  g.n = int(d.n);
  g.k = int(d.k);
  g.a_stride = d.a_stride ? d.a_stride : accept_block_stride(d.k);
  g.b_stride = d.b_stride ? d.b_stride : accept_block_stride(d.k);
  g.y_stride = d.y_stride ? d.y_stride : d.n;
  g.sa_rows = blocks_of(d.m, d.a_group);
  g.sb_rows = blocks_of(d.n, d.b_group);
  g.sa_shift = d.a_group == kQBlock ? 7 : 0;
  g.sb_shift = d.b_group == kQBlock ? 7 : 0;
  g.blocks = int(blocks_of(d.k, kQBlock));
  g.splits = p.splits;
  const bool f32 = d.out_dtype == ACCEPT_F32;
  if (d.k == 0) return f32 ? join<float>(g, nullptr, 0, y, s) : join<bf16_t>(g, nullptr, 0, y, s);
  if (p.splits == 1) {
    g.y = y;
    return f32 ? by_code<float, true>(d.a_code, d.b_code, g, p, s) : by_code<bf16_t, false>(d.a_code, d.b_code, g, p, s);
  }
  g.y = ws;
  g.y_stride = d.n;
  const hipError_t e = f32 ? by_code<float, true>(d.a_code, d.b_code, g, p, s) : by_code<float, false>(d.a_code, d.b_code, g, p, s);
  if (e != hipSuccess) return e;
  g.y_stride = d.y_stride ? d.y_stride : d.n;
  return f32 ? join<float>(g, ws, p.splits, y, s) : join<bf16_t>(g, ws, p.splits, y, s);
}

}  // namespace accept
