// Quantization to 8-bit floating point with a power-of-two scale for each block of 128.
#include "stage.hpp"

namespace accept {
namespace {

struct BlockArgs {
  const void* x;
  uint8_t* codes;
  uint8_t* scales;
  uint8_t* codes_t;
  uint8_t* scales_t;
  int64_t rows, cols, x_stride, stride, stride_t;
  int64_t row_blocks, col_blocks;
  int code;
};

// Rows only, a scale for 128 of one: 16 (bfloat16) or 32 (float32) neighbouring lanes hold a block, and a thread takes kBlocks blocks next
// to each other, all loaded before the first is converted; a workgroup's rows are consecutive, so the bytes of the scales lie
// together.  Bound by memory.  us with one block a turn / two / four: 16384 x 8192 bfloat16 100.4 / 86.2 / 85.1
// (4.7 TB/s), 8144 x 2048 10.5 / 10.6 / 11.7.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const BlockArgs a) {
  constexpr int VEC = Elem<T>::VEC, LANES = kQBlock / VEC, kBlocks = 2;
  const int64_t row = (int64_t(blockIdx.z) * gridDim.x + blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  if (row >= a.rows) return;  // whole groups of lanes
  const T* const x = static_cast<const T*>(a.x) + row * a.x_stride;
  for (int64_t first = int64_t(blockIdx.y) * kBlocks; first < a.col_blocks; first += int64_t(gridDim.y) * kBlocks) {
    float f[kBlocks][VEC];
    if (a.cols >= VEC) {  // the same in all lanes
      Raw<T, VEC> raw[kBlocks];
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) {
        const int64_t col = (first + u) * kQBlock + threadIdx.x % LANES * VEC;
        raw[u] = load_values<T, VEC>(x, col < a.cols - VEC ? col : a.cols - VEC);
      }
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) {
        const int64_t col = (first + u) * kQBlock + threadIdx.x % LANES * VEC;
        widened(raw[u], f[u]);
        moved_up(f[u], col < a.cols - VEC ? 0 : col - (a.cols - VEC));
      }
    } else {
#pragma unroll
      for (int u = 0; u < kBlocks; ++u) load_short(x, (first + u) * kQBlock + threadIdx.x % LANES * VEC, a.cols, f[u]);
    }
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      const int64_t block = first + u;
      if (block >= a.col_blocks) break;
      float c = 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) c = fmaxf(c, fabsf(f[u][j]));
      const int e = block_exponent(group_max<LANES>(c), a.code);
      const float inv = inverse_scale(e);
      uint8_t* const to = a.codes + row * a.stride + block * kQBlock + threadIdx.x % LANES * VEC;
      const uint32_t lo = four_codes(f[u][0] * inv, f[u][1] * inv, f[u][2] * inv, f[u][3] * inv, a.code);
      if constexpr (VEC == 8)
        *reinterpret_cast<uint2*>(to) = make_uint2(lo, four_codes(f[u][4] * inv, f[u][5] * inv, f[u][6] * inv, f[u][7] * inv, a.code));
      else
        *reinterpret_cast<uint32_t*>(to) = lo;
      if (threadIdx.x % LANES == 0) a.scales[block * a.rows + row] = uint8_t(e + 127);
    }
  }
}

// A square of 128 x 128 per workgroup, held in registers: thread t has rows 8*(t/16) .. +7 and columns 8*(t%16) .. +7, so
// a row's block lies in 16 neighbouring lanes, and a thread's part of a column is 8 bytes of codes.  The transposed codes
// go through shared memory, to be written in whole lines.  Bound by memory: 8192 x 8192 float32 in squares, both ways, 79 us (5.1 TB/s);
// 8144 x 2048 bfloat16, both ways, 15.4 (4.3 TB/s), columns only 13.0, of which two are the launch and the first rows' way from memory.
template <typename T, int GROUP, bool ROWS, bool COLS>
__global__ __launch_bounds__(256) void quantize_square_kernel(const BlockArgs a) {
  constexpr int kPad = 8;  // bytes behind a column of codes, so that its neighbours lie in other banks
  __shared__ float most[4][kQBlock];
  __shared__ __align__(16) uint8_t turned[COLS ? kQBlock * (kQBlock + kPad) : 16];
  const int t = threadIdx.x, cx = t % 16, ry = t / 16, wave = t / kWave;
  const uint32_t square = blockIdx.y * gridDim.x + blockIdx.x, col_blocks = uint32_t(a.col_blocks);
  if (square >= uint32_t(a.row_blocks) * col_blocks) return;  // the whole workgroup
  const int64_t rb = square / col_blocks, cb = square % col_blocks;
  const int64_t row0 = rb * kQBlock + 8 * ry, col0 = cb * kQBlock + 8 * cx;
  float f[8][8];
  if (a.cols >= 8) {  // the same in all lanes
    const int64_t at = col0 < a.cols - 8 ? col0 : a.cols - 8;
    Raw<T, 8> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + i < a.rows ? row0 + i : a.rows - 1;
      raw[i] = load_values<T, 8>(static_cast<const T*>(a.x) + row * a.x_stride, at);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      widened(raw[i], f[i]);
      moved_up(f[i], col0 - at);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      load_short(static_cast<const T*>(a.x) + (row0 + i < a.rows ? row0 + i : a.rows - 1) * a.x_stride, col0, a.cols, f[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (row0 + i >= a.rows) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = 0.0f;
    }
  float inv_square = 0.0f;
  if constexpr (GROUP == kQBlock) {
    float c = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) c = fmaxf(c, fabsf(f[i][j]));
    c = wave_max(c);
    if (t % kWave == 0) most[0][wave] = c;
    __syncthreads();
    c = fmaxf(fmaxf(most[0][0], most[0][1]), fmaxf(most[0][2], most[0][3]));
    const int e = block_exponent(c, a.code);
    inv_square = inverse_scale(e);
    if (t == 0) {
      if (ROWS) a.scales[cb * a.row_blocks + rb] = uint8_t(e + 127);
      if (COLS) a.scales_t[rb * a.col_blocks + cb] = uint8_t(e + 127);
    }
  }
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float inv = inv_square;
      if constexpr (GROUP == 1) {
        float c = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) c = fmaxf(c, fabsf(f[i][j]));
        const int e = block_exponent(group_max<16>(c), a.code);
        inv = inverse_scale(e);
        if (cx == 0 && row0 + i < a.rows) a.scales[cb * a.rows + row0 + i] = uint8_t(e + 127);
      }
      if (row0 + i < a.rows)
        *reinterpret_cast<uint2*>(a.codes + (row0 + i) * a.stride + col0) =
            make_uint2(four_codes(f[i][0] * inv, f[i][1] * inv, f[i][2] * inv, f[i][3] * inv, a.code),
                       four_codes(f[i][4] * inv, f[i][5] * inv, f[i][6] * inv, f[i][7] * inv, a.code));
    }
  }
  if constexpr (COLS) {
    float inv[8];
    if constexpr (GROUP == 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float c = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) c = fmaxf(c, fabsf(f[i][j]));
        c = fmaxf(c, __shfl_xor(c, 16, kWave));
        c = fmaxf(c, __shfl_xor(c, 32, kWave));
        if (t % kWave < 16) most[wave][8 * cx + j] = c;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = 8 * cx + j;
        const int e = block_exponent(fmaxf(fmaxf(most[0][at], most[1][at]), fmaxf(most[2][at], most[3][at])), a.code);
        inv[j] = inverse_scale(e);
        if (ry == 0 && col0 + j < a.cols) a.scales_t[rb * a.cols + col0 + j] = uint8_t(e + 127);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) inv[j] = inv_square;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float s = inv[j];
      *reinterpret_cast<uint2*>(turned + (8 * cx + j) * (kQBlock + kPad) + 8 * ry) =
          make_uint2(four_codes(f[0][j] * s, f[1][j] * s, f[2][j] * s, f[3][j] * s, a.code),
                     four_codes(f[4][j] * s, f[5][j] * s, f[6][j] * s, f[7][j] * s, a.code));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = i * 256 + t, col = at / 16, part = at % 16;
      if (cb * kQBlock + col < a.cols)
        *reinterpret_cast<uint2*>(a.codes_t + (cb * kQBlock + col) * a.stride_t + rb * kQBlock + 8 * part) =
            *reinterpret_cast<const uint2*>(turned + col * (kQBlock + kPad) + 8 * part);
    }
  }
}

template <typename T>
hipError_t quantize(const BlockArgs& a, int group, hipStream_t s) {
  if (group == 1 && !a.codes_t) {
    constexpr int kRows = 256 / (kQBlock / Elem<T>::VEC);
    const int64_t turns = blocks_of(a.col_blocks, 2), y = turns < 65535 ? turns : 65535, groups = blocks_of(a.rows, kRows);
    quantize_rows_kernel<T><<<dim3(grid_x(groups), uint32_t(y), grid_rest(groups)), 256, 0, s>>>(a);
    return hipGetLastError();
  }
  const int64_t squares = a.row_blocks * a.col_blocks;  // (below 2^27 by the limits on sizes)
  const dim3 grid = dim3(grid_x(squares), grid_rest(squares));
  if (group == 1) {
    if (a.codes) quantize_square_kernel<T, 1, true, true><<<grid, 256, 0, s>>>(a);
    else quantize_square_kernel<T, 1, false, true><<<grid, 256, 0, s>>>(a);
  } else {
    if (a.codes && a.codes_t) quantize_square_kernel<T, kQBlock, true, true><<<grid, 256, 0, s>>>(a);
    else if (a.codes) quantize_square_kernel<T, kQBlock, true, false><<<grid, 256, 0, s>>>(a);
    else quantize_square_kernel<T, kQBlock, false, true><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_quantize(const accept_block_desc& d, const void* x, void* codes, void* scales, void* codes_t,
                                 void* scales_t, hipStream_t s) {
  if (d.rows == 0 || d.cols == 0) return hipSuccess;
  BlockArgs a{};
  a.x = x;
  a.codes = static_cast<uint8_t*>(codes);
  a.scales = static_cast<uint8_t*>(scales);
  a.codes_t = static_cast<uint8_t*>(codes_t);
  a.scales_t = static_cast<uint8_t*>(scales_t);
  a.rows = d.rows;
  a.cols = d.cols;
  a.x_stride = d.x_stride ? d.x_stride : d.cols;
  a.stride = accept_block_stride(d.cols);
  a.stride_t = accept_block_stride(d.rows);
  a.row_blocks = blocks_of(d.rows, kQBlock);
  a.col_blocks = blocks_of(d.cols, kQBlock);
  a.code = d.code;
  return d.in_dtype == ACCEPT_F32 ? quantize<float>(a, d.group, s) : quantize<bf16_t>(a, d.group, s);
}

}  // namespace accept
