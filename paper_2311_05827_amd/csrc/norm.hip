// Layer norm: forward (to values, or to 8-bit codes with a scale per 128) and backward.
#include "stage.hpp"

namespace accept {
namespace {

struct Codes {};  // in TY's place: the output is codes and scales

struct NormArgs {
  const void* x;
  const void* weight;  // or null
  const void* bias;    // or null
  void* y;             // values, or codes
  uint8_t* scales;
  float* stats;        // or null
  int64_t rows, cols, x_stride, y_stride;
  float eps, inv_cols;
  int param_bf16, code;
};

struct NormBackArgs {
  const void* dy;
  const void* x;
  const void* weight;  // or null
  const float* stats;
  void* dx;
  float* partials;     // [workgroup][dweight, dbias][cols], or null
  int64_t rows, cols, x_stride, dy_stride, dx_stride;
  float inv_cols;
  int param_bf16;
};

template <typename T>
__device__ __forceinline__ void widen_raw(const uint4 r, float (&f)[Elem<T>::VEC]) { widen(r, f); }

// N values of any element alignment, widened; zeros from `left` on.
template <typename T, int N>
__device__ __forceinline__ void load_values(const T* p, int64_t left, float (&f)[N]) {
  constexpr int VEC = Elem<T>::VEC;
  if constexpr (N >= VEC) {
#pragma unroll
    for (int i = 0; i < N; i += VEC) {
      float part[VEC];
      widen(load_raw(p + i, left - i), part);
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[i + j] = part[j];
    }
  } else {  // half a vector of bfloat16
    typedef uint32_t v2u_elem_t __attribute__((ext_vector_type(2), aligned(2)));
    uint32_t w[2] = {0, 0};
    if (left >= N) {
      const v2u_elem_t v = *reinterpret_cast<const v2u_elem_t*>(p);
      w[0] = v.x;
      w[1] = v.y;
    } else if (left > 0) {
#pragma unroll
      for (int j = 0; j < N - 1; ++j)
        if (j < left) w[j / 2] |= uint32_t(p[j].bits) << (16 * (j & 1));
    }
    f[0] = u32_as_f32(w[0] << 16); f[1] = u32_as_f32(w[0] & 0xFFFF0000u);
    f[2] = u32_as_f32(w[1] << 16); f[3] = u32_as_f32(w[1] & 0xFFFF0000u);
  }
}

// VEC parameters from column `col` on; `none` where there are no parameters, 0 behind the last column.
template <int VEC>
__device__ __forceinline__ void load_param(const void* p, int bf16, int64_t col, int64_t cols, float none, float (&f)[VEC]) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) f[j] = 0.0f;
  if (!p) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) f[j] = none;
  } else if (bf16) {
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (col + j < cols) f[j] = load_one(static_cast<const bf16_t*>(p) + col + j);
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (col + j < cols) f[j] = static_cast<const float*>(p)[col + j];
  }
}

// Sum over the lanes of the WAVES wavefronts that share a row, in a fixed order.  `slots` is WAVES floats of the
// row's own; one barrier.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* slots) {
  v = wave_sum_f32(v);
  if constexpr (WAVES == 1) {
    return v;
  } else {
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0) slots[wave] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) s += slots[i];
    return s;
  }
}

// y of one vector of a row, written as values or as codes.
template <typename TY, int VEC>
__device__ __forceinline__ void put(const NormArgs& a, int64_t row, int64_t col, const float (&y)[VEC]) {
  if constexpr (__is_same(TY, Codes)) {
    const int64_t stride = a.y_stride;  // whole blocks
    float c = 0.0f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) c = fmaxf(c, fabsf(y[j]));
    constexpr int LANES = kQBlock / VEC;
    c = group_max<LANES>(c);
    const int e = block_exponent(c, a.code);
    const float inv = inverse_scale(e);
    if (col < stride) {
      uint8_t* const to = static_cast<uint8_t*>(a.y) + row * stride + col;
      const uint32_t lo = four_codes(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv, a.code);
      if constexpr (VEC == 8) {
        const uint32_t hi = four_codes(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv, a.code);
        *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
      } else {
        *reinterpret_cast<uint32_t*>(to) = lo;
      }
      if (col % kQBlock == 0) a.scales[col / kQBlock * a.rows + row] = uint8_t(e + 127);
    }
  } else {
    store_values(static_cast<TY*>(a.y) + row * a.y_stride + col, y, a.cols - col);
  }
}

// One row at a time per WAVES wavefronts, C vectors of it in a lane's registers: x is read once, the variance is that of the
// differences.  Bound by memory.
template <typename TX, typename TY, int WAVES, int C>
__global__ __launch_bounds__(WAVES == 8 ? 512 : 256) void norm_kernel(const NormArgs a) {
  constexpr int VEC = Elem<TX>::VEC;
  constexpr int kRows = WAVES == 1 ? 4 : 1;  // rows of a workgroup at a time
  __shared__ float slots[2][2][WAVES];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t first_col = int64_t((WAVES == 1 ? 0 : wave) * kWave + lane) * VEC;
  constexpr int64_t kColStep = int64_t(WAVES) * kWave * VEC;
  float w[C][VEC], b[C][VEC];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_param(a.weight, a.param_bf16, first_col + c * kColStep, a.cols, 1.0f, w[c]);
    load_param(a.bias, a.param_bf16, first_col + c * kColStep, a.cols, 0.0f, b[c]);
  }
  int parity = 0;
  for (int64_t row = int64_t(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0); row < a.rows; row += int64_t(gridDim.x) * kRows) {
    const TX* const x = static_cast<const TX*>(a.x) + row * a.x_stride;
    float f[C][VEC];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
      widen_raw<TX>(load_raw(x + col, a.cols - col), f[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum += f[c][j];
    const float mean = row_sum<WAVES>(sum, slots[parity][0]) * a.inv_cols;
    float square = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float d = col + j < a.cols ? f[c][j] - mean : 0.0f;
        f[c][j] = d;
        square = fmaf(d, d, square);
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum<WAVES>(square, slots[parity][1]) * a.inv_cols + a.eps);
    parity ^= 1;
    if (a.stats && lane == 0 && (WAVES == 1 || wave == 0)) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
      float y[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) y[j] = col + j < a.cols ? fmaf(f[c][j] * rstd, w[c][j], b[c][j]) : 0.0f;
      put<TY>(a, row, col, y);
    }
  }
}

// Rows longer than a workgroup's registers hold: read three times, from the caches the second and third.
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormArgs a) {
  constexpr int VEC = Elem<TX>::VEC, WAVES = 16;
  __shared__ float slots[2][2][WAVES];
  int parity = 0;
  const int64_t end = __is_same(TY, Codes) ? a.y_stride : a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TX* const x = static_cast<const TX*>(a.x) + row * a.x_stride;
    constexpr int64_t kStep = 1024 * VEC;
    float f[VEC], sum = 0.0f, square = 0.0f;
    for (int64_t col = int64_t(threadIdx.x) * VEC; col < a.cols; col += kStep) {
      widen_raw<TX>(load_raw(x + col, a.cols - col), f);
      float part = 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) part += f[j];
      sum += part;
    }
    const float mean = row_sum<WAVES>(sum, slots[parity][0]) * a.inv_cols;
    for (int64_t col = int64_t(threadIdx.x) * VEC; col < a.cols; col += kStep) {
      widen_raw<TX>(load_raw(x + col, a.cols - col), f);
      float part = 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float d = col + j < a.cols ? f[j] - mean : 0.0f;
        part = fmaf(d, d, part);
      }
      square += part;
    }
    const float rstd = 1.0f / sqrtf(row_sum<WAVES>(square, slots[parity][1]) * a.inv_cols + a.eps);
    parity ^= 1;
    if (a.stats && threadIdx.x == 0) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
    }
    // all lanes stay in the loop as long as one is: a block's lanes look at each other
    for (int64_t base = 0; base < end; base += kStep) {
      const int64_t col = base + int64_t(threadIdx.x) * VEC;
      float w[VEC], b[VEC], y[VEC];
      widen_raw<TX>(load_raw(x + col, a.cols - col), f);
      load_param(a.weight, a.param_bf16, col, a.cols, 1.0f, w);
      load_param(a.bias, a.param_bf16, col, a.cols, 0.0f, b);
#pragma unroll
      for (int j = 0; j < VEC; ++j) y[j] = col + j < a.cols ? fmaf((f[j] - mean) * rstd, w[j], b[j]) : 0.0f;
      put<TY>(a, row, col, y);
    }
  }
}

// Backward: rows as in norm_kernel, with the two row sums that dx needs; every lane sums its columns' dy*h and dy over the rows
// that it meets, and the workgroup leaves these sums for join_kernel.  One read of x and dy.
template <typename TX, typename TY, int WAVES, int C>
__global__ __launch_bounds__(WAVES == 8 ? 512 : 256) void norm_back_kernel(const NormBackArgs a) {
  constexpr int VEC = Elem<TX>::VEC;
  constexpr int kRows = WAVES == 1 ? 4 : 1;
  __shared__ float slots[2][2][WAVES];
  __shared__ float joined[WAVES == 1 ? 3 * kWave * VEC * C : 1];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t first_col = int64_t((WAVES == 1 ? 0 : wave) * kWave + lane) * VEC;
  constexpr int64_t kColStep = int64_t(WAVES) * kWave * VEC;
  float w[C][VEC], dw[C][VEC], db[C][VEC];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_param(a.weight, a.param_bf16, first_col + c * kColStep, a.cols, 1.0f, w[c]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[c][j] = db[c][j] = 0.0f;
  }
  int parity = 0;
  for (int64_t row = int64_t(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0); row < a.rows; row += int64_t(gridDim.x) * kRows) {
    const TX* const x = static_cast<const TX*>(a.x) + row * a.x_stride;
    const TY* const dy = static_cast<const TY*>(a.dy) + row * a.dy_stride;
    const float mean = a.stats[row], rstd = a.stats[a.rows + row];
    float h[C][VEC], g[C][VEC];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
      widen_raw<TX>(load_raw(x + col, a.cols - col), h[c]);
      load_values(dy + col, a.cols - col, g[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float hh = col + j < a.cols ? (h[c][j] - mean) * rstd : 0.0f;
        const float d = g[c][j];
        dw[c][j] = fmaf(d, hh, dw[c][j]);
        db[c][j] += d;
        const float gg = d * w[c][j];
        h[c][j] = hh;
        g[c][j] = gg;
        s1 += gg;
        s2 = fmaf(gg, hh, s2);
      }
    }
    const float m1 = row_sum<WAVES>(s1, slots[parity][0]) * a.inv_cols;
    const float m2 = row_sum<WAVES>(s2, slots[parity][1]) * a.inv_cols;
    parity ^= 1;
    TX* const dx = static_cast<TX*>(a.dx) + row * a.dx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
      float o[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) o[j] = rstd * (g[c][j] - m1 - h[c][j] * m2);
      store_values(dx + col, o, a.cols - col);
    }
  }
  if (!a.partials) return;
  float* const to = a.partials + int64_t(blockIdx.x) * 2 * a.cols;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if constexpr (WAVES == 1) {  // the four wavefronts had the same columns
      if (which) __syncthreads();
      if (wave) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int j = 0; j < VEC; ++j) joined[((wave - 1) * C * VEC + c * VEC + j) * kWave + lane] = which ? db[c][j] : dw[c][j];
      }
      __syncthreads();
      if (wave) continue;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          float& v = which ? db[c][j] : dw[c][j];
#pragma unroll
          for (int i = 0; i < 3; ++i) v += joined[(i * C * VEC + c * VEC + j) * kWave + lane];
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t col = first_col + c * kColStep;
      store_values(to + which * a.cols + col, which ? db[c] : dw[c], a.cols - col);
    }
  }
}

// dx of rows longer than a workgroup's registers hold: two reads.
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void norm_back_long_kernel(const NormBackArgs a) {
  constexpr int VEC = Elem<TX>::VEC, WAVES = 16;
  __shared__ float slots[2][2][WAVES];
  int parity = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TX* const x = static_cast<const TX*>(a.x) + row * a.x_stride;
    const TY* const dy = static_cast<const TY*>(a.dy) + row * a.dy_stride;
    TX* const dx = static_cast<TX*>(a.dx) + row * a.dx_stride;
    const float mean = a.stats[row], rstd = a.stats[a.rows + row];
    float s1 = 0.0f, s2 = 0.0f, m1 = 0.0f, m2 = 0.0f;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      for (int64_t col = int64_t(threadIdx.x) * VEC; col < a.cols; col += 1024 * VEC) {
        float h[VEC], g[VEC], w[VEC], o[VEC], p1 = 0.0f, p2 = 0.0f;
        widen_raw<TX>(load_raw(x + col, a.cols - col), h);
        load_values(dy + col, a.cols - col, g);
        load_param(a.weight, a.param_bf16, col, a.cols, 1.0f, w);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float hh = (h[j] - mean) * rstd, gg = g[j] * w[j];
          if (col + j < a.cols) {
            p1 += gg;
            p2 = fmaf(gg, hh, p2);
          }
          o[j] = rstd * (gg - m1 - hh * m2);
        }
        s1 += p1;
        s2 += p2;
        if (pass) store_values(dx + col, o, a.cols - col);
      }
      if (!pass) {
        m1 = row_sum<WAVES>(s1, slots[parity][0]) * a.inv_cols;
        m2 = row_sum<WAVES>(s2, slots[parity][1]) * a.inv_cols;
      }
    }
    parity ^= 1;
  }
}

// The column sums for such rows: a thread per column and group of rows.
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormBackArgs a, int64_t rows_each) {
  const int64_t col = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (col >= a.cols) return;
  const int64_t from = blockIdx.y * rows_each, to = from + rows_each < a.rows ? from + rows_each : a.rows;
  float dw = 0.0f, db = 0.0f;
  for (int64_t row = from; row < to; ++row) {
    const float h = (load_one(static_cast<const TX*>(a.x) + row * a.x_stride + col) - a.stats[row]) * a.stats[a.rows + row];
    const float d = load_one(static_cast<const TY*>(a.dy) + row * a.dy_stride + col);
    dw = fmaf(d, h, dw);
    db += d;
  }
  a.partials[(int64_t(blockIdx.y) * 2 + 0) * a.cols + col] = dw;
  a.partials[(int64_t(blockIdx.y) * 2 + 1) * a.cols + col] = db;
}

// Sums of the workgroups' column sums: 64 columns a workgroup, its 16 wavefronts take every 16th record each.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* partials, int records, int64_t cols, void* dweight,
                                                         void* dbias, int param_bf16) {
  __shared__ float part[16][kWave];
  void* const to = blockIdx.y ? dbias : dweight;
  if (!to) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t col = int64_t(blockIdx.x) * kWave + lane;
  float sum = 0.0f;
  if (col < cols)
    for (int r = wave; r < records; r += 16) sum += partials[(int64_t(r) * 2 + blockIdx.y) * cols + col];
  part[wave][lane] = sum;
  __syncthreads();
  if (wave || col >= cols) return;
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += part[i][lane];
  if (param_bf16) static_cast<bf16_t*>(to)[col].bits = uint16_t(bf16_pair(sum, 0.0f));
  else static_cast<float*>(to)[col] = sum;
}

// ---- dispatch ---------------------------------------------------------------------------------
// Wavefronts per row and vectors per lane: one wavefront while a row fits in its registers with 32 values a lane (16 in the
// backward pass, which holds five of them), then 4, then 8.
template <typename TX, template <int, int> class Launch, int FLOATS, typename... Args>
hipError_t by_width(int64_t cols, Args&&... args) {
  constexpr int VEC = Elem<TX>::VEC, F = FLOATS / VEC;
  const int64_t v = blocks_of(cols, kWave * VEC);  // wavefronts' vectors in a row
#define ACCEPT_WIDTH(WAVES, CC) \
  if constexpr (CC <= F) if (v <= WAVES * CC) return Launch<WAVES, CC>::run(args...);
  ACCEPT_WIDTH(1, 1) ACCEPT_WIDTH(1, 2) ACCEPT_WIDTH(1, 3) ACCEPT_WIDTH(1, 4) ACCEPT_WIDTH(1, 6) ACCEPT_WIDTH(1, 8)
  ACCEPT_WIDTH(4, 2) ACCEPT_WIDTH(4, 3) ACCEPT_WIDTH(4, 4) ACCEPT_WIDTH(4, 6) ACCEPT_WIDTH(4, 8)
  ACCEPT_WIDTH(8, 2) ACCEPT_WIDTH(8, 3) ACCEPT_WIDTH(8, 4) ACCEPT_WIDTH(8, 6) ACCEPT_WIDTH(8, 8)
#undef ACCEPT_WIDTH
  return Launch<0, 0>::run(args...);
}

constexpr int64_t kForwardGrid = 2048;

template <typename TX, typename TY>
struct Forward {
  template <int WAVES, int C>
  struct At {
    static hipError_t run(const NormArgs& a, hipStream_t s) {
      if constexpr (WAVES == 0) {
        const int grid = int(a.rows < kForwardGrid ? a.rows : kForwardGrid);
        norm_long_kernel<TX, TY><<<grid, 1024, 0, s>>>(a);
      } else {
        const int64_t want = blocks_of(a.rows, WAVES == 1 ? 4 : 1);
        const int grid = int(want < kForwardGrid ? want : kForwardGrid);
        norm_kernel<TX, TY, WAVES, C><<<grid, WAVES == 8 ? 512 : 256, 0, s>>>(a);
      }
      return hipGetLastError();
    }
  };
};

template <typename TY>
hipError_t forward(int x_dtype, const NormArgs& a, hipStream_t s) {
  return x_dtype == ACCEPT_F32 ? by_width<float, Forward<float, TY>::template At, 32>(a.cols, a, s)
                               : by_width<bf16_t, Forward<bf16_t, TY>::template At, 32>(a.cols, a, s);
}

constexpr int64_t kBackGrid = 512;
constexpr int64_t kHeldCols = 8 * kWave * 16;  // longest row of norm_back_kernel

template <typename TX, typename TY>
struct Backward {
  template <int WAVES, int C>
  struct At {
    static hipError_t run(const NormBackArgs& a, int records, hipStream_t s) {
      if constexpr (WAVES == 0) {
        norm_back_long_kernel<TX, TY><<<int(a.rows < kForwardGrid ? a.rows : kForwardGrid), 1024, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || !a.partials) return e;
        norm_columns_kernel<TX, TY><<<dim3(uint32_t(blocks_of(a.cols, 256)), uint32_t(records)), 256, 0, s>>>(a, blocks_of(a.rows, records));
      } else {
        norm_back_kernel<TX, TY, WAVES, C><<<records, WAVES == 8 ? 512 : 256, 0, s>>>(a);
      }
      return hipGetLastError();
    }
  };
};

template <typename TX, typename TY>
hipError_t backward(const NormBackArgs& a, int records, hipStream_t s) {
  return by_width<TX, Backward<TX, TY>::template At, 16>(a.cols, a, records, s);
}

NormArgs forward_args(const accept_norm_desc& d, const void* x, const void* weight, const void* bias, void* y, float* stats) {
  NormArgs a{};
  a.x = x;
  a.weight = weight;
  a.bias = bias;
  a.y = y;
  a.stats = stats;
  a.rows = d.rows;
  a.cols = d.cols;
  a.x_stride = d.x_stride ? d.x_stride : d.cols;
  a.y_stride = d.y_stride ? d.y_stride : d.cols;
  a.eps = float(d.eps);
  a.inv_cols = float(1.0 / double(d.cols));
  a.param_bf16 = d.param_dtype == ACCEPT_BF16;
  a.code = d.code;
  return a;
}

}  // namespace

NormPlan make_nplan(const accept_norm_desc& d) {
  NormPlan p{};
  const int64_t units = d.cols > kHeldCols ? blocks_of(d.rows, 64) : blocks_of(d.rows, 4);
  const int64_t most = d.cols > kHeldCols ? 64 : kBackGrid;
  p.back_grid = int(units < 1 ? 1 : units < most ? units : most);
  p.bytes = size_t(up_to(int64_t(p.back_grid) * 2 * d.cols * 4, 256));
  return p;
}

hipError_t launch_norm(const accept_norm_desc& d, const void* x, const void* weight, const void* bias, void* y,
                       float* stats, hipStream_t s) {
  const NormArgs a = forward_args(d, x, weight, bias, y, stats);
  return d.y_dtype == ACCEPT_F32 ? forward<float>(d.x_dtype, a, s) : forward<bf16_t>(d.x_dtype, a, s);
}

hipError_t launch_norm_quantize(const accept_norm_desc& d, const void* x, const void* weight, const void* bias, void* codes,
                                void* scales, float* stats, hipStream_t s) {
  NormArgs a = forward_args(d, x, weight, bias, codes, stats);
  a.y_stride = accept_block_stride(d.cols);
  a.scales = static_cast<uint8_t*>(scales);
  return forward<Codes>(d.x_dtype, a, s);
}

hipError_t launch_norm_backward(const accept_norm_desc& d, const NormPlan& p, const void* dy, const void* x,
                                const void* weight, const float* stats, void* dx, void* dweight, void* dbias, void* ws,
                                hipStream_t s) {
  NormBackArgs a{};
  a.dy = dy;
  a.x = x;
  a.weight = weight;
  a.stats = stats;
  a.dx = dx;
  a.partials = dweight || dbias ? static_cast<float*>(ws) : nullptr;
  a.rows = d.rows;
  a.cols = d.cols;
  a.x_stride = d.x_stride ? d.x_stride : d.cols;
  a.dy_stride = d.y_stride ? d.y_stride : d.cols;
  a.dx_stride = d.dx_stride ? d.dx_stride : d.cols;
  a.inv_cols = float(1.0 / double(d.cols));
  a.param_bf16 = d.param_dtype == ACCEPT_BF16;
  int records = 0;  // no rows: sums of nothing
  if (d.rows > 0) {
    records = p.back_grid;
    hipError_t e;
    if (d.x_dtype == ACCEPT_F32)
      e = d.y_dtype == ACCEPT_F32 ? backward<float, float>(a, records, s) : backward<float, bf16_t>(a, records, s);
    else
      e = d.y_dtype == ACCEPT_F32 ? backward<bf16_t, float>(a, records, s) : backward<bf16_t, bf16_t>(a, records, s);
    if (e != hipSuccess) return e;
  }
  if (!a.partials) return hipSuccess;
  norm_join_kernel<<<dim3(uint32_t(blocks_of(d.cols, kWave)), 2), 1024, 0, s>>>(a.partials, records, d.cols, dweight, dbias,
                                                                               a.param_bf16);
  return hipGetLastError();
}

}  // namespace accept
