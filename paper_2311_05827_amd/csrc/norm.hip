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

// N parameters from column `at` on; `none` where there are no parameters.
template <int N, typename Col>
__device__ __forceinline__ void load_param(const void* p, int bf16, Col at, float none, float (&f)[N]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = none;
  } else if (bf16) {
    widened(load_values<bf16_t, N>(static_cast<const bf16_t*>(p), at), f);
  } else {
    widened(load_values<float, N>(static_cast<const float*>(p), at), f);
  }
}
// The same lane by lane, 0 behind the last column.
template <int N>
__device__ __forceinline__ void load_param_short(const void* p, int bf16, int64_t col, int64_t cols, float none, float (&f)[N]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = none;
  } else if (bf16) {
    load_short(static_cast<const bf16_t*>(p), col, cols, f);
  } else {
    load_short(static_cast<const float*>(p), col, cols, f);
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

// y of the vector of a row at `col`, zeros behind the last column, as codes.
template <int VEC, typename Col>
__device__ __forceinline__ void put_codes(const NormArgs& a, int64_t row, Col col, const float (&y)[VEC]) {
  float c = 0.0f;
#pragma unroll
  for (int j = 0; j < VEC; ++j) c = fmaxf(c, fabsf(y[j]));
  constexpr int LANES = kQBlock / VEC;
  c = group_max<LANES>(c);
  const int e = block_exponent(c, a.code);
  const float inv = inverse_scale(e);
  if (col < a.y_stride) {  // whole blocks
    uint8_t* const to = static_cast<uint8_t*>(a.y) + row * a.y_stride + col;
    const uint32_t lo = four_codes(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv, a.code);
    if constexpr (VEC == 8) {
      const uint32_t hi = four_codes(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv, a.code);
      *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
    } else {
      *reinterpret_cast<uint32_t*>(to) = lo;
    }
    if (col % kQBlock == 0) a.scales[col / kQBlock * a.rows + row] = uint8_t(e + 127);
  }
}

// Where a lane's vector of a row begins: at `col`, or, where the row ends before, so that it ends with the row.  Its
// first `over` columns are then the neighbour's too (all of them where the row ends before `col`): they count in no sum of the row, and
// what both write there is the same.  So no lane reads or writes a vector in pieces.  (Lane by lane and value by value, 1531 rows of
// 5003 bfloat16 took 15.3 us where they now take 9.2.)
struct Place {
  int at, over;
};
template <int VEC>
__device__ __forceinline__ Place place_of(int col, int cols) {
  const int at = col < cols - VEC ? col : cols - VEC;
  return {at, col - at};
}

// One row at a time per WAVES wavefronts, C vectors of it in a lane's registers and the next row's asked for before this one's sums: x is
// read once, the variance is that of the differences.  Bound by memory: 8144 x 768 float32 8.2 us a call (6.1 TB/s, part of it in the
// memory-side cache), 16384 x 4096 bfloat16 43.7 (6.1 TB/s), to codes 42.9; 1531 x 5003 bfloat16 9.2 (3.3 TB/s): two rows a workgroup, and
// the second one's turn begins with a wait for all that is on its way, the first one's stores too (the compiler cannot tell there whether the
// parameters have come); one row of 4096 to codes 2.6 in the kernel: two trips to memory and two meetings of four wavefronts.  Parameters in
// bfloat16 come one vector after the other, each waited for (load_param widens them in the branch that loads them): 2 * C trips at
// a kernel's start, where float32 ones are one.
template <typename TX, typename TY, int WAVES, int C>
__global__ __launch_bounds__(WAVES == 8 ? 512 : 256) void norm_kernel(const NormArgs a) {
  constexpr int VEC = Elem<TX>::VEC;
  constexpr int kRows = WAVES == 1 ? 4 : 1;  // rows of a workgroup at a time
  __shared__ float slots[2][2][WAVES];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int cols = int(a.cols), first_col = ((WAVES == 1 ? 0 : wave) * kWave + lane) * VEC;
  constexpr int kColStep = WAVES * kWave * VEC;
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t row = int64_t(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0);
  Place place[C];
#pragma unroll
  for (int c = 0; c < C; ++c) place[c] = place_of<VEC>(first_col + c * kColStep, cols);
  Raw<TX, VEC> next[C];
  auto fetch = [&](int64_t r) {
    const TX* const x = static_cast<const TX*>(a.x) + r * a.x_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) next[c] = load_values<TX, VEC>(x, place[c].at);
  };
  if (row < a.rows) fetch(row);
  float w[C][VEC], b[C][VEC];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_param(a.weight, a.param_bf16, place[c].at, 1.0f, w[c]);
    load_param(a.bias, a.param_bf16, place[c].at, 0.0f, b[c]);
  }
  int parity = 0;
  for (; row < a.rows; row += step) {
    float f[C][VEC];
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) widened(next[c], f[c]);
    if (row + step < a.rows) fetch(row + step);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum += j < place[c].over ? 0.0f : f[c][j];
    const float mean = row_sum<WAVES>(sum, slots[parity][0]) * a.inv_cols;
    float square = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        f[c][j] -= mean;
        const float d = j < place[c].over ? 0.0f : f[c][j];
        square = fmaf(d, d, square);
      }
    const float rstd = 1.0f / sqrtf(row_sum<WAVES>(square, slots[parity][1]) * a.inv_cols + a.eps);
    parity ^= 1;
    if (a.stats && lane == 0 && (WAVES == 1 || wave == 0)) {
      a.stats[row] = mean;
      a.stats[a.rows + row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float y[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) y[j] = fmaf(f[c][j] * rstd, w[c][j], b[c][j]);
      if constexpr (__is_same(TY, Codes)) {
        // a block's lanes hold its columns in order: back to where `col` is, zeros behind the last one
        moved_up(y, place[c].over);
        put_codes(a, row, first_col + c * kColStep, y);
      } else {
        store_some<TY, VEC>(static_cast<TY*>(a.y) + row * a.y_stride + place[c].at, y);
      }
    }
  }
}

// Rows longer than a workgroup's registers hold, or shorter than a vector: read three times, from the caches the second and third.
// 2048 x 20000 bfloat16 67.7 us (2.4 TB/s of one read; 16384 values a row, in registers, 30.2).
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormArgs a) {
  constexpr int VEC = Elem<TX>::VEC, WAVES = 16;
  __shared__ float slots[2][2][WAVES];
  int parity = 0;
  const int64_t cols = a.cols, end = __is_same(TY, Codes) ? a.y_stride : a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TX* const x = static_cast<const TX*>(a.x) + row * a.x_stride;
    constexpr int64_t kStep = 1024 * VEC;
    float f[VEC], sum = 0.0f, square = 0.0f;
    for (int64_t col = int64_t(threadIdx.x) * VEC; col < cols; col += kStep) {
      load_short(x, col, cols, f);
      float part = 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) part += f[j];
      sum += part;
    }
    const float mean = row_sum<WAVES>(sum, slots[parity][0]) * a.inv_cols;
    for (int64_t col = int64_t(threadIdx.x) * VEC; col < cols; col += kStep) {
      load_short(x, col, cols, f);
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[j] -= mean;
      float part = 0.0f;
#pragma unroll
      for (int j = 0; j < VEC; ++j) part = col + j < cols ? fmaf(f[j], f[j], part) : part;
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
      load_short(x, col, cols, f);
      load_param_short(a.weight, a.param_bf16, col, cols, 1.0f, w);
      load_param_short(a.bias, a.param_bf16, col, cols, 0.0f, b);
#pragma unroll
      for (int j = 0; j < VEC; ++j) y[j] = col + j < cols ? fmaf((f[j] - mean) * rstd, w[j], b[j]) : 0.0f;
      if constexpr (__is_same(TY, Codes)) put_codes(a, row, col, y);
      else store_values(static_cast<TY*>(a.y) + row * a.y_stride + col, y, cols - col);
    }
  }
}

// Backward: rows as in norm_kernel, with the two row sums that dx needs; every lane sums its columns' dy*h and dy over the rows
// that it meets, and the workgroup leaves these sums for norm_join_kernel.  One read of x and dy.  With the join, bfloat16: 16384 x 8192 158 us
// (5.1 TB/s), 8192 x 2048 25.6, 8144 x 768 12.1 (3.1 TB/s: 11 of this kernel, 9.3 without sums, 3.8 of the join).  The next row's loads
// ahead of this one's sums cost registers and with them wavefronts: 164 us at 16384 x 8192.
// (Rows of a workgroup at a time: 16 wavefronts where their 128 registers do for one's vectors, so that there are few partial sums.)
constexpr int back_rows(int vec, int waves, int c) { return waves != 1 ? 1 : vec == 4 && c == 4 ? 8 : 16; }
constexpr int back_threads(int vec, int waves, int c) { return back_rows(vec, waves, c) * waves * kWave; }
template <typename TX, typename TY, int WAVES, int C>
__global__ __launch_bounds__(back_threads(Elem<TX>::VEC, WAVES, C)) void norm_back_kernel(const NormBackArgs a) {
  constexpr int VEC = Elem<TX>::VEC;
  constexpr int kRows = back_rows(VEC, WAVES, C);
  __shared__ float slots[2][2][WAVES];
  __shared__ float joined[WAVES == 1 ? kRows : 1][2 * C * VEC][WAVES == 1 ? kWave : 1];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int cols = int(a.cols), first_col = ((WAVES == 1 ? 0 : wave) * kWave + lane) * VEC;
  constexpr int kColStep = WAVES * kWave * VEC;
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t row = int64_t(blockIdx.x) * kRows + (WAVES == 1 ? wave : 0);
  Place place[C];
#pragma unroll
  for (int c = 0; c < C; ++c) place[c] = place_of<VEC>(first_col + c * kColStep, cols);
  float w[C][VEC], dw[C][VEC], db[C][VEC];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_param(a.weight, a.param_bf16, place[c].at, 1.0f, w[c]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dw[c][j] = db[c][j] = 0.0f;
  }
  int parity = 0;
  for (; row < a.rows; row += step) {
    const TX* const x_row = static_cast<const TX*>(a.x) + row * a.x_stride;
    const TY* const dy_row = static_cast<const TY*>(a.dy) + row * a.dy_stride;
    Raw<TX, VEC> raw_x[C];
    Raw<TY, VEC> raw_dy[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      raw_x[c] = load_values<TX, VEC>(x_row, place[c].at);
      raw_dy[c] = load_values<TY, VEC>(dy_row, place[c].at);
    }
    const float mean = a.stats[row], rstd = a.stats[a.rows + row];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float x[VEC], d[VEC];
      widened(raw_x[c], x);
      widened(raw_dy[c], d);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float h = (x[j] - mean) * rstd, g = d[j] * w[c][j];
        dw[c][j] = fmaf(d[j], h, dw[c][j]);
        db[c][j] += d[j];
        s1 += j < place[c].over ? 0.0f : g;
        s2 = j < place[c].over ? s2 : fmaf(g, h, s2);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    const float m1 = row_sum<WAVES>(s1, slots[parity][0]) * a.inv_cols;
    const float m2 = row_sum<WAVES>(s2, slots[parity][1]) * a.inv_cols;
    parity ^= 1;
    TX* const dx = static_cast<TX*>(a.dx) + row * a.dx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      // h and g once more, from what was loaded: held from above they would take a register for every value
#pragma unroll
      for (uint32_t& v : raw_x[c].w) asm("" : "+v"(v));
#pragma unroll
      for (uint32_t& v : raw_dy[c].w) asm("" : "+v"(v));
      float x[VEC], d[VEC];
      widened(raw_x[c], x);
      widened(raw_dy[c], d);
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[j] = rstd * (d[j] * w[c][j] - m1 - (x[j] - mean) * rstd * m2);
      store_some<TX, VEC>(dx + place[c].at, x);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (!a.partials) return;
  float* const to = a.partials + int64_t(blockIdx.x) * 2 * cols;
  if constexpr (WAVES == 1) {  // the wavefronts had the same columns: each adds up a part of them
    constexpr int kSums = 2 * C * VEC;
#pragma unroll
    for (int i = 0; i < kSums; ++i) joined[wave][i][lane] = i < C * VEC ? dw[i / VEC % C][i % VEC] : db[i / VEC % C][i % VEC];
    __syncthreads();
    for (int i = wave; i < kSums; i += kRows) {
      const int at = i % (C * VEC);
      float v = joined[0][i][lane];
#pragma unroll
      for (int k = 1; k < kRows; ++k) v += joined[k][i][lane];
      to[i / (C * VEC) * cols + place_of<VEC>(first_col + at / VEC * kColStep, cols).at + at % VEC] = v;
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      store_some<float, VEC>(to + place[c].at, dw[c]);
      store_some<float, VEC>(to + cols + place[c].at, db[c]);
    }
  }
}

// dx of rows longer than a workgroup's registers hold, or shorter than a vector: two reads.  With the sums below, 2048 x 20000
// bfloat16 115 us.
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void norm_back_long_kernel(const NormBackArgs a) {
  constexpr int VEC = Elem<TX>::VEC, WAVES = 16;
  __shared__ float slots[2][2][WAVES];
  int parity = 0;
  const int64_t cols = a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const TX* const x = static_cast<const TX*>(a.x) + row * a.x_stride;
    const TY* const dy = static_cast<const TY*>(a.dy) + row * a.dy_stride;
    TX* const dx = static_cast<TX*>(a.dx) + row * a.dx_stride;
    const float mean = a.stats[row], rstd = a.stats[a.rows + row];
    float s1 = 0.0f, s2 = 0.0f, m1 = 0.0f, m2 = 0.0f;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      for (int64_t col = int64_t(threadIdx.x) * VEC; col < cols; col += 1024 * VEC) {
        float h[VEC], g[VEC], w[VEC], o[VEC], p1 = 0.0f, p2 = 0.0f;
        load_short(x, col, cols, h);
        load_short(dy, col, cols, g);
        load_param_short(a.weight, a.param_bf16, col, cols, 1.0f, w);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float hh = (h[j] - mean) * rstd, gg = g[j] * w[j];
          p1 += gg;
          p2 = fmaf(gg, hh, p2);
          o[j] = rstd * (gg - m1 - hh * m2);
        }
        s1 += p1;
        s2 += p2;
        if (pass) store_values(dx + col, o, cols - col);
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
#pragma unroll 4
  for (int64_t row = from; row < to; ++row) {
    const float h = (load_one(static_cast<const TX*>(a.x) + row * a.x_stride + col) - a.stats[row]) * a.stats[a.rows + row];
    const float d = load_one(static_cast<const TY*>(a.dy) + row * a.dy_stride + col);
    dw = fmaf(d, h, dw);
    db += d;
  }
  a.partials[(int64_t(blockIdx.y) * 2 + 0) * a.cols + col] = dw;
  a.partials[(int64_t(blockIdx.y) * 2 + 1) * a.cols + col] = db;
}

// Sums of the workgroups' column sums: 64 columns a workgroup, its 16 wavefronts take every 16th record each, 16 loads on their way at a
// time (one after the other: 10.5 us for 512 records of 768 columns, now 3.8 for 256).  Bound by the trips to memory.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* partials, int records, int64_t cols, void* dweight,
                                                         void* dbias, int param_bf16) {
  __shared__ float part[16][kWave];
  void* const to = blockIdx.y ? dbias : dweight;
  if (!to) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t col = (int64_t(blockIdx.z) * gridDim.x + blockIdx.x) * kWave + lane;
  float sum = 0.0f;
  if (col < cols)
#pragma unroll 16
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
// backward pass, which holds five of them), then 4, then 8, and 16 in the backward pass.
template <typename TX, template <int, int> class Launch, int FLOATS, typename... Args>
hipError_t by_width(int64_t cols, Args&&... args) {
  constexpr int VEC = Elem<TX>::VEC, F = FLOATS / VEC;
  if (cols < 8) return Launch<0, 0>::run(args...);  // for both types' vectors
  const int64_t v = blocks_of(cols, kWave * VEC);   // wavefronts' vectors in a row
  // (a form is built where the one with fewer wavefronts and all its vectors does not reach)
#define ACCEPT_WIDTH(WAVES, FEWER, CC) \
  if constexpr (CC <= F && WAVES * CC > FEWER * F) if (v <= WAVES * CC) return Launch<WAVES, CC>::run(args...);
  ACCEPT_WIDTH(1, 0, 1) ACCEPT_WIDTH(1, 0, 2) ACCEPT_WIDTH(1, 0, 3) ACCEPT_WIDTH(1, 0, 4) ACCEPT_WIDTH(1, 0, 6) ACCEPT_WIDTH(1, 0, 8)
  ACCEPT_WIDTH(4, 1, 1) ACCEPT_WIDTH(4, 1, 2) ACCEPT_WIDTH(4, 1, 3) ACCEPT_WIDTH(4, 1, 4) ACCEPT_WIDTH(4, 1, 6) ACCEPT_WIDTH(4, 1, 8)
  ACCEPT_WIDTH(8, 4, 2) ACCEPT_WIDTH(8, 4, 3) ACCEPT_WIDTH(8, 4, 4) ACCEPT_WIDTH(8, 4, 6) ACCEPT_WIDTH(8, 4, 8)
  if constexpr (FLOATS == 16) {  // the backward pass: 128 registers hold 16 bfloat16 or 12 float32 values' sums and inputs
    if constexpr (VEC == 8) { ACCEPT_WIDTH(16, 8, 2) }
    if constexpr (VEC == 4) { ACCEPT_WIDTH(16, 8, 3) }
  }
#undef ACCEPT_WIDTH
  return Launch<0, 0>::run(args...);
}

// Workgroups of the forward pass: few enough that each has several rows, loads its parameters once and has the next row on its way. Kernel,
// us, with up to 512 / 1024 / 2048: 8144 x 768 float32 9.1 / 8.8 / 11.6, 1531 x 5003 bfloat16 9.9 / 10.3 / 12.6.
constexpr int64_t kForwardGrid = 1024;

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
        const int grid = int(blocks_of(want, blocks_of(want, kForwardGrid)));  // all with the same number of turns
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

constexpr int64_t kWaveCols = kWave * 16;      // longest row of norm_back_kernel for one wavefront
// longest row of norm_back_kernel
constexpr int64_t held_cols(int x_dtype) { return x_dtype == ACCEPT_F32 ? 12 * kWaveCols : 16 * kWaveCols; }

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
        norm_back_kernel<TX, TY, WAVES, C><<<records, back_threads(Elem<TX>::VEC, WAVES, C), 0, s>>>(a);
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

// Workgroups of the backward pass: as many as the chip holds at a time, or fewer, so that their partial sums (8 bytes a column
// each, written and read) stay small beside the rows that they have.  us of the whole call with 256 / 512 / 768 of them, bfloat16:
// 4096 x 4096 29.4 / 26.1 / 27.6, 2048 x 8192 26.9 / 29.7 / 37.1, 600 x 8192 16.6 / 20.7 / 24.8.
NormPlan make_nplan(const accept_norm_desc& d) {
  NormPlan p{};
  const bool held = d.cols >= 8 && d.cols <= held_cols(d.x_dtype);
  int64_t grid;
  if (!held) {
    grid = blocks_of(d.rows, 64) < 64 ? blocks_of(d.rows, 64) : 64;
  } else if (d.cols <= kWaveCols) {
    grid = blocks_of(d.rows, 16) < 256 ? blocks_of(d.rows, 16) : 256;
  } else {
    const int64_t most = d.cols <= 4 * kWaveCols ? 768 : d.cols <= 8 * kWaveCols ? 512 : 256, by_rows = d.rows / 8 > 256 ? d.rows / 8 : 256;
    grid = d.rows < by_rows ? d.rows : by_rows;
    grid = grid < most ? grid : most;
  }
  p.back_grid = int(grid < 1 ? 1 : grid);
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
  const int64_t groups = blocks_of(d.cols, kWave);
  norm_join_kernel<<<dim3(grid_x(groups), 2, grid_rest(groups)), 1024, 0, s>>>(a.partials, records, d.cols, dweight, dbias,
                                                                              a.param_bf16);
  return hipGetLastError();
}

}  // namespace accept
