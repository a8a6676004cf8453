// Internal declarations of the stage operators: layer norm, blocks in 8-bit floating point, their product.
#pragma once

#include "accept_stage.h"
#include "common.hpp"

namespace accept {

constexpr int kQBlock = 128;         // values along the contracted axis that share a scale
constexpr int kMinExponent = -100;   // of a scale

inline int64_t up_to(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t blocks_of(int64_t v, int64_t by) { return (v + by - 1) / by; }
// Workgroups in a launch's x: a launch takes fewer than 2^32 threads in a dimension, so where there are more workgroups than
// this, another dimension has the rest (65535 at most).
constexpr int64_t kGridX = int64_t(1) << 21;
inline uint32_t grid_x(int64_t groups) { return uint32_t(groups < kGridX ? groups : kGridX); }
inline uint32_t grid_rest(int64_t groups) { return uint32_t(blocks_of(groups, kGridX)); }

struct NormPlan {
  int back_grid;  // workgroups of the backward pass = number of partial column sums
  size_t bytes;   // workspace
};
NormPlan make_nplan(const accept_norm_desc& d);
hipError_t launch_norm(const accept_norm_desc& d, const void* x, const void* weight, const void* bias, void* y,
                       float* stats, hipStream_t s);
hipError_t launch_norm_quantize(const accept_norm_desc& d, const void* x, const void* weight, const void* bias, void* codes,
                                void* scales, float* stats, hipStream_t s);
hipError_t launch_norm_backward(const accept_norm_desc& d, const NormPlan& p, const void* dy, const void* x,
                                const void* weight, const float* stats, void* dx, void* dweight, void* dbias, void* ws,
                                hipStream_t s);

hipError_t launch_block_quantize(const accept_block_desc& d, const void* x, void* codes, void* scales, void* codes_t,
                                 void* scales_t, hipStream_t s);

struct MatmulPlan {
  int tile;      // which kernel (see make_matmul_plan)
  int few_n;     // few rows: 16 columns of results a workgroup, or 32
  int splits;    // parts of the contracted axis, joined by a second kernel where there are several
  size_t bytes;  // workspace
};
MatmulPlan make_matmul_plan(const accept_matmul_desc& d);
hipError_t launch_matmul(const accept_matmul_desc& d, const MatmulPlan& p, const void* a, const void* a_scales, const void* b,
                         const void* b_scales, void* y, void* ws, hipStream_t s);

#if defined(__HIPCC__)

// N consecutive values of a row, as they lie in memory.
template <typename T, int N>
struct Raw {
  static constexpr int kWords = N * int(sizeof(T)) / 4;
  uint32_t w[kWords];
};

// Values at .. at+N-1 of a row, from any element's alignment (vector memory takes it).
template <typename T, int N, typename Col>
__device__ __forceinline__ Raw<T, N> load_values(const T* row, Col at) {
  const char* p = reinterpret_cast<const char*>(row);
  if constexpr (sizeof(Col) == 4) p += uint32_t(at) * uint32_t(sizeof(T));  // one base for all lanes, 32 bits of each
  else p += at * int64_t(sizeof(T));
  constexpr int kPart = Raw<T, N>::kWords < 4 ? 2 : 4;
  typedef uint32_t part_t __attribute__((ext_vector_type(kPart), aligned(sizeof(T))));
  Raw<T, N> r;
#pragma unroll
  for (int i = 0; i < Raw<T, N>::kWords; i += kPart) {
    const part_t v = *reinterpret_cast<const part_t*>(p + 4 * i);
#pragma unroll
    for (int j = 0; j < kPart; ++j) r.w[i + j] = v[j];
  }
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void widened(const Raw<T, N>& r, float (&f)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if constexpr (sizeof(T) == 4) f[j] = u32_as_f32(r.w[j]);
    else f[j] = u32_as_f32(j & 1 ? r.w[j / 2] & 0xFFFF0000u : r.w[j / 2] << 16);
  }
}
// The values from `over` >= 0 on, moved to the front; zeros behind them.
template <int N, typename Over>
__device__ __forceinline__ void moved_up(float (&f)[N], Over over) {
  if (over > 0) {
#pragma unroll
    for (int s = N / 2; s; s /= 2)
      if (over & s) {
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = j + s < N ? f[j + s < N ? j + s : 0] : 0.0f;
      }
    if (over >= N) {
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = 0.0f;
    }
  }
}
// Values col .. col+N-1 of a row of `cols`, zeros behind its last one; nothing outside the row is read.
template <typename T, int N, typename Col>
__device__ __forceinline__ void load_short(const T* row, Col col, Col cols, float (&f)[N]) {
  if (cols >= N) {
    const Col at = col < cols - N ? col : cols - N;
    widened(load_values<T, N>(row, at), f);
    moved_up(f, col - at);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = col + j < cols ? load_one(row + col + j) : 0.0f;
  }
}

// N values as elements of T from any element's alignment on; those from `left` on are not written.
template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, const float* f) {
  if constexpr (sizeof(T) == 4) {
    typedef float vec_t __attribute__((ext_vector_type(N < 4 ? N : 4), aligned(4)));
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      vec_t v;
#pragma unroll
      for (int j = 0; j < (N < 4 ? N : 4); ++j) v[j] = f[i + j];
      *reinterpret_cast<vec_t*>(p + i) = v;
    }
  } else if constexpr (N == 1) {
    p->bits = uint16_t(bf16_pair(f[0], 0.0f));
  } else {
    typedef uint32_t vec_t __attribute__((ext_vector_type(N / 2), aligned(2)));
    vec_t v;
#pragma unroll
    for (int i = 0; i < N; i += 2) v[i / 2] = bf16_pair(f[i], f[i + 1]);
    *reinterpret_cast<vec_t*>(p) = v;
  }
}
template <typename T, int N, typename Left>
__device__ __forceinline__ void store_values(T* p, const float (&f)[N], Left left) {
  static_assert(N == 4 || N == 8, "a vector");
  if (left >= N) {
    store_some<T, N>(p, f);
  } else if (left > 0) {
    float g[N];
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = f[j];
#pragma unroll
    for (int s = N / 2; s; s /= 2)
      if (left & s) {
        if (s == 4) store_some<T, 4>(p, g);
        else if (s == 2) store_some<T, 2>(p, g);
        else store_some<T, 1>(p, g);
        p += s;
#pragma unroll
        for (int j = 0; j < N; ++j) g[j] = j + s < N ? g[j + s < N ? j + s : 0] : 0.0f;
      }
  }
}

// Sum over the 64 lanes, in a fixed order; every lane receives it.
__device__ __forceinline__ float wave_sum_f32(float v) {
  v += u32_as_f32(dpp_u32<kDppQuadSwap1>(f32_as_u32(v)));
  v += u32_as_f32(dpp_u32<kDppQuadSwap2>(f32_as_u32(v)));
  v += u32_as_f32(dpp_u32<kDppRowHalfMirror>(f32_as_u32(v)));
  v += u32_as_f32(dpp_u32<kDppRowMirror>(f32_as_u32(v)));
  const float r0 = u32_as_f32(__builtin_amdgcn_readlane(f32_as_u32(v), 0));
  const float r1 = u32_as_f32(__builtin_amdgcn_readlane(f32_as_u32(v), 16));
  const float r2 = u32_as_f32(__builtin_amdgcn_readlane(f32_as_u32(v), 32));
  const float r3 = u32_as_f32(__builtin_amdgcn_readlane(f32_as_u32(v), 48));
  return (r0 + r1) + (r2 + r3);
}

// Maximum over 16 or 32 neighbouring lanes; every one of them receives it.
template <int LANES>
__device__ __forceinline__ float group_max(float v) {
  static_assert(LANES == 16 || LANES == 32, "a row of lanes, or two");
  v = fmaxf(v, u32_as_f32(dpp_u32<kDppQuadSwap1>(f32_as_u32(v))));
  v = fmaxf(v, u32_as_f32(dpp_u32<kDppQuadSwap2>(f32_as_u32(v))));
  v = fmaxf(v, u32_as_f32(dpp_u32<kDppRowHalfMirror>(f32_as_u32(v))));
  v = fmaxf(v, u32_as_f32(dpp_u32<kDppRowMirror>(f32_as_u32(v))));
  if constexpr (LANES == 32) v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return v;
}

// The exponent of a block's scale from its largest magnitude c: the smallest e >= kMinExponent with c <= 1.75 * 2^(top + e),
// top = 8 (E4M3, whose largest value is 448) or 15 (E5M2, 57344).  c's exponent field less top, and one more where
// its fraction is over .75: no rounding.  (A denormal c has the field 0 and ends at kMinExponent like all that small.)
__device__ __forceinline__ int block_exponent(float c, int code) {
  const uint32_t b = f32_as_u32(c);
  const int e = int(b >> 23) - 127 - (code == ACCEPT_E5M2 ? 15 : 8) + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < kMinExponent ? kMinExponent : e;
}
// 2^-e
__device__ __forceinline__ float inverse_scale(int e) { return u32_as_f32(uint32_t(127 - e) << 23); }

// Four values to four codes, the first in the low byte: the conversion instructions round to nearest even, and nothing here is
// beyond the largest code but infinities and NaN (E4M3: NaN; E5M2: themselves).
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, int code) {
  int r = 0;
  if (code == ACCEPT_E5M2) {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  }
  return uint32_t(r);
}

#endif  // __HIPCC__

}  // namespace accept
