// C ABI of the stage operators: argument validation and sizes, before anything is launched.
#include <math.h>

#include "stage.hpp"

using namespace accept;

namespace {

constexpr int64_t kMaxElems = int64_t(1) << 40;
constexpr int64_t kMaxSide = 0x7FFFFFFF;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t element(int32_t dtype) { return dtype == ACCEPT_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == ACCEPT_F32 || d == ACCEPT_BF16; }
bool is_code(int32_t c) { return c == ACCEPT_E4M3 || c == ACCEPT_E5M2; }
// rows >= 0 of `length` >= 0 elements, `stride` (0: `length`) apart
bool is_matrix(int64_t rows, int64_t length, int64_t stride) {
  if (rows < 0 || rows > kMaxSide || length < 0 || length > kMaxSide) return false;
  if (stride != 0 && stride < length) return false;
  const int64_t apart = stride ? stride : length;
  return apart == 0 || rows <= kMaxElems / apart;
}

accept_status check_norm(const accept_norm_desc* d) {
  if (!d || !is_dtype(d->x_dtype) || !is_dtype(d->y_dtype) || !is_dtype(d->param_dtype) || !is_code(d->code))
    return ACCEPT_ERR_INVALID_ARG;
  if (d->cols < 1 || !is_matrix(d->rows, d->cols, d->x_stride) || !is_matrix(d->rows, d->cols, d->y_stride) ||
      !is_matrix(d->rows, d->cols, d->dx_stride))
    return ACCEPT_ERR_INVALID_ARG;
  if (!isfinite(d->eps) || d->eps < 0) return ACCEPT_ERR_INVALID_ARG;
  return ACCEPT_OK;
}

accept_status check_block(const accept_block_desc* d) {
  if (!d || !is_dtype(d->in_dtype) || !is_code(d->code) || (d->group != 1 && d->group != kQBlock) || d->reserved != 0)
    return ACCEPT_ERR_INVALID_ARG;
  return is_matrix(d->rows, d->cols, d->x_stride) ? ACCEPT_OK : ACCEPT_ERR_INVALID_ARG;
}

accept_status check_matmul(const accept_matmul_desc* d) {
  if (!d || !is_dtype(d->out_dtype) || !is_code(d->a_code) || !is_code(d->b_code) || d->reserved != 0)
    return ACCEPT_ERR_INVALID_ARG;
  if ((d->a_group != 1 && d->a_group != kQBlock) || (d->b_group != 1 && d->b_group != kQBlock)) return ACCEPT_ERR_INVALID_ARG;
  const int64_t most = kMaxSide - kQBlock;
  if (d->m > most || d->n > most || d->k < 0 || d->k > most) return ACCEPT_ERR_INVALID_ARG;
  if (d->k > 0 && (d->a_stride % 16 != 0 || d->b_stride % 16 != 0)) return ACCEPT_ERR_INVALID_ARG;
  const int64_t k16 = up_to(d->k, 16), whole = accept_block_stride(d->k);
  if ((d->a_stride != 0 && d->a_stride < k16) || (d->b_stride != 0 && d->b_stride < k16)) return ACCEPT_ERR_INVALID_ARG;
  if (!is_matrix(d->m, d->n, d->y_stride) || !is_matrix(d->m, d->k, d->a_stride ? d->a_stride : whole) ||
      !is_matrix(d->n, d->k, d->b_stride ? d->b_stride : whole))
    return ACCEPT_ERR_INVALID_ARG;
  return ACCEPT_OK;
}

accept_status status(hipError_t e) { return e == hipSuccess ? ACCEPT_OK : ACCEPT_ERR_HIP; }

}  // namespace

extern "C" {

accept_status accept_layer_norm(const accept_norm_desc* desc, const void* x_dev, const void* weight_dev, const void* bias_dev,
                                void* y_dev, float* stats_dev, void* hip_stream) {
  const accept_status st = check_norm(desc);
  if (st != ACCEPT_OK) return st;
  if (desc->rows == 0) return ACCEPT_OK;
  if (!x_dev || !y_dev || !aligned(x_dev, element(desc->x_dtype)) || !aligned(y_dev, element(desc->y_dtype)) ||
      !aligned(weight_dev, element(desc->param_dtype)) || !aligned(bias_dev, element(desc->param_dtype)) || !aligned(stats_dev, 4))
    return ACCEPT_ERR_INVALID_ARG;
  return status(launch_norm(*desc, x_dev, weight_dev, bias_dev, y_dev, stats_dev, static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_layer_norm_quantize(const accept_norm_desc* desc, const void* x_dev, const void* weight_dev,
                                         const void* bias_dev, void* codes_dev, void* scales_dev, float* stats_dev,
                                         void* hip_stream) {
  const accept_status st = check_norm(desc);
  if (st != ACCEPT_OK) return st;
  if (desc->rows == 0) return ACCEPT_OK;
  if (!x_dev || !codes_dev || !scales_dev || !aligned(x_dev, element(desc->x_dtype)) || !aligned(codes_dev, 8) ||
      !aligned(weight_dev, element(desc->param_dtype)) || !aligned(bias_dev, element(desc->param_dtype)) || !aligned(stats_dev, 4))
    return ACCEPT_ERR_INVALID_ARG;
  return status(launch_norm_quantize(*desc, x_dev, weight_dev, bias_dev, codes_dev, scales_dev, stats_dev,
                                     static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_norm_workspace_size(const accept_norm_desc* desc, size_t* bytes) {
  const accept_status st = check_norm(desc);
  if (st != ACCEPT_OK) return st;
  if (!bytes) return ACCEPT_ERR_INVALID_ARG;
  *bytes = make_nplan(*desc).bytes;
  return ACCEPT_OK;
}

accept_status accept_layer_norm_backward(const accept_norm_desc* desc, const void* dy_dev, const void* x_dev,
                                         const void* weight_dev, const float* stats_dev, void* dx_dev, void* dweight_dev,
                                         void* dbias_dev, void* workspace_dev, void* hip_stream) {
  const accept_status st = check_norm(desc);
  if (st != ACCEPT_OK) return st;
  if (desc->rows > 0 && (!dy_dev || !x_dev || !stats_dev || !dx_dev)) return ACCEPT_ERR_INVALID_ARG;
  if ((dweight_dev || dbias_dev) && (!workspace_dev || !aligned(workspace_dev, 16))) return ACCEPT_ERR_INVALID_ARG;
  if (!aligned(dy_dev, element(desc->y_dtype)) || !aligned(x_dev, element(desc->x_dtype)) || !aligned(stats_dev, 4) ||
      !aligned(weight_dev, element(desc->param_dtype)) || !aligned(dx_dev, element(desc->x_dtype)) ||
      !aligned(dweight_dev, element(desc->param_dtype)) || !aligned(dbias_dev, element(desc->param_dtype)))
    return ACCEPT_ERR_INVALID_ARG;
  return status(launch_norm_backward(*desc, make_nplan(*desc), dy_dev, x_dev, weight_dev, stats_dev, dx_dev, dweight_dev,
                                     dbias_dev, workspace_dev, static_cast<hipStream_t>(hip_stream)));
}

int64_t accept_block_stride(int64_t length) { return length < 0 || length > kMaxElems ? -1 : up_to(length, kQBlock); }

accept_status accept_block_quantize(const accept_block_desc* desc, const void* x_dev, void* codes_dev, void* scales_dev,
                                    void* codes_t_dev, void* scales_t_dev, void* hip_stream) {
  const accept_status st = check_block(desc);
  if (st != ACCEPT_OK) return st;
  if (desc->rows == 0 || desc->cols == 0) return ACCEPT_OK;  // nothing to write
  if (!x_dev || (!codes_dev && !codes_t_dev) || !codes_dev != !scales_dev || !codes_t_dev != !scales_t_dev)
    return ACCEPT_ERR_INVALID_ARG;
  if (!aligned(x_dev, element(desc->in_dtype)) || !aligned(codes_dev, 16) || !aligned(codes_t_dev, 16))
    return ACCEPT_ERR_INVALID_ARG;
  return status(launch_block_quantize(*desc, x_dev, codes_dev, scales_dev, codes_t_dev, scales_t_dev,
                                      static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_matmul_workspace_size(const accept_matmul_desc* desc, size_t* bytes) {
  const accept_status st = check_matmul(desc);
  if (st != ACCEPT_OK) return st;
  if (!bytes) return ACCEPT_ERR_INVALID_ARG;
  *bytes = make_matmul_plan(*desc).bytes;
  return ACCEPT_OK;
}

accept_status accept_block_matmul(const accept_matmul_desc* desc, const void* a_dev, const void* a_scales_dev,
                                  const void* b_dev, const void* b_scales_dev, void* y_dev, void* workspace_dev, void* hip_stream) {
  const accept_status st = check_matmul(desc);
  if (st != ACCEPT_OK) return st;
  if (desc->m == 0 || desc->n == 0) return ACCEPT_OK;
  if (!y_dev || !aligned(y_dev, element(desc->out_dtype))) return ACCEPT_ERR_INVALID_ARG;
  if (desc->k > 0 && (!a_dev || !a_scales_dev || !b_dev || !b_scales_dev || !aligned(a_dev, 16) || !aligned(b_dev, 16)))
    return ACCEPT_ERR_INVALID_ARG;
  const MatmulPlan p = make_matmul_plan(*desc);
  if (p.bytes && (!workspace_dev || !aligned(workspace_dev, 16))) return ACCEPT_ERR_INVALID_ARG;
  return status(launch_matmul(*desc, p, a_dev, a_scales_dev, b_dev, b_scales_dev, y_dev, workspace_dev,
                              static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
