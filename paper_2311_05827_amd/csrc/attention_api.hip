// C ABI of the attention operators: argument validation and sizes, before anything is launched.
#include "attention.hpp"

using namespace accept;

namespace {

constexpr int64_t kMaxElems = int64_t(1) << 40;
constexpr int64_t kMaxCount = 0x7FFFFFFF;
constexpr int kMaxHeads = 65535;
constexpr int64_t kMaxGroups = int64_t(1) << 23;  // workgroups of a launch: fewer than 2^32 threads

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool is_dtype(int32_t d) { return d == ACCEPT_F32 || d == ACCEPT_BF16; }
// float32 holds it times log2(e), and what it multiplies by that: masked products are minus infinity, whose multiple by 0 would be NaN
bool is_scale(double s) { return s >= 0x1p-100 && s <= 0x1p100; }
bool is_flag(int32_t v) { return v == 0 || v == 1; }
bool is_count(int64_t v) { return v >= 0 && v <= kMaxCount; }
bool are_heads(int32_t heads, int32_t kv_heads, int32_t head_size) {
  return kv_heads >= 1 && heads >= kv_heads && heads <= kMaxHeads && heads % kv_heads == 0 && head_size >= 8 && head_size <= 256 &&
         head_size % 8 == 0;
}
// tokens of heads * head_size elements, `stride` (0: as many) apart
bool are_tokens(int64_t tokens, int64_t heads, int64_t head_size, int64_t stride, int32_t dtype) {
  const int64_t whole = heads * head_size, apart = stride ? stride : whole;
  return apart >= whole && apart <= kMaxTokenStride && apart % (dtype == ACCEPT_F32 ? 4 : 8) == 0 && tokens <= kMaxElems / apart;
}
// sequences without offsets have tokens / sequences tokens each
bool divides(const void* offsets, int64_t sequences, int64_t tokens) {
  return offsets || (sequences == 0 ? tokens == 0 : tokens % sequences == 0);
}
bool same_stride(int64_t a, int64_t b, int64_t whole) { return (a ? a : whole) == (b ? b : whole); }
bool all_there(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!p || !aligned(p, 16)) return false;
  return true;
}

accept_status check_rotate(const accept_rotate_desc* d) {
  if (!d || !is_dtype(d->dtype) || !are_heads(d->heads, 1, d->head_size) || d->rotated < 0 || d->rotated > d->head_size || d->rotated % 2 ||
      !is_flag(d->pairs) || !is_flag(d->inverse) || !is_flag(d->rest) || d->reserved != 0)
    return ACCEPT_ERR_INVALID_ARG;
  if (!is_count(d->sequences) || !is_count(d->tokens) || !are_tokens(d->tokens, d->heads, d->head_size, d->x_stride, d->dtype) ||
      !are_tokens(d->tokens, d->heads, d->head_size, d->y_stride, d->dtype))
    return ACCEPT_ERR_INVALID_ARG;
  return ACCEPT_OK;
}

accept_status check_attention(const accept_attention_desc* d) {
  if (!d || !is_dtype(d->dtype) || !are_heads(d->heads, d->kv_heads, d->head_size) || !is_flag(d->causal) || !is_flag(d->rest))
    return ACCEPT_ERR_INVALID_ARG;
  if (!is_count(d->sequences) || !is_count(d->q_tokens) || !is_count(d->k_tokens) || !is_scale(d->scale))
    return ACCEPT_ERR_INVALID_ARG;
  for (const int64_t stride : {d->q_stride, d->o_stride, d->dq_stride})
    if (!are_tokens(d->q_tokens, d->heads, d->head_size, stride, d->dtype)) return ACCEPT_ERR_INVALID_ARG;
  for (const int64_t stride : {d->k_stride, d->v_stride, d->dk_stride, d->dv_stride})
    if (!are_tokens(d->k_tokens, d->kv_heads, d->head_size, stride, d->dtype)) return ACCEPT_ERR_INVALID_ARG;
  // a launch's workgroups: pieces of 32 tokens at least
  if (d->heads * ((d->q_tokens > d->k_tokens ? d->q_tokens : d->k_tokens) / 32 + 2 * d->sequences + 2) > kMaxGroups)
    return ACCEPT_ERR_UNSUPPORTED;
  return ACCEPT_OK;
}

accept_status check_cache(const accept_cache_desc* d) {
  if (!d || !is_dtype(d->dtype) || !are_heads(d->heads, d->kv_heads, d->head_size) || d->rotated < 0 || d->rotated > d->head_size ||
      d->rotated % 2 || !is_flag(d->pairs) || !is_flag(d->rest) || d->reserved != 0 || d->tree_words < 0 || d->tree_words > 64)
    return ACCEPT_ERR_INVALID_ARG;
  if (d->page_size < 16 || d->page_size > 65536 || (d->page_size & (d->page_size - 1)) != 0) return ACCEPT_ERR_INVALID_ARG;
  if (!is_count(d->sequences) || !is_count(d->tokens) || !is_count(d->pages) || !is_count(d->table_pages) ||
      d->table_pages * d->page_size > kMaxCount || !is_scale(d->scale))
    return ACCEPT_ERR_INVALID_ARG;
  if (d->pages > kMaxElems / (int64_t(d->kv_heads) * d->page_size * d->head_size)) return ACCEPT_ERR_INVALID_ARG;
  for (const int64_t stride : {d->q_stride, d->o_stride, d->qo_stride})
    if (!are_tokens(d->tokens, d->heads, d->head_size, stride, d->dtype)) return ACCEPT_ERR_INVALID_ARG;
  for (const int64_t stride : {d->k_stride, d->v_stride})
    if (!are_tokens(d->tokens, d->kv_heads, d->head_size, stride, d->dtype)) return ACCEPT_ERR_INVALID_ARG;
  if (d->kv_heads * (d->tokens * (d->heads / d->kv_heads) / 32 + d->sequences + 1) > kMaxGroups) return ACCEPT_ERR_UNSUPPORTED;
  return ACCEPT_OK;
}

accept_status status(hipError_t e) { return e == hipSuccess ? ACCEPT_OK : ACCEPT_ERR_HIP; }

}  // namespace

extern "C" {

accept_status accept_rotate(const accept_rotate_desc* desc, const void* x_dev, const float* frequencies_dev, const int32_t* offsets_dev,
                            const int32_t* positions_dev, void* y_dev, void* hip_stream) {
  const accept_status st = check_rotate(desc);
  if (st != ACCEPT_OK) return st;
  if (!positions_dev && !divides(offsets_dev, desc->sequences, desc->tokens)) return ACCEPT_ERR_INVALID_ARG;
  if (desc->tokens == 0) return ACCEPT_OK;
  if (!all_there({x_dev, y_dev}) || (desc->rotated > 0 && !frequencies_dev) || !aligned(frequencies_dev, 4) || !aligned(offsets_dev, 4) ||
      !aligned(positions_dev, 4) || (x_dev == y_dev && !same_stride(desc->x_stride, desc->y_stride, int64_t(desc->heads) * desc->head_size)))
    return ACCEPT_ERR_INVALID_ARG;
  return status(launch_rotate(*desc, x_dev, frequencies_dev, offsets_dev, positions_dev, y_dev, static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_attention_workspace_size(const accept_attention_desc* desc, size_t* bytes) {
  const accept_status st = check_attention(desc);
  if (st != ACCEPT_OK) return st;
  if (!bytes) return ACCEPT_ERR_INVALID_ARG;
  *bytes = make_attention_plan(*desc).bytes;
  return ACCEPT_OK;
}

accept_status accept_attention(const accept_attention_desc* desc, const void* q_dev, const void* k_dev, const void* v_dev,
                               const int32_t* q_offsets_dev, const int32_t* k_offsets_dev, void* o_dev, float* lse_dev,
                               void* workspace_dev, void* hip_stream) {
  const accept_status st = check_attention(desc);
  if (st != ACCEPT_OK) return st;
  if (!divides(q_offsets_dev, desc->sequences, desc->q_tokens) || !divides(k_offsets_dev, desc->sequences, desc->k_tokens))
    return ACCEPT_ERR_INVALID_ARG;
  if (desc->q_tokens == 0) return ACCEPT_OK;
  if (!all_there({q_dev, o_dev}) || (desc->k_tokens > 0 && !all_there({k_dev, v_dev})) || !aligned(q_offsets_dev, 4) ||
      !aligned(k_offsets_dev, 4) || !aligned(lse_dev, 4))
    return ACCEPT_ERR_INVALID_ARG;
  const AttentionPlan p = make_attention_plan(*desc);
  if (p.bytes && !all_there({workspace_dev})) return ACCEPT_ERR_INVALID_ARG;
  return status(launch_attention(*desc, p, q_dev, k_dev, v_dev, q_offsets_dev, k_offsets_dev, o_dev, lse_dev, workspace_dev,
                                 static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_attention_backward_workspace_size(const accept_attention_desc* desc, size_t* bytes) {
  const accept_status st = check_attention(desc);
  if (st != ACCEPT_OK) return st;
  if (!bytes) return ACCEPT_ERR_INVALID_ARG;
  *bytes = make_attention_back_plan(*desc).bytes;
  return ACCEPT_OK;
}

accept_status accept_attention_backward(const accept_attention_desc* desc, const void* do_dev, const void* q_dev, const void* k_dev,
                                        const void* v_dev, const void* o_dev, const float* lse_dev, const int32_t* q_offsets_dev,
                                        const int32_t* k_offsets_dev, void* dq_dev, void* dk_dev, void* dv_dev,
                                        void* workspace_dev, void* hip_stream) {
  const accept_status st = check_attention(desc);
  if (st != ACCEPT_OK) return st;
  if (!divides(q_offsets_dev, desc->sequences, desc->q_tokens) || !divides(k_offsets_dev, desc->sequences, desc->k_tokens))
    return ACCEPT_ERR_INVALID_ARG;
  if (desc->q_tokens == 0 && desc->k_tokens == 0) return ACCEPT_OK;
  if ((desc->q_tokens > 0 && (!all_there({do_dev, q_dev, o_dev, dq_dev}) || !lse_dev)) ||
      (desc->k_tokens > 0 && !all_there({k_dev, v_dev, dk_dev, dv_dev})) || !aligned(lse_dev, 4) || !aligned(q_offsets_dev, 4) ||
      !aligned(k_offsets_dev, 4))
    return ACCEPT_ERR_INVALID_ARG;
  const AttentionBackPlan p = make_attention_back_plan(*desc);
  if (p.bytes && !all_there({workspace_dev})) return ACCEPT_ERR_INVALID_ARG;
  return status(launch_attention_backward(*desc, p, do_dev, q_dev, k_dev, v_dev, o_dev, lse_dev, q_offsets_dev, k_offsets_dev, dq_dev,
                                          dk_dev, dv_dev, workspace_dev, static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_cache_append(const accept_cache_desc* desc, const void* q_dev, const void* k_dev, const void* v_dev,
                                  const float* frequencies_dev, const int32_t* offsets_dev, const int32_t* lengths_dev,
                                  const int32_t* positions_dev, const int32_t* table_dev, void* qo_dev, void* k_cache_dev,
                                  void* v_cache_dev, void* hip_stream) {
  const accept_status st = check_cache(desc);
  if (st != ACCEPT_OK) return st;
  if (!divides(offsets_dev, desc->sequences, desc->tokens)) return ACCEPT_ERR_INVALID_ARG;
  if (desc->tokens == 0) return ACCEPT_OK;
  if (!all_there({k_dev, v_dev}) || !q_dev != !qo_dev || !aligned(q_dev, 16) || !aligned(qo_dev, 16) ||
      (q_dev && q_dev == qo_dev && !same_stride(desc->q_stride, desc->qo_stride, int64_t(desc->heads) * desc->head_size)) || (desc->rotated > 0 && !frequencies_dev) ||
      !aligned(frequencies_dev, 4) || !aligned(offsets_dev, 4) || !aligned(positions_dev, 4))
    return ACCEPT_ERR_INVALID_ARG;
  if (desc->sequences > 0 && (!lengths_dev || !aligned(lengths_dev, 4) || (desc->table_pages > 0 && (!table_dev || !aligned(table_dev, 4)))))
    return ACCEPT_ERR_INVALID_ARG;
  if (desc->pages > 0 && !all_there({k_cache_dev, v_cache_dev})) return ACCEPT_ERR_INVALID_ARG;
  return status(launch_cache_append(*desc, q_dev, k_dev, v_dev, frequencies_dev, offsets_dev, lengths_dev, positions_dev, table_dev, qo_dev,
                                    k_cache_dev, v_cache_dev, static_cast<hipStream_t>(hip_stream)));
}

accept_status accept_cache_workspace_size(const accept_cache_desc* desc, size_t* bytes) {
  const accept_status st = check_cache(desc);
  if (st != ACCEPT_OK) return st;
  if (!bytes) return ACCEPT_ERR_INVALID_ARG;
  *bytes = make_cache_plan(*desc).bytes;
  return ACCEPT_OK;
}

accept_status accept_cache_attention(const accept_cache_desc* desc, const void* q_dev, const void* k_cache_dev, const void* v_cache_dev,
                                     const int32_t* offsets_dev, const int32_t* lengths_dev, const int32_t* table_dev,
                                     const uint64_t* tree_dev, void* o_dev, void* workspace_dev, void* hip_stream) {
  const accept_status st = check_cache(desc);
  if (st != ACCEPT_OK) return st;
  if (!divides(offsets_dev, desc->sequences, desc->tokens)) return ACCEPT_ERR_INVALID_ARG;
  if (desc->tokens == 0) return ACCEPT_OK;
  if (!all_there({q_dev, o_dev}) || !aligned(offsets_dev, 4) || (desc->tree_words > 0 && !tree_dev) || !aligned(tree_dev, 8))
    return ACCEPT_ERR_INVALID_ARG;
  if (desc->sequences > 0 && (!lengths_dev || !aligned(lengths_dev, 4) || (desc->table_pages > 0 && (!table_dev || !aligned(table_dev, 4)))))
    return ACCEPT_ERR_INVALID_ARG;
  if (desc->pages > 0 && !all_there({k_cache_dev, v_cache_dev})) return ACCEPT_ERR_INVALID_ARG;
  const CachePlan p = make_cache_plan(*desc);
  if (p.bytes && !all_there({workspace_dev})) return ACCEPT_ERR_INVALID_ARG;
  return status(launch_cache_attention(*desc, p, q_dev, k_cache_dev, v_cache_dev, offsets_dev, lengths_dev, table_dev, tree_dev, o_dev,
                                       workspace_dev, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
