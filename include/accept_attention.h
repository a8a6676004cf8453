/*
 * accept_attention.h -- what a pipeline stage of a transformer computes between the product behind its norm and its second
 * product, for MI355X (gfx950): rotation of queries and keys by their position, attention over sequences with its gradients
 * for training, and keys and values in a cache of pages with the attention over it for serving.
 *
 * The conventions are those of accept.h and accept_stage.h: pointers named *_dev are DEVICE memory of the current HIP device;
 * the caller owns all buffers; kernels are enqueued on the given stream and not waited for; a call that fails validation
 * launches nothing and writes nothing; workspaces are scratch, one for each of the calls that overlap; outputs may not overlap
 * inputs or each other unless it is said; results do not depend on timing.
 *
 * Queries, keys, values and outputs are (tokens, heads, head_size): the values of a head next to each other, heads behind each
 * other, tokens `stride` elements apart (0: heads * head_size; at most 2^22), so a product's result that holds the three side by side is
 * taken as it is.  Pointers to them and to caches are 16-byte aligned and strides multiples of 16 bytes.  head_size is a multiple of 8, 8 to
 * 256.  heads is a multiple of kv_heads, 1 to 65535: query head h goes with key head h / (heads / kv_heads).
 *
 * Sequences lie behind each other, the tokens of sequence s from offsets_dev[s] to offsets_dev[s + 1] (sequences + 1 int32, the
 * first 0, none below the one before it; a sequence may be empty); a null pointer stands for sequences of tokens / sequences tokens each, which
 * has to divide.  Numbers beyond `tokens` are taken as `tokens`.  Tokens behind the last sequence belong to none: nothing of theirs is used, and their
 * outputs are left as they were (ACCEPT_REST_KEPT) or become zeros (ACCEPT_REST_ZEROS; logarithms of sums: minus infinity).
 */
#ifndef ACCEPT_ATTENTION_H
#define ACCEPT_ATTENTION_H

#include "accept_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ACCEPT_REST_KEPT = 0, ACCEPT_REST_ZEROS = 1 };
/* The two values of a pair that turns: values i and rotated/2 + i of a head, or 2i and 2i + 1. */
enum { ACCEPT_ROTATE_HALVES = 0, ACCEPT_ROTATE_NEIGHBOURS = 1 };

/*
 * ---- rotation by position ----------------------------------------------------------------------
 *
 *  dtype     of x and y (ACCEPT_F32, ACCEPT_BF16).
 *  rotated   values of a head that turn, its first ones: even, 0 to head_size; the others are copied.
 *  inverse   1: by the negative angle, which gives the gradient of x from that of y.
 *  tokens, sequences >= 0, below 2^31; tokens * stride <= 2^40.
 */
typedef struct {
  int32_t dtype;
  int32_t heads;
  int32_t head_size;
  int32_t rotated;
  int32_t pairs;
  int32_t inverse;
  int32_t rest;
  int32_t reserved; /* 0 */
  int64_t sequences;
  int64_t tokens;
  int64_t x_stride;
  int64_t y_stride;
} accept_rotate_desc;

/*
 * Pair i of a token at position p: (a, b) becomes (a cos t - b sin t, a sin t + b cos t) with t = p * frequencies_dev[i]
 * (rotated / 2 floats; the angle's remainder by a full turn is taken to 2^-100 of it, so far positions lose nothing),
 * rounded once.  positions_dev (tokens int32) null: a token's place in its sequence.  With positions offsets_dev is needed only to tell the
 * tokens of no sequence (null: there are none), and any number of sequences will do.  y_dev may be x_dev (with equal strides).
 */
accept_status accept_rotate(const accept_rotate_desc* desc, const void* x_dev, const float* frequencies_dev, const int32_t* offsets_dev,
                            const int32_t* positions_dev, void* y_dev, void* hip_stream);

/*
 * ---- attention over sequences ------------------------------------------------------------------
 *
 *  dtype     of all tensors but lse.
 *  causal    0: a query sees all keys of its sequence.  1: query i of n sees keys 0 .. i + m - n of m, so the last query sees
 *            the last key, and where there are more queries than keys the first ones see none.
 *  q_tokens, k_tokens, sequences  >= 0, below 2^31; tokens * stride <= 2^40.
 *  o_stride  of o and do;  dq_stride, dk_stride, dv_stride of the gradients.
 *  scale     of the products, 2^-100 to 2^100.
 *
 * heads * (larger of q_tokens and k_tokens / 32 + 2 * sequences + 2) is at most 2^23 (else ACCEPT_ERR_UNSUPPORTED): a launch's workgroups.
 */
typedef struct {
  int32_t dtype;
  int32_t heads;
  int32_t kv_heads;
  int32_t head_size;
  int32_t causal;
  int32_t rest;
  int64_t sequences;
  int64_t q_tokens;
  int64_t k_tokens;
  int64_t q_stride;
  int64_t k_stride;
  int64_t v_stride;
  int64_t o_stride;
  int64_t dq_stride;
  int64_t dk_stride;
  int64_t dv_stride;
  double  scale;
} accept_attention_desc;

/*
 * o_i = sum over the keys j that i sees of p_ij v_j, p_ij = exp(scale * q_i k_j - lse_i), lse_i = log(sum over j of exp(scale * q_i k_j)).
 * Rows that see no key: o = 0, lse = minus infinity.  Rows that see scores of minus infinity only: o = NaN, as the formula has it, lse = minus infinity,
 * and gradients as from there.  Rows that see a score that is NaN or plus infinity (also one that float32 does not hold): o and lse NaN.  What a row does not see has no effect on it,
 * infinities and NaN included.
 * lse_dev (heads x q_tokens floats) may be null.  Products and sums are float32's; with bfloat16 tensors p is rounded to
 * bfloat16 for its product with v, as an operand of the matrix instruction.  workspace_dev: accept_attention_workspace_size bytes, 16-byte aligned (null where that is 0).
 */
accept_status accept_attention_workspace_size(const accept_attention_desc* desc, size_t* bytes);
accept_status accept_attention(const accept_attention_desc* desc, const void* q_dev, const void* k_dev, const void* v_dev,
                               const int32_t* q_offsets_dev, const int32_t* k_offsets_dev, void* o_dev, float* lse_dev,
                               void* workspace_dev, void* hip_stream);

/*
 * Gradients, from what accept_attention returned: p_ij as above, with e_i = sum of do_i o_i and ds_ij = p_ij (do_i v_j - e_i) scale:
 * dq_i = sum of ds_ij k_j over the keys it sees, dk_j = sum of ds_ij q_i and dv_j = sum of p_ij do_i over the queries that see it, those of all
 * heads that share key head j.  Sums are float32's, in a fixed order; with bfloat16 tensors p and ds are rounded for their products.
 */
accept_status accept_attention_backward_workspace_size(const accept_attention_desc* desc, size_t* bytes);
accept_status accept_attention_backward(const accept_attention_desc* desc, const void* do_dev, const void* q_dev, const void* k_dev,
                                        const void* v_dev, const void* o_dev, const float* lse_dev, const int32_t* q_offsets_dev,
                                        const int32_t* k_offsets_dev, void* dq_dev, void* dk_dev, void* dv_dev,
                                        void* workspace_dev, void* hip_stream);

/*
 * ---- a cache of pages --------------------------------------------------------------------------
 *
 * k_cache_dev, v_cache_dev  (pages, kv_heads, page_size, head_size), all of it next to each other.
 * table_dev    (sequences, table_pages) int32: the pages of a sequence in order.  Place j of a sequence is place
 *              j % page_size of page table[j / page_size].  What a table holds behind a sequence's last page is not read.
 *              A page number outside 0 .. pages-1, and a place behind table_pages, is a place that does not exist: what goes
 *              there is dropped, and no token sees it.
 * lengths_dev  sequences int32: tokens of each in the cache before this step's (below 0: taken as 0).
 *
 * A step appends its new tokens (those of offsets_dev) to the places behind their sequence's length, then attends; both calls take
 * the same lengths, and the caller adds the new tokens to them for the next step.
 *
 *  dtype       of q, k, v, o and the caches.
 *  page_size   a power of two, 16 to 65536.  pages >= 0, table_pages >= 0, table_pages * page_size < 2^31;
 *              pages * kv_heads * page_size * head_size <= 2^40.
 *  rotated, pairs  as in accept_rotate_desc.
 *  tree_words  0: new token i of a sequence sees the cached ones and new tokens 0 .. i.  Otherwise it sees the cached ones
 *              and new token j where bit j % 64 of word tree_dev[token * tree_words + j / 64] is set (its own bit is no exception).  0 to 64.
 *  q_stride    of q (accept_cache_append: of its input);  qo_stride of its rotated output.  o_stride of o.
 *  scale       as in accept_attention_desc.
 *
 * tokens * heads / 32 + kv_heads * (sequences + 1) is at most 2^23 (else ACCEPT_ERR_UNSUPPORTED).
 */
typedef struct {
  int32_t dtype;
  int32_t heads;
  int32_t kv_heads;
  int32_t head_size;
  int32_t page_size;
  int32_t rotated;
  int32_t pairs;
  int32_t tree_words;
  int32_t rest;
  int32_t reserved; /* 0 */
  int64_t sequences;
  int64_t tokens;
  int64_t pages;
  int64_t table_pages;
  int64_t q_stride;
  int64_t k_stride;
  int64_t v_stride;
  int64_t o_stride;
  int64_t qo_stride;
  double  scale;
} accept_cache_desc;

/*
 * k (rotated) and v of the new tokens into their places, q (rotated) into qo_dev, which may be q_dev (with equal strides); both may be null.
 * A token's position is its place, unless positions_dev (tokens int32) says another (tokens of a tree: all that continue the
 * same one share a position).  frequencies_dev may be null where rotated is 0.  Two tokens that the table gives one place leave either's values.
 */
accept_status accept_cache_append(const accept_cache_desc* desc, const void* q_dev, const void* k_dev, const void* v_dev,
                                  const float* frequencies_dev, const int32_t* offsets_dev, const int32_t* lengths_dev,
                                  const int32_t* positions_dev, const int32_t* table_dev, void* qo_dev, void* k_cache_dev,
                                  void* v_cache_dev, void* hip_stream);

/*
 * o as accept_attention computes it, over a sequence's places 0 .. length + new - 1.  tree_dev (tokens, tree_words) uint64, null
 * where tree_words is 0.  A row that sees nothing becomes zeros.  workspace_dev: accept_cache_workspace_size bytes, 16-byte aligned.
 */
accept_status accept_cache_workspace_size(const accept_cache_desc* desc, size_t* bytes);
accept_status accept_cache_attention(const accept_cache_desc* desc, const void* q_dev, const void* k_cache_dev, const void* v_cache_dev,
                                     const int32_t* offsets_dev, const int32_t* lengths_dev, const int32_t* table_dev,
                                     const uint64_t* tree_dev, void* o_dev, void* workspace_dev, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ACCEPT_ATTENTION_H */
