/*
 * bs_qkv.h -- C ABI of the operators that stand around the attention of bs_attn.h, in the same
 * library (libbs_attn.so): queries and keys on their way from a model's projection to the attention
 * (norm per head, position rotation), and serving from a paged key/value cache (appending to it,
 * attention over it).
 *
 * Conventions are those of bs_attn.h (device pointers owned by the caller, no allocation, asynchronous
 * on `stream`, a status and bs_last_error() for what the host can check, BS_BF16 or BS_F32 data with
 * float32 arithmetic rounded once on the store, but where a call says otherwise, head_dim 64 or 128), and:
 *   - dims->total_q is the number of tokens T; dims->total_k is not used.
 *   - "strided" operands [T, heads, head_dim] have contiguous heads (heads x head_dim elements) and
 *     `stride` elements from one token to the next: at least heads x head_dim, a multiple of 16 bytes.
 *     So q, k and v may be parts of the one buffer that a fused projection writes.
 *   - An output may be the same memory as the input that it is computed from (same pointer, same
 *     stride); it must not overlap any other operand, nor that one in another way.
 */
#ifndef BS_QKV_H
#define BS_QKV_H

#include "bs_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What is done to each head x of a query or key at position t:
 *   norm (with a weight):  y = x / sqrt(mean(x^2) + eps) * weight;   without one y = x;
 *   rotation of the pairs (a_i, b_i), i < rot_dim / 2, of the first rot_dim elements by t inv_freq[i]:
 *     a' = a cos - b sin,  b' = b cos + a sin;
 *   pairs are elements (i, i + rot_dim / 2), or (2i, 2i + 1) with interleaved != 0; the other
 *   head_dim - rot_dim elements are not rotated.
 * The angle is formed and reduced in float64 (for |t| < 2^31 it is within 1e-6 of t inv_freq[i]), then rounded to a
 * float32 part of a turn; sine, cosine and the root are float32 functions of it (float32 results within some 6e-6 of
 * a head's largest element, 1.3e-7 in the norm of the whole). */
typedef struct {
  const float* inv_freq;  /* float32 [rot_dim / 2] on the device; NULL with rot_dim == 0 */
  int32_t rot_dim;        /* 0 (no rotation) .. head_dim, a multiple of 16 */
  int32_t interleaved;
  const void* q_weight;   /* [head_dim] of weight_dtype on the device, or NULL: queries are not normed */
  const void* k_weight;   /* the same for keys */
  int32_t weight_dtype;   /* bs_dtype; not looked at without weights */
  float eps;              /* finite, >= 0 */
} bs_qk_params;

/* q, k (strided) -> q_out [T, hq, head_dim], k_out [T, hkv, head_dim] (contiguous, as the attention
 * takes them).  positions: int64 [T].  Sequences packed into one buffer and shards of a longer one
 * (Sec. 2.3, Sec. 7 of the paper) differ in their positions only. */
int bs_qk_norm_rope_fwd(const bs_dims* dims, const bs_qk_params* params, const void* q,
                        int64_t q_stride, const void* k, int64_t k_stride,
                        const int64_t* positions, void* q_out, void* k_out, void* stream);

/* Bytes of workspace of the backward (0: invalid arguments). */
size_t bs_qk_norm_rope_workspace_size(const bs_dims* dims);

/* Gradients: dq_out [T, hq, head_dim], dk_out [T, hkv, head_dim] (contiguous) are those of q_out and
 * k_out; dq, dk (strided) those of q and k.  q and k are the forward's inputs (looked at only where
 * there is a weight; NULL is accepted otherwise).  dq_weight, dk_weight: float32 [head_dim],
 * overwritten with the sums over all tokens and heads; NULL where they are not wanted.  The sums run
 * in a fixed order: the same call gives the same bits.  The workspace needs no initialisation. */
int bs_qk_norm_rope_bwd(const bs_dims* dims, const bs_qk_params* params, const void* q,
                        int64_t q_stride, const void* k, int64_t k_stride,
                        const int64_t* positions, const void* dq_out, const void* dk_out, void* dq,
                        int64_t dq_stride, void* dk, int64_t dk_stride, float* dq_weight,
                        float* dk_weight, void* workspace, size_t workspace_bytes, void* stream);

/* A paged key/value cache.  Token t of sequence b, KV head h, lies in page
 * block_table[b * table_stride + t / page_size] at
 *   page * page_stride + (t % page_size) * token_stride + h * head_stride   (elements, in k and in v),
 * head_dim elements that follow one another.  [num_pages, page_size, hkv, head_dim] and
 * [num_pages, hkv, page_size, head_dim] are two such layouts.  An entry of the table outside
 * [0, num_pages) stands for a page that is not there: it is neither read nor written, and its keys
 * are visible to no query. */
typedef struct {
  void* k;
  void* v;
  int64_t num_pages;            /* 1 .. 2^31 - 1 */
  int64_t page_stride, token_stride, head_stride; /* > 0, multiples of 16 bytes */
  const int32_t* block_table;   /* on the device: num_seqs rows of max_pages entries */
  int64_t table_stride;         /* entries from one row to the next, >= max_pages */
  int32_t max_pages;            /* pages of a sequence at most */
  int32_t page_size;            /* tokens: a power of two from 16 to 4096; page_size * token_stride < 2^30 bytes */
  const int32_t* kv_lens;       /* on the device, [num_seqs]: tokens of each sequence, the new ones included */
} bs_paged_cache;

/* Appends the new tokens of a step: sequence b's are rows cu_seqlens_q[b] .. cu_seqlens_q[b+1]-1 (int32
 * [num_seqs + 1] on the device) of q, k, v (strided) and the last of its kv_lens[b] tokens, so row i
 * of n has position t = kv_lens[b] - n + i.  k goes through `params` (NULL: as it is) at that position
 * into the cache; v as it is.  With q != NULL, q goes through `params` into q_out [T, hq, head_dim]
 * (contiguous), which bs_attn_paged_fwd takes.
 *   - Rows from cu_seqlens_q[num_seqs] on (the padding of a captured batch) are left alone, and so is
 *     every other byte of the cache.  Tokens with t < 0 and tokens whose page is not there, or past
 *     max_pages, are not stored; their q_out is.
 *   - Whatever the three arrays hold, nothing outside the pages and q_out is written.
 *   - Two tokens of one call must not share a place in the cache; k and v share no element. */
int bs_kv_append(const bs_dims* dims, const bs_qk_params* params, const bs_paged_cache* cache,
                 const int32_t* cu_seqlens_q, int32_t num_seqs, const void* q, int64_t q_stride,
                 const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                 void* stream);

/* Bytes of workspace of bs_attn_paged_fwd (0: invalid arguments).  It depends on dims, num_seqs and
 * max_seqlen_k only, needs no initialisation, and holds nothing across calls except what
 * bs_read_device_status() reads.  A smaller call may need more than a larger one (its row blocks come in
 * parts); 66 MiB are enough for every call. */
size_t bs_attn_paged_workspace_size(const bs_dims* dims, int32_t num_seqs, int32_t max_seqlen_k);

/* Attention of the new tokens of each sequence (rows of q as in bs_kv_append; one, some or all of the
 * sequence's tokens) over its kv_lens[b] cached ones, formulas as in bs_attn.h.  With causal != 0 key
 * j is visible to row i of n iff j <= i + kv_lens[b] - n, otherwise all are.  q [T, hq, head_dim]
 * contiguous; writes out [T, hq, head_dim] and lse [hq, T]; a row that sees no key gets out = 0,
 * lse = -inf.  Rows from cu_seqlens_q[num_seqs] on are left as they were.  What the pages hold behind
 * a sequence's last token is not looked at (it may be NaN). Among what is: a key of NaN gives NaN in out and
 * lse of the rows that see it, and in no others; a value of NaN or infinity may also
 * give NaN in out of rows shortly before its token, which do not see it (0 times it).
 *   - bf16: a sequence of more than 32 rows (queries x heads of a KV group) has its probabilities rounded to
 *     bf16 before their product with V, as in bs_attn_varlen_fwd; of up to 32 rows they are within 2^-17.  LSE
 *     is that of the unrounded ones.
 *   - max_seqlen_k (below 2^30) bounds kv_lens.  num_seqs is at most 16,384, T hq below 2^31; sizes whose
 *     work cannot be numbered in 32 bits (some 2^31 blocks of 128 rows and 64 keys per KV head) are
 *     refused with BS_ERR_UNSUPPORTED.  lse overlaps no other operand either.
 *   - cu_seqlens_q and kv_lens are checked on the device: first entry not 0, a negative length, more
 *     rows than T, kv_lens beyond max_seqlen_k or the table give a status (BS_DEV_BAD_FIRST,
 *     BS_DEV_NOT_MONOTONE, BS_DEV_BAD_TOTAL, BS_DEV_TOO_LONG) that bs_read_device_status(workspace)
 *     reports, and nothing is written.
 *   - The shapes, and not the lengths, choose what is launched: a captured call may be replayed with
 *     other lengths, tables and numbers of rows (up to T) in the same arrays. */
int bs_attn_paged_fwd(const bs_dims* dims, const void* q, const bs_paged_cache* cache,
                      const int32_t* cu_seqlens_q, int32_t num_seqs, int32_t max_seqlen_k,
                      int causal, float scale, void* out, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BS_QKV_H */
