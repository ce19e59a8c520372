// C ABI of bs_qkv.h: argument validation and launch order.
#include <math.h>

#include "capi.hpp"
#include "qkv.hpp"

namespace bs {
namespace {

int64_t esize(const bs_dims& d) { return d.dtype == BS_BF16 ? 2 : 4; }

// Sizes of a call on T tokens (total_k plays no part).
int check_sizes(const bs_dims* dims, bs_dims* d) {
  if (dims == nullptr) return fail(BS_ERR_INVALID_ARG, "dims is NULL");
  *d = *dims;
  d->total_k = 0;
  return check_dims(d, true);
}

int check_params(const bs_dims& d, const bs_qk_params* P) {
  if (P == nullptr) return fail(BS_ERR_INVALID_ARG, "params is NULL");
  if (P->rot_dim < 0 || P->rot_dim > d.head_dim || P->rot_dim % 16 != 0)
    return fail(BS_ERR_INVALID_ARG, "rot_dim = %d is not a multiple of 16 in [0, head_dim = %d]", P->rot_dim,
                d.head_dim);
  if (P->rot_dim > 0 && P->inv_freq == nullptr) return fail(BS_ERR_INVALID_ARG, "inv_freq is NULL");
  if (reinterpret_cast<uintptr_t>(P->inv_freq) % 4 != 0)
    return fail(BS_ERR_INVALID_ARG, "inv_freq is not aligned to its element size");
  if (P->q_weight == nullptr && P->k_weight == nullptr) return BS_OK;
  if (P->weight_dtype != BS_F32 && P->weight_dtype != BS_BF16)
    return fail(BS_ERR_UNSUPPORTED, "weight_dtype %d is not BS_F32 or BS_BF16", P->weight_dtype);
  const uintptr_t wsize = P->weight_dtype == BS_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(P->q_weight) % wsize != 0 || reinterpret_cast<uintptr_t>(P->k_weight) % wsize != 0)
    return fail(BS_ERR_INVALID_ARG, "a weight is not aligned to its element size");
  if (!isfinite(P->eps) || P->eps < 0.f) return fail(BS_ERR_INVALID_ARG, "eps must be finite and >= 0");
  return BS_OK;
}

// Strided heads of the call's tokens.
struct Rows {
  const void* p;
  int64_t stride, n;  // elements from token to token, and of a token
  const char* name;
};

int check_rows(const bs_dims& d, const Rows& r) {
  BS_TRY(check_ptr(r.p, d.total_q, r.name));
  if (r.stride < r.n || r.stride % (16 / esize(d)) != 0 || r.stride > INT64_MAX / 8 / (d.total_q + 1))
    return fail(BS_ERR_INVALID_ARG, "the stride of %s (%lld) must be at least %lld and a multiple of 16 bytes",
                r.name, (long long)r.stride, (long long)r.n);
  return BS_OK;
}

int64_t extent(const bs_dims& d, const Rows& r) {
  return d.total_q == 0 ? 0 : ((d.total_q - 1) * r.stride + r.n) * esize(d);
}

// Whether two operands share an element.  Rows of equal stride may lie between one another's.
bool share(const bs_dims& d, const Rows& a, const Rows& b) {
  if (a.p == nullptr || b.p == nullptr) return false;
  if (!overlaps(a.p, extent(d, a), b.p, extent(d, b))) return false;
  if (a.stride != b.stride) return true;
  const int64_t es = esize(d), s = a.stride * es;
  int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % s;
  if (off < 0) off += s;
  return off < a.n * es || off + b.n * es > s;
}

// An output may be the very operand `of` it is computed from, and shares nothing with the others.
int check_output(const bs_dims& d, const Rows& out, const Rows& of) {
  const bool same = out.p == of.p && out.stride == of.stride;
  if (!same && share(d, out, of))
    return fail(BS_ERR_INVALID_ARG, "%s overlaps %s without being equal to it", out.name, of.name);
  return BS_OK;
}
int check_apart(const bs_dims& d, const Rows& out, const Rows& other) {
  if (share(d, out, other)) return fail(BS_ERR_INVALID_ARG, "%s overlaps %s", out.name, other.name);
  return BS_OK;
}

int check_cache(const bs_dims& d, const bs_paged_cache* C, int32_t num_seqs) {
  if (C == nullptr) return fail(BS_ERR_INVALID_ARG, "cache is NULL");
  const int64_t es = esize(d), unit = 16 / es;
  if (C->num_pages < 1 || C->num_pages > INT32_MAX)
    return fail(BS_ERR_INVALID_ARG, "num_pages = %lld out of [1, 2^31)", (long long)C->num_pages);
  if (C->page_size < 16 || C->page_size > 4096 || (C->page_size & (C->page_size - 1)) != 0)
    return fail(BS_ERR_UNSUPPORTED, "page_size = %d is not a power of two from 16 to 4096", C->page_size);
  const int64_t strides[3] = {C->page_stride, C->token_stride, C->head_stride};
  for (int64_t s : strides)
    if (s <= 0 || s % unit != 0)
      return fail(BS_ERR_INVALID_ARG, "the cache's strides must be positive multiples of 16 bytes");
  if (C->token_stride >= (int64_t(1) << 30) / es / C->page_size)
    return fail(BS_ERR_UNSUPPORTED, "page_size * token_stride must be below 2^30 bytes");
  if (C->head_stride > INT64_MAX / 64 / kMaxHeads || C->page_stride > INT64_MAX / 64 / C->num_pages)
    return fail(BS_ERR_INVALID_ARG, "the cache's strides exceed the address range");
  BS_TRY(check_ptr(C->k, 1, "cache k"));
  BS_TRY(check_ptr(C->v, 1, "cache v"));
  if (C->max_pages < 0 || C->table_stride < C->max_pages || C->table_stride > INT32_MAX)
    return fail(BS_ERR_INVALID_ARG, "max_pages = %d must be in [0, table_stride = %lld]", C->max_pages,
                (long long)C->table_stride);
  if (num_seqs > 0 && (C->kv_lens == nullptr || (C->block_table == nullptr && C->max_pages > 0)))
    return fail(BS_ERR_INVALID_ARG, "block_table or kv_lens is NULL");
  if (reinterpret_cast<uintptr_t>(C->kv_lens) % 4 != 0 || reinterpret_cast<uintptr_t>(C->block_table) % 4 != 0)
    return fail(BS_ERR_INVALID_ARG, "block_table / kv_lens not aligned to their element size");
  return BS_OK;
}

int check_seqs(const int32_t* cu_q, int32_t num_seqs) {
  if (num_seqs < 0) return fail(BS_ERR_INVALID_ARG, "num_seqs = %d < 0", num_seqs);
  if (cu_q == nullptr) return fail(BS_ERR_INVALID_ARG, "cu_seqlens is NULL");
  if (reinterpret_cast<uintptr_t>(cu_q) % 4 != 0)
    return fail(BS_ERR_INVALID_ARG, "cu_seqlens is not aligned to its element size");
  return BS_OK;
}

// Bytes from the cache's first element to its last.
int64_t cache_extent(const bs_dims& d, const bs_paged_cache& C) {
  return ((C.num_pages - 1) * C.page_stride + (C.page_size - 1) * C.token_stride + (d.hkv - 1) * C.head_stride +
          d.head_dim) * esize(d);
}

int check_paged(const bs_dims& d, int32_t num_seqs, int32_t max_seqlen_k) {
  if (num_seqs < 0 || max_seqlen_k < 0)
    return fail(BS_ERR_INVALID_ARG, "num_seqs and max_seqlen_k must be >= 0");
  if (num_seqs > kPagedMaxSeqs)
    return fail(BS_ERR_UNSUPPORTED, "num_seqs = %d is above %d", num_seqs, kPagedMaxSeqs);
  if (max_seqlen_k >= kMaxTokens) return fail(BS_ERR_INVALID_ARG, "max_seqlen_k = %d is not below 2^30", max_seqlen_k);
  if (d.total_q * d.hq > INT32_MAX)
    return fail(BS_ERR_UNSUPPORTED, "total_q * hq = %lld is not below 2^31", (long long)(d.total_q * d.hq));
  return BS_OK;
}

Heads heads(const void* p, int64_t stride) { return Heads{const_cast<void*>(p), stride}; }

}  // namespace
}  // namespace bs

using namespace bs;

extern "C" {

int bs_qk_norm_rope_fwd(const bs_dims* dims, const bs_qk_params* params, const void* q,
                        int64_t q_stride, const void* k, int64_t k_stride,
                        const int64_t* positions, void* q_out, void* k_out, void* stream) {
  bs_dims d;
  BS_TRY(check_sizes(dims, &d));
  BS_TRY(check_params(d, params));
  const int64_t nq = (int64_t)d.hq * d.head_dim, nk = (int64_t)d.hkv * d.head_dim;
  const Rows Q = {q, q_stride, nq, "q"}, K = {k, k_stride, nk, "k"};
  const Rows QO = {q_out, nq, nq, "q_out"}, KO = {k_out, nk, nk, "k_out"};
  for (const Rows* r : {&Q, &K, &QO, &KO}) BS_TRY(check_rows(d, *r));
  if (d.total_q > 0 && (positions == nullptr || reinterpret_cast<uintptr_t>(positions) % 8 != 0))
    return fail(BS_ERR_INVALID_ARG, "positions is NULL or not 8-byte aligned");
  BS_TRY(check_output(d, QO, Q));
  BS_TRY(check_output(d, KO, K));
  BS_TRY(check_apart(d, QO, K));
  BS_TRY(check_apart(d, KO, Q));
  BS_TRY(check_apart(d, QO, KO));
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(BS_KERNEL_QK_ROPE, s);
  BS_HIP(launch_qk_rope_fwd(d, *params, heads(q, q_stride), heads(k, k_stride), positions, q_out, k_out, s),
         "norm and rotation launch");
  return ok();
}

size_t bs_qk_norm_rope_workspace_size(const bs_dims* dims) {
  bs_dims d;
  if (check_sizes(dims, &d) != BS_OK) return 0;
  ok();
  return rope_bwd_bytes(d.head_dim);
}

int bs_qk_norm_rope_bwd(const bs_dims* dims, const bs_qk_params* params, const void* q,
                        int64_t q_stride, const void* k, int64_t k_stride,
                        const int64_t* positions, const void* dq_out, const void* dk_out, void* dq,
                        int64_t dq_stride, void* dk, int64_t dk_stride, float* dq_weight,
                        float* dk_weight, void* workspace, size_t workspace_bytes, void* stream) {
  bs_dims d;
  BS_TRY(check_sizes(dims, &d));
  BS_TRY(check_params(d, params));
  const int64_t nq = (int64_t)d.hq * d.head_dim, nk = (int64_t)d.hkv * d.head_dim;
  // q and k are read only where their norm is undone
  const Rows Q = {params->q_weight != nullptr ? q : nullptr, q_stride, nq, "q"};
  const Rows K = {params->k_weight != nullptr ? k : nullptr, k_stride, nk, "k"};
  const Rows GQ = {dq_out, nq, nq, "dq_out"}, GK = {dk_out, nk, nk, "dk_out"};
  const Rows DQ = {dq, dq_stride, nq, "dq"}, DK = {dk, dk_stride, nk, "dk"};
  if (params->q_weight != nullptr) BS_TRY(check_rows(d, Q));
  if (params->k_weight != nullptr) BS_TRY(check_rows(d, K));
  for (const Rows* r : {&GQ, &GK, &DQ, &DK}) BS_TRY(check_rows(d, *r));
  if (d.total_q > 0 && (positions == nullptr || reinterpret_cast<uintptr_t>(positions) % 8 != 0))
    return fail(BS_ERR_INVALID_ARG, "positions is NULL or not 8-byte aligned");
  BS_TRY(check_output(d, DQ, Q));
  BS_TRY(check_output(d, DQ, GQ));
  BS_TRY(check_output(d, DK, K));
  BS_TRY(check_output(d, DK, GK));
  BS_TRY(check_apart(d, DQ, K));
  BS_TRY(check_apart(d, DQ, GK));
  BS_TRY(check_apart(d, DK, Q));
  BS_TRY(check_apart(d, DK, GQ));
  BS_TRY(check_apart(d, DQ, DK));
  if ((dq_weight != nullptr && params->q_weight == nullptr) || (dk_weight != nullptr && params->k_weight == nullptr))
    return fail(BS_ERR_INVALID_ARG, "the gradient of a weight that is NULL");
  if (dq_weight != nullptr || dk_weight != nullptr) {
    if (workspace == nullptr || reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
      return fail(BS_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < rope_bwd_bytes(d.head_dim))
      return fail(BS_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes,
                  rope_bwd_bytes(d.head_dim));
    if (reinterpret_cast<uintptr_t>(dq_weight) % 4 != 0 || reinterpret_cast<uintptr_t>(dk_weight) % 4 != 0)
      return fail(BS_ERR_INVALID_ARG, "dq_weight / dk_weight not aligned to their element size");
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(BS_KERNEL_QK_ROPE, s);
  BS_HIP(launch_qk_rope_bwd(d, *params, heads(q, q_stride), heads(k, k_stride), positions, dq_out, dk_out,
                            heads(dq, dq_stride), heads(dk, dk_stride), dq_weight, dk_weight,
                            static_cast<float*>(workspace), s),
         "norm and rotation backward launch");
  return ok();
}

int bs_kv_append(const bs_dims* dims, const bs_qk_params* params, const bs_paged_cache* cache,
                 const int32_t* cu_seqlens_q, int32_t num_seqs, const void* q, int64_t q_stride,
                 const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                 void* stream) {
  bs_dims d;
  BS_TRY(check_sizes(dims, &d));
  const bs_qk_params none = {};
  if (params == nullptr) params = &none;
  BS_TRY(check_params(d, params));
  BS_TRY(check_seqs(cu_seqlens_q, num_seqs));
  BS_TRY(check_cache(d, cache, num_seqs));
  const int64_t nq = (int64_t)d.hq * d.head_dim, nk = (int64_t)d.hkv * d.head_dim;
  const Rows Q = {q, q_stride, nq, "q"}, K = {k, k_stride, nk, "k"}, V = {v, v_stride, nk, "v"};
  const Rows QO = {q != nullptr ? q_out : nullptr, nq, nq, "q_out"};
  BS_TRY(check_rows(d, K));
  BS_TRY(check_rows(d, V));
  if (q != nullptr) {
    BS_TRY(check_rows(d, Q));
    BS_TRY(check_rows(d, QO));
    BS_TRY(check_output(d, QO, Q));
    BS_TRY(check_apart(d, QO, K));
    BS_TRY(check_apart(d, QO, V));
  }
  const int64_t bytes = cache_extent(d, *cache);
  for (const Rows* r : {&Q, &K, &V, &QO})
    if (r->p != nullptr && (overlaps(cache->k, bytes, r->p, extent(d, *r)) || overlaps(cache->v, bytes, r->p, extent(d, *r))))
      return fail(BS_ERR_INVALID_ARG, "%s overlaps the cache", r->name);
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(BS_KERNEL_KV_APPEND, s);
  BS_HIP(launch_kv_append(d, *params, *cache, cu_seqlens_q, num_seqs, heads(q, q_stride), heads(k, k_stride),
                          heads(v, v_stride), q_out, s),
         "cache append launch");
  return ok();
}

size_t bs_attn_paged_workspace_size(const bs_dims* dims, int32_t num_seqs, int32_t max_seqlen_k) {
  bs_dims d;
  if (check_sizes(dims, &d) != BS_OK || check_paged(d, num_seqs, max_seqlen_k) != BS_OK) return 0;
  ok();
  return paged_bytes(d, num_seqs, max_seqlen_k);
}

int bs_attn_paged_fwd(const bs_dims* dims, const void* q, const bs_paged_cache* cache,
                      const int32_t* cu_seqlens_q, int32_t num_seqs, int32_t max_seqlen_k,
                      int causal, float scale, void* out, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream) {
  bs_dims d;
  BS_TRY(check_sizes(dims, &d));
  BS_TRY(check_paged(d, num_seqs, max_seqlen_k));
  BS_TRY(check_seqs(cu_seqlens_q, num_seqs));
  BS_TRY(check_cache(d, cache, num_seqs));
  const int64_t qn = d.total_q * d.hq * d.head_dim, bytes = qn * esize(d), cb = cache_extent(d, *cache);
  BS_TRY(check_ptr(q, qn, "q"));
  BS_TRY(check_ptr(out, qn, "out"));
  BS_TRY(check_ptr(lse, d.total_q * d.hq, "lse"));
  if (overlaps(out, bytes, q, bytes)) return fail(BS_ERR_INVALID_ARG, "out overlaps q");
  if (overlaps(out, bytes, cache->k, cb) || overlaps(out, bytes, cache->v, cb))
    return fail(BS_ERR_INVALID_ARG, "out overlaps the cache");
  BS_TRY(check_scale(scale));
  const int64_t room = (int64_t)cache->max_pages * cache->page_size, most = max_seqlen_k < room ? max_seqlen_k : room;
  if (!paged_fits(d, num_seqs, max_seqlen_k, most))
    return fail(BS_ERR_UNSUPPORTED, "%lld rows of %d sequences over up to %lld keys are too many for one call",
                (long long)(d.total_q * d.hq), num_seqs, (long long)most);
  const size_t need = paged_bytes(d, num_seqs, max_seqlen_k);
  if (workspace == nullptr) return fail(BS_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) % 256 != 0)
    return fail(BS_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (workspace_bytes < need)
    return fail(BS_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
  const int64_t lb = d.total_q * d.hq * 4;
  if (overlaps(lse, lb, q, bytes) || overlaps(lse, lb, out, bytes) || overlaps(lse, lb, cache->k, cb) ||
      overlaps(lse, lb, cache->v, cb))
    return fail(BS_ERR_INVALID_ARG, "lse overlaps another operand");
  hipStream_t s = static_cast<hipStream_t>(stream);
  ProfScope ps(BS_KERNEL_PAGED, s);
  BS_HIP(launch_paged_fwd(d, q, *cache, cu_seqlens_q, num_seqs, max_seqlen_k, causal, scale, out, lse, workspace, s),
         "paged attention launch");
  return ok();
}

}  // extern "C"
