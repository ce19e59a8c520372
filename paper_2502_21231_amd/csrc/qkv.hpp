// Launchers behind bs_qkv.h: norm and rotation of queries and keys (qkv.hip), appending to a paged
// cache (qkv.hip), attention over it (paged.hip).  All enqueue on `stream`.
#pragma once

#include "../../include/bs_qkv.h"
#include "common.hpp"

namespace bs {

// Strided heads of tokens: element e of head h of token t at p[t * stride + h * head_dim + e].
struct Heads {
  void* p;
  int64_t stride;
};

hipError_t launch_qk_rope_fwd(const bs_dims& d, const bs_qk_params& P, Heads q, Heads k,
                              const int64_t* pos, void* q_out, void* k_out, hipStream_t stream);

// Workgroups of the backward at most, and so rows of its partial weight gradients.
constexpr int kRopeBwdBlocks = 1024;
inline size_t rope_bwd_bytes(int head_dim) {
  return sizeof(float) * 2 * (size_t)kRopeBwdBlocks * head_dim;
}
hipError_t launch_qk_rope_bwd(const bs_dims& d, const bs_qk_params& P, Heads q, Heads k,
                              const int64_t* pos, const void* dq_out, const void* dk_out, Heads dq,
                              Heads dk, float* dwq, float* dwk, float* part, hipStream_t stream);

// P.rot_dim == 0 and no weights: the tokens as they are.  q.p == NULL: keys and values only.
hipError_t launch_kv_append(const bs_dims& d, const bs_qk_params& P, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, Heads q, Heads k, Heads v,
                            void* q_out, hipStream_t stream);

constexpr int32_t kPagedMaxSeqs = 16384;
size_t paged_bytes(const bs_dims& d, int32_t num_seqs, int32_t max_seqlen_k);
// Whether one launch holds the call and its blocks can be counted in 32 bits (keys: of a sequence at most).
bool paged_fits(const bs_dims& d, int32_t num_seqs, int32_t max_seqlen_k, int64_t keys);
hipError_t launch_paged_fwd(const bs_dims& d, const void* q, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, int32_t max_seqlen_k, int causal,
                            float scale, void* out, float* lse, void* ws, hipStream_t stream);

}  // namespace bs
