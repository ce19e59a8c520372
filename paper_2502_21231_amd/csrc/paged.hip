// Attention of new tokens over a paged key/value cache (gfx950).
//
// One wave per token and query head: a lane per key for the scores of 64 keys, a running maximum and
// sum, then a lane per D/64 elements of the head for the sum of the values.
#include "attn.hpp"
#include "qkv.hpp"

namespace bs {
namespace {

struct PagedParams {
  const void* q;
  void* o;
  float* lse;
  const char* kc;
  const char* vc;
  int64_t page_stride, token_stride, head_stride;  // bytes
  int64_t num_pages, table_stride;
  const int32_t* table;
  const int32_t* kv_lens;
  const int32_t* cu_q;
  WsHeader* hdr;
  int64_t total_q;
  int32_t num_seqs, max_pages, page_shift, max_len;
  int32_t hq, hkv, group;
  int32_t causal;
  float scale_log2;
};

// Checks cu_q and kv_lens (all threads of a workgroup); block 0 writes the header.
__device__ __forceinline__ bool paged_valid(const PagedParams& p) {
  __shared__ int32_t bad;
  const int tid = threadIdx.x;
  if (tid == 0) bad = BS_DEV_OK;
  __syncthreads();
  for (int b = tid; b < p.num_seqs; b += blockDim.x) {
    const int64_t n = (int64_t)p.cu_q[b + 1] - p.cu_q[b];
    const int32_t len = p.kv_lens[b];
    if (n < 0 || len < 0) atomicCAS(&bad, 0, BS_DEV_NOT_MONOTONE);
    else if (len > p.max_len) atomicCAS(&bad, 0, BS_DEV_TOO_LONG);
  }
  __syncthreads();
  if (tid == 0) {
    if (p.cu_q[0] != 0) bad = BS_DEV_BAD_FIRST;
    else if (p.cu_q[p.num_seqs] > p.total_q) bad = BS_DEV_BAD_TOTAL;
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    p.hdr->status = bad;
    p.hdr->n_items = 0;
  }
  return bad == BS_DEV_OK;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_row_kernel(const PagedParams p) {
  constexpr int E = D / 64;
  __shared__ float Q[4][D];
  if (!paged_valid(p)) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + w;
  if (row >= (int64_t)p.cu_q[p.num_seqs] * p.hq) return;
  const int64_t tok = row / p.hq;
  const int h = (int)(row - tok * p.hq), hk = h / p.group;
  int b = 0, hi = p.num_seqs - 1;
  while (b < hi) {
    const int mid = (b + hi + 1) >> 1;
    if (p.cu_q[mid] <= tok) b = mid; else hi = mid - 1;
  }
  const int len = p.kv_lens[b];
  const int64_t seen = p.causal ? (int64_t)len - p.cu_q[b + 1] + tok + 1 : len;
  const int keys = (int)(seen < 0 ? 0 : seen);
  const int32_t* table = p.table + b * p.table_stride;
  for (int e = 0; e < E; ++e) Q[w][lane * E + e] = (float)static_cast<const T*>(p.q)[row * D + lane * E + e];
  float m = -INFINITY, l = 0.f, o[E];
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  const int64_t head = hk * p.head_stride;
  auto place = [&](int key, bool& there) {
    const int64_t page = table[key >> p.page_shift];
    there = page >= 0 && page < p.num_pages;
    return (there ? page : 0) * p.page_stride + (int64_t)(key & ((1 << p.page_shift) - 1)) * p.token_stride + head;
  };
  for (int k0 = 0; k0 < keys; k0 += 64) {
    const int key = k0 + lane;
    bool there = false;
    float s = -INFINITY;
    int64_t at = 0;
    if (key < keys) at = place(key, there);
    if (there) {
      const T* kr = reinterpret_cast<const T*>(p.kc + at);
      float x = 0.f;
      for (int e = 0; e < D; ++e) x += (float)kr[e] * Q[w][e];
      s = x * p.scale_log2;
    }
    float mx = s;
    for (int off = 1; off < 64; off <<= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    if (mx == -INFINITY) continue;
    const float mn = fmaxf(m, mx);
    const float alpha = fast_exp2(m - mn), pr = there ? fast_exp2(s - mn) : 0.f;
    m = mn;
    l = l * alpha + pr;
    for (int e = 0; e < E; ++e) o[e] *= alpha;
    for (int j = 0; j < min(64, keys - k0); ++j) {
      const float pj = __shfl(pr, j);
      if (!__shfl((int)there, j)) continue;
      const T* vr = reinterpret_cast<const T*>(p.vc + __shfl(at, j));
      for (int e = 0; e < E; ++e) o[e] += pj * (float)vr[lane * E + e];
    }
  }
  for (int off = 1; off < 64; off <<= 1) l += __shfl_xor(l, off);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  for (int e = 0; e < E; ++e) static_cast<T*>(p.o)[row * D + lane * E + e] = (T)(o[e] * inv);
  if (lane == 0) p.lse[h * p.total_q + tok] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
}

}  // namespace

size_t paged_bytes(const bs_dims&, int32_t, int32_t) { return sizeof(WsHeader); }

hipError_t launch_paged_fwd(const bs_dims& d, const void* q, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, int32_t max_seqlen_k, int causal,
                            float scale, void* out, float* lse, void* ws, hipStream_t stream) {
  const int es = d.dtype == BS_BF16 ? 2 : 4;
  PagedParams p;
  p.q = q;
  p.o = out;
  p.lse = lse;
  p.kc = static_cast<const char*>(C.k);
  p.vc = static_cast<const char*>(C.v);
  p.page_stride = C.page_stride * es;
  p.token_stride = C.token_stride * es;
  p.head_stride = C.head_stride * es;
  p.num_pages = C.num_pages;
  p.table_stride = C.table_stride;
  p.table = C.block_table;
  p.kv_lens = C.kv_lens;
  p.cu_q = cu_q;
  p.hdr = static_cast<WsHeader*>(ws);
  p.total_q = d.total_q;
  p.num_seqs = num_seqs;
  p.max_pages = C.max_pages;
  p.page_shift = __builtin_ctz((unsigned)C.page_size);
  const int64_t room = (int64_t)C.max_pages * C.page_size;
  p.max_len = (int32_t)(max_seqlen_k < room ? max_seqlen_k : room);
  p.hq = d.hq;
  p.hkv = d.hkv;
  p.group = d.hq / d.hkv;
  p.causal = causal;
  p.scale_log2 = scale * kLog2e;
  const dim3 grid((unsigned)((d.total_q * d.hq + 3) / 4 + (d.total_q == 0)));
#define BS_CALL(T, D) hipLaunchKernelGGL((paged_row_kernel<T, D>), grid, dim3(256), 0, stream, p)
  if (d.dtype == BS_BF16) {
    if (d.head_dim == 128) BS_CALL(bf16, 128); else BS_CALL(bf16, 64);
  } else {
    if (d.head_dim == 128) BS_CALL(float, 128); else BS_CALL(float, 64);
  }
#undef BS_CALL
  return hipGetLastError();
}

}  // namespace bs
