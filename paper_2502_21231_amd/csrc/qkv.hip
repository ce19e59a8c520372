// Norm per head and position rotation of queries and keys, forward and backward, and appending to a
// paged key/value cache (gfx950).
//
// With x one head of one token, r = 1 / sqrt(mean(x^2) + eps), and R(t) the rotation of the pairs
// (a_i, b_i) by t f_i:
//   y = R(t) (x r w);
//   backward: g = R(-t) dy,  dw = sum g x r,  dx = r (g w - x r mean(g w x r)).
// All of it is read and written once, so the kernels are bound by memory.
//
// A head is held by D/8 lanes of eight elements, four pairs of the rotation in each: pairs (i, i +
// rot/2) are loaded as two runs of four elements from the two halves, so that no lane needs another's
// elements (for the norm's sum a few exchanges among the D/8 lanes are left).  A workgroup takes a
// token; its rows of lanes share the token's heads, and its angles, whose sines are taken once.
//
// Angles: t f in float64, reduced to a part of a turn there; at t = 2M a float32 angle would be off
// by up to 0.06.
#include "qkv.hpp"

namespace bs {
namespace {

struct RopeParams {
  const float* freq;
  const void* wq;
  const void* wk;
  int32_t rot, w_f32;
  float eps;
  const int64_t* pos;
  int64_t tokens;
  int32_t hq, hkv;
  Heads q, k, v;          // forward's inputs (v: append)
  void* q_out;
  void* k_out;
  const void* gq;         // backward: gradients of q_out, k_out
  const void* gk;
  Heads dq, dk;
  float* part;            // [blocks][2][D]: partial gradients of the weights, or NULL
  // append
  char* kc;
  char* vc;
  int64_t page_stride, token_stride, head_stride;  // elements
  int64_t num_pages, table_stride;
  const int32_t* table;
  const int32_t* kv_lens;
  const int32_t* cu_q;
  int32_t num_seqs, max_pages, page_shift;
};

// Four consecutive elements, as float.
__device__ __forceinline__ f32x4 load4(const bf16* p) {
  const bf16x4 x = *reinterpret_cast<const bf16x4*>(p);
  return f32x4{bf2f(x[0]), bf2f(x[1]), bf2f(x[2]), bf2f(x[3])};
}
__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ void store4(bf16* p, f32x4 x) {
  *reinterpret_cast<bf16x4*>(p) = bf16x4{f2bf(x[0]), f2bf(x[1]), f2bf(x[2]), f2bf(x[3])};
}
__device__ __forceinline__ void store4(float* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }

// The lane's eight elements of a head: pairs (a[e], b[e]).
struct Pairs {
  f32x4 a, b;
};

template <int D, bool kInter>
struct Lane {
  int ca, cb;   // element offsets of its two runs of four
  bool turned;  // whether its pairs are rotated, by frequencies f0 .. f0 + 3
  int f0;
  __device__ __forceinline__ Lane(int l, int rot) {
    turned = l < rot / 8;
    f0 = 4 * l;
    if (kInter) {
      ca = 8 * l;
      cb = ca + 4;
    } else if (turned) {
      ca = 4 * l;
      cb = ca + rot / 2;
    } else {  // the rest of the head, halved in the same way
      ca = rot + 4 * (l - rot / 8);
      cb = ca + (D - rot) / 2;
    }
  }
  template <typename T>
  __device__ __forceinline__ Pairs load(const T* row) const {
    const f32x4 x = load4(row + ca), y = load4(row + cb);
    if (kInter) return {f32x4{x[0], x[2], y[0], y[2]}, f32x4{x[1], x[3], y[1], y[3]}};
    return {x, y};
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const Pairs& p) const {
    if (kInter) {
      store4(row + ca, f32x4{p.a[0], p.b[0], p.a[1], p.b[1]});
      store4(row + cb, f32x4{p.a[2], p.b[2], p.a[3], p.b[3]});
    } else {
      store4(row + ca, p.a);
      store4(row + cb, p.b);
    }
  }
  __device__ __forceinline__ Pairs weight(const void* w, int is_f32) const {
    Pairs p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ia = kInter ? ca + 2 * e : ca + e, ib = kInter ? ca + 2 * e + 1 : cb + e;
      p.a[e] = is_f32 ? static_cast<const float*>(w)[ia] : bf2f(static_cast<const bf16*>(w)[ia]);
      p.b[e] = is_f32 ? static_cast<const float*>(w)[ib] : bf2f(static_cast<const bf16*>(w)[ib]);
    }
    return p;
  }
};

// Sum over the N lanes (a power of two up to 16) of a row; every lane gets the same bits.
template <int N>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int off = 1; off < N; off <<= 1) x += __shfl_xor(x, off);
  return x;
}

__device__ __forceinline__ float dot(const Pairs& x, const Pairs& y) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) s += x.a[e] * y.a[e] + x.b[e] * y.b[e];
  return s;
}

__device__ __forceinline__ void turn(Pairs& x, f32x4 c, f32x4 s) {
  const f32x4 a = x.a;
  x.a = a * c - x.b * s;
  x.b = x.b * c + a * s;
}

// cos and sin of t f: f32 arrays in LDS, written by the workgroup's first rot / 2 threads.
__device__ __forceinline__ void angles(const RopeParams& p, int64_t t, float* cs, float* sn) {
  const int i = threadIdx.x;
  if (i < p.rot / 2) {
    const double turns = (double)t * ((double)p.freq[i] * 0.15915494309189533577);  // 1 / 2 pi
    sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
  }
}

// One workgroup per token.  kAppend: keys and values into the cache, positions from its lengths.
template <typename T, int D, bool kInter, bool kAppend>
__global__ __launch_bounds__(256) void rope_fwd_kernel(const RopeParams p) {
  constexpr int LPR = D / 8, ROWS = 256 / LPR;
  __shared__ __attribute__((aligned(16))) float cs[D / 2], sn[D / 2];
  const int tid = threadIdx.x, l = tid % LPR;
  const int64_t tok = blockIdx.x;
  int64_t t;
  T* kd = nullptr;  // the token's place in the cache (head 0)
  T* vd = nullptr;
  if constexpr (kAppend) {
    // the sequence of the token: the last b with cu_q[b] <= tok (empty ones skipped)
    int lo = 0, hi = p.num_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.cu_q[mid] <= tok) lo = mid; else hi = mid - 1;
    }
    const int64_t first = p.cu_q[lo], end = p.cu_q[lo + 1];
    if (tok < first || tok >= end) return;  // behind the last sequence
    t = p.kv_lens[lo] - end + tok;
    const int64_t pg = t >> p.page_shift;
    if (t >= 0 && pg < p.max_pages) {
      const int64_t page = p.table[lo * p.table_stride + pg];
      if (page >= 0 && page < p.num_pages) {
        const int64_t at = page * p.page_stride + (t - (pg << p.page_shift)) * p.token_stride;
        kd = reinterpret_cast<T*>(p.kc) + at;
        vd = reinterpret_cast<T*>(p.vc) + at;
      }
    }
  } else {
    t = p.pos[tok];
  }
  angles(p, t, cs, sn);
  __syncthreads();
  const Lane<D, kInter> lane(l, p.rot);
  f32x4 c = f32x4{}, s = f32x4{};
  if (lane.turned) {
    c = *reinterpret_cast<const f32x4*>(cs + lane.f0);
    s = *reinterpret_cast<const f32x4*>(sn + lane.f0);
  }
  const T* q = static_cast<const T*>(p.q.p) + tok * p.q.stride;
  const T* k = static_cast<const T*>(p.k.p) + tok * p.k.stride;
  const int nq = p.q.p != nullptr ? p.hq : 0;
  for (int h = tid / LPR; h < nq + p.hkv; h += ROWS) {
    const bool is_q = h < nq;
    T* dst = is_q ? static_cast<T*>(p.q_out) + (tok * p.hq + h) * D
                  : (kAppend ? (kd != nullptr ? kd + (h - nq) * p.head_stride : nullptr)
                             : static_cast<T*>(p.k_out) + (tok * p.hkv + h - nq) * D);
    if (kAppend && dst == nullptr) continue;
    Pairs x = lane.load(is_q ? q + h * D : k + (h - nq) * D);
    const void* w = is_q ? p.wq : p.wk;
    if (w != nullptr) {
      const float r = rsqrtf(row_sum<LPR>(dot(x, x)) * (1.f / D) + p.eps);
      const Pairs wt = lane.weight(w, p.w_f32);
      x.a *= wt.a * r;
      x.b *= wt.b * r;
    }
    if (lane.turned) turn(x, c, s);
    lane.store(dst, x);
  }
  if constexpr (kAppend) {
    if (vd == nullptr) return;
    const T* v = static_cast<const T*>(p.v.p) + tok * p.v.stride;
    constexpr int E = 16 / sizeof(T);  // bits as they are
    for (int u = tid; u < p.hkv * (D / E); u += 256) {
      const int h = u / (D / E), e = u % (D / E) * E;
      *reinterpret_cast<u32x4*>(vd + h * p.head_stride + e) = *reinterpret_cast<const u32x4*>(v + h * D + e);
    }
  }
}

template <typename T, int D, bool kInter>
__global__ __launch_bounds__(256) void rope_bwd_kernel(const RopeParams p) {
  constexpr int LPR = D / 8, ROWS = 256 / LPR;
  __shared__ __attribute__((aligned(16))) float cs[D / 2], sn[D / 2];
  __shared__ __attribute__((aligned(16))) float acc[ROWS][D];
  const int tid = threadIdx.x, l = tid % LPR, row = tid / LPR;
  const Lane<D, kInter> lane(l, p.rot);
  Pairs dw[2] = {{f32x4{}, f32x4{}}, {f32x4{}, f32x4{}}};  // of the query's weight and the key's
  for (int64_t tok = blockIdx.x; tok < p.tokens; tok += gridDim.x) {
    __syncthreads();
    angles(p, p.pos[tok], cs, sn);
    __syncthreads();
    f32x4 c = f32x4{}, s = f32x4{};
    if (lane.turned) {
      c = *reinterpret_cast<const f32x4*>(cs + lane.f0);
      s = *reinterpret_cast<const f32x4*>(sn + lane.f0);
    }
    auto heads = [&](const Heads& x, const void* g, const Heads& dx, int n, const void* w, Pairs& dwx) {
      const Pairs wt = w != nullptr ? lane.weight(w, p.w_f32) : Pairs{f32x4{}, f32x4{}};
      for (int h = row; h < n; h += ROWS) {
        Pairs y = lane.load(static_cast<const T*>(g) + (tok * n + h) * D);
        if (lane.turned) turn(y, c, -s);
        if (w != nullptr) {
          Pairs xx = lane.load(static_cast<const T*>(x.p) + tok * x.stride + h * D);
          const float r = rsqrtf(row_sum<LPR>(dot(xx, xx)) * (1.f / D) + p.eps);
          xx.a *= r;
          xx.b *= r;
          dwx.a += y.a * xx.a;
          dwx.b += y.b * xx.b;
          y.a *= wt.a;
          y.b *= wt.b;
          const float m = row_sum<LPR>(dot(y, xx)) * (1.f / D);
          y.a = (y.a - xx.a * m) * r;
          y.b = (y.b - xx.b * m) * r;
        }
        lane.store(static_cast<T*>(dx.p) + tok * dx.stride + h * D, y);
      }
    };
    heads(p.q, p.gq, p.dq, p.hq, p.wq, dw[0]);
    heads(p.k, p.gk, p.dk, p.hkv, p.wk, dw[1]);
  }
  if (p.part == nullptr) return;
  for (int i = 0; i < 2; ++i) {
    __syncthreads();
    lane.store(acc[row], dw[i]);
    __syncthreads();
    for (int e = tid; e < D; e += 256) {
      float s = 0.f;
      for (int j = 0; j < ROWS; ++j) s += acc[j][e];
      p.part[((int64_t)blockIdx.x * 2 + i) * D + e] = s;
    }
  }
}

// dw[i][e] = sum over blocks of part[block][i][e]; one workgroup per (i, 16 elements).
__global__ __launch_bounds__(256) void rope_dw_kernel(const float* __restrict__ part, int blocks, int D,
                                                      float* dwq, float* dwk) {
  __shared__ float acc[16][17];
  const int e = threadIdx.x & 15, j = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + e;
  float s = 0.f;
  for (int b = j; b < blocks; b += 16) s += part[(int64_t)b * 2 * D + col];
  acc[j][e] = s;
  __syncthreads();
  if (j != 0) return;
  s = 0.f;
  for (int i = 0; i < 16; ++i) s += acc[i][e];
  float* out = col < D ? dwq : dwk;
  if (out != nullptr) out[col < D ? col : col - D] = s;
}

RopeParams params_of(const bs_dims& d, const bs_qk_params& P) {
  RopeParams p = {};
  p.freq = P.inv_freq;
  p.wq = P.q_weight;
  p.wk = P.k_weight;
  p.rot = P.rot_dim;
  p.w_f32 = P.weight_dtype == BS_F32;
  p.eps = P.eps;
  p.tokens = d.total_q;
  p.hq = d.hq;
  p.hkv = d.hkv;
  return p;
}

// Calls F<T, D, kInter> with the types of the call.
#define BS_ROPE_DISPATCH(CALL)                                                        \
  do {                                                                                \
    const bool inter = P.interleaved != 0, wide = d.head_dim == 128;                  \
    if (d.dtype == BS_BF16) {                                                         \
      if (wide) { if (inter) CALL(bf16, 128, true); else CALL(bf16, 128, false); }    \
      else { if (inter) CALL(bf16, 64, true); else CALL(bf16, 64, false); }           \
    } else {                                                                          \
      if (wide) { if (inter) CALL(float, 128, true); else CALL(float, 128, false); }  \
      else { if (inter) CALL(float, 64, true); else CALL(float, 64, false); }         \
    }                                                                                 \
  } while (0)

}  // namespace

hipError_t launch_qk_rope_fwd(const bs_dims& d, const bs_qk_params& P, Heads q, Heads k,
                              const int64_t* pos, void* q_out, void* k_out, hipStream_t stream) {
  if (d.total_q == 0) return hipSuccess;
  RopeParams p = params_of(d, P);
  p.pos = pos;
  p.q = q;
  p.k = k;
  p.q_out = q_out;
  p.k_out = k_out;
  const dim3 grid((unsigned)d.total_q);
#define BS_CALL(T, D, I) hipLaunchKernelGGL((rope_fwd_kernel<T, D, I, false>), grid, dim3(256), 0, stream, p)
  BS_ROPE_DISPATCH(BS_CALL);
#undef BS_CALL
  return hipGetLastError();
}

hipError_t launch_kv_append(const bs_dims& d, const bs_qk_params& P, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, Heads q, Heads k, Heads v,
                            void* q_out, hipStream_t stream) {
  if (d.total_q == 0 || num_seqs == 0) return hipSuccess;
  RopeParams p = params_of(d, P);
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_out = q_out;
  p.kc = static_cast<char*>(C.k);
  p.vc = static_cast<char*>(C.v);
  p.page_stride = C.page_stride;
  p.token_stride = C.token_stride;
  p.head_stride = C.head_stride;
  p.num_pages = C.num_pages;
  p.table_stride = C.table_stride;
  p.table = C.block_table;
  p.kv_lens = C.kv_lens;
  p.cu_q = cu_q;
  p.num_seqs = num_seqs;
  p.max_pages = C.max_pages;
  p.page_shift = __builtin_ctz((unsigned)C.page_size);
  const dim3 grid((unsigned)d.total_q);
#define BS_CALL(T, D, I) hipLaunchKernelGGL((rope_fwd_kernel<T, D, I, true>), grid, dim3(256), 0, stream, p)
  BS_ROPE_DISPATCH(BS_CALL);
#undef BS_CALL
  return hipGetLastError();
}

hipError_t launch_qk_rope_bwd(const bs_dims& d, const bs_qk_params& P, Heads q, Heads k,
                              const int64_t* pos, const void* dq_out, const void* dk_out, Heads dq,
                              Heads dk, float* dwq, float* dwk, float* part, hipStream_t stream) {
  RopeParams p = params_of(d, P);
  p.pos = pos;
  p.q = q;
  p.k = k;
  p.gq = dq_out;
  p.gk = dk_out;
  p.dq = dq;
  p.dk = dk;
  const bool sums = dwq != nullptr || dwk != nullptr;
  p.part = sums ? part : nullptr;
  const int blocks = (int)(d.total_q < kRopeBwdBlocks ? d.total_q : kRopeBwdBlocks);
  const dim3 grid((unsigned)blocks);
  if (blocks > 0) {
#define BS_CALL(T, D, I) hipLaunchKernelGGL((rope_bwd_kernel<T, D, I>), grid, dim3(256), 0, stream, p)
    BS_ROPE_DISPATCH(BS_CALL);
#undef BS_CALL
  }
  if (sums)
    hipLaunchKernelGGL(rope_dw_kernel, dim3((unsigned)(2 * d.head_dim / 16)), dim3(256), 0, stream, part, blocks,
                       d.head_dim, dwq, dwk);
  return hipGetLastError();
}

}  // namespace bs
