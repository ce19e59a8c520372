// Norm per head and position rotation of queries and keys, forward and backward, and appending to a
// paged key/value cache (gfx950).
//
// With x one head of one token, r = 1 / sqrt(mean(x^2) + eps), and R(t) the rotation of the pairs
// (a_i, b_i) by t f_i:
//   y = R(t) (x r w);
//   backward: g = R(-t) dy,  dw = sum g x r,  dx = r (g w - x r mean(g w x r)).
// All of it is read and written once, so the kernels are bound by memory: 32,768 tokens of 32/32 heads of 128 in bf16
// take 496 us forward and backward, 2.7 GB at 5.4 TB/s (a plain copy reaches 4.9), of which the backward's kernel 300;
// 8,191 tokens of 16/16 heads of 64 interleaved 34 us, 4.0 TB/s, since part of each launch is its start; a few tokens
// 8 us a call, the host's share of it.
//
// A head is held by D/8 lanes of eight elements, four pairs of the rotation in each: pairs (i, i +
// rot/2) are loaded as two runs of four elements from the two halves, so that no lane needs another's
// elements (for the norm's sum a few exchanges among the D/8 lanes are left).  A workgroup takes one, two or four
// tokens at a time, so many that each of its rows of lanes has up to four heads to request at once; a
// token's sines are taken once and shared through LDS.
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
  int32_t together;       // tokens of a workgroup at a time: 1, 2 or 4
};

// Four consecutive elements, as they are in memory and as float.
template <typename T> struct Four;
template <> struct Four<bf16> { typedef bf16x4 type; };
template <> struct Four<float> { typedef f32x4 type; };
__device__ __forceinline__ f32x4 wide(bf16x4 x) { return f32x4{bf2f(x[0]), bf2f(x[1]), bf2f(x[2]), bf2f(x[3])}; }
__device__ __forceinline__ f32x4 wide(f32x4 x) { return x; }
__device__ __forceinline__ bf16x4 narrow(f32x4 x, bf16*) { return bf16x4{f2bf(x[0]), f2bf(x[1]), f2bf(x[2]), f2bf(x[3])}; }
__device__ __forceinline__ f32x4 narrow(f32x4 x, float*) { return x; }
// kOnce: past the caches, for outputs that they could not hold.
template <bool kOnce, typename V>
__device__ __forceinline__ void put(V* p, V x) {
  if constexpr (kOnce) __builtin_nontemporal_store(x, p);
  else *p = x;
}
template <bool kOnce, typename T>
__device__ __forceinline__ void store4(T* p, f32x4 x) {
  put<kOnce>(reinterpret_cast<typename Four<T>::type*>(p), narrow(x, p));
}

// The lane's eight elements of a head: pairs (a[e], b[e]); as loaded, its two runs of four.
struct Pairs {
  f32x4 a, b;
};
template <typename T>
struct Runs {
  typename Four<T>::type a, b;
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
  __device__ __forceinline__ Runs<T> load(const T* row) const {
    typedef typename Four<T>::type V;
    return {*reinterpret_cast<const V*>(row + ca), *reinterpret_cast<const V*>(row + cb)};
  }
  template <typename T>
  __device__ __forceinline__ static Pairs pairs(const Runs<T>& r) {
    const f32x4 x = wide(r.a), y = wide(r.b);
    if (kInter) return {f32x4{x[0], x[2], y[0], y[2]}, f32x4{x[1], x[3], y[1], y[3]}};
    return {x, y};
  }
  template <bool kOnce, typename T>
  __device__ __forceinline__ void store(T* row, const Pairs& p) const {
    if (kInter) {
      store4<kOnce>(row + ca, f32x4{p.a[0], p.b[0], p.a[1], p.b[1]});
      store4<kOnce>(row + cb, f32x4{p.a[2], p.b[2], p.a[3], p.b[3]});
    } else {
      store4<kOnce>(row + ca, p.a);
      store4<kOnce>(row + cb, p.b);
    }
  }
};

// Sum over the N lanes (8 or 16 of a row of lanes) of a head; every lane gets the same bits.  Exchanges inside
// a row of 16 lanes are operands of the additions, not LDS traffic as a shuffle is.
template <int kCtrl>
__device__ __forceinline__ float row_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ float row_sum(float x) {
  x += row_move<0xB1>(x);   // quad_perm 1 0 3 2
  x += row_move<0x4E>(x);   // quad_perm 2 3 0 1
  x += row_move<0x141>(x);  // lane 7 - i of each 8
  if constexpr (N == 16) x += row_move<0x140>(x);  // lane 15 - i
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

// cos and sin of t f of a wave's token in LDS, by the lanes below rot / 2 <= 64.
template <int D>
__device__ __forceinline__ void angles(const RopeParams& p, int64_t t, float* cs, float* sn) {
  const int i = threadIdx.x & 63;
  if (i < p.rot / 2) {
    const double turns = (double)t * ((double)p.freq[i] * 0.15915494309189533577);  // 1 / 2 pi
    sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
  }
}

// The norms' weights as float in LDS (256 threads): the query's, then the key's.
template <int D>
__device__ __forceinline__ void stage_weights(const RopeParams& p, float* wt) {
  const int i = threadIdx.x / D, e = threadIdx.x % D;
  const void* w = i == 0 ? p.wq : p.wk;
  if (i < 2 && w != nullptr)
    wt[threadIdx.x] = p.w_f32 ? static_cast<const float*>(w)[e] : bf2f(static_cast<const bf16*>(w)[e]);
}

// The last b with cu_q[b] <= tok, by the lanes of a wave: 64 places at a time.
__device__ __forceinline__ int sequence_of(const int32_t* cu_q, int n, int64_t tok) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;  // among entries lo .. lo + len - 1
  while (len > 1) {
    const int step = (len + 63) >> 6, i = lane * step;
    const uint64_t m = __ballot(i < len && cu_q[lo + min(i, len - 1)] <= tok);
    const int k = m == 0 ? 0 : 63 - __clzll(m);
    lo += k * step;
    len = min(step, len - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Rows of lanes of a workgroup by token: `together` tokens share them, whole waves each.
struct Share {
  int sub, row, rows;  // this thread's token, its row among that token's, and how many those are
  bool first;          // whether its wave is the token's first
  template <int ROWS>
  static __device__ __forceinline__ Share of(int together, int row) {
    const int per = ROWS / together;
    Share s;
    s.sub = __builtin_amdgcn_readfirstlane(row / per);
    s.row = row - s.sub * per;
    s.rows = per;
    s.first = (threadIdx.x >> 6) * together % 4 == 0;
    return s;
  }
};

// A workgroup takes n = p.together tokens (one after another, 2,048 workgroups took
// 541 us for what takes 521 so); a row of D/8 lanes takes kRows heads at a time, all of them requested before the
// first is used (four: appending 10,000 tokens 46 us instead of 41).  kAppend: keys and values into the cache,
// positions from its lengths.
constexpr int kRows = 2;

template <typename T, int D, bool kInter, bool kAppend, bool kOnce>
__global__ __launch_bounds__(256) void rope_fwd_kernel(const RopeParams p) {
  constexpr int LPR = D / 8, ROWS = 256 / LPR, E = 16 / sizeof(T);
  __shared__ __attribute__((aligned(16))) float cs[4][D / 2], sn[4][D / 2];
  __shared__ __attribute__((aligned(16))) float wt[2 * D];
  const int tid = threadIdx.x, l = tid % LPR;
  const Lane<D, kInter> lane(l, p.rot);
  const Share sh = Share::of<ROWS>(p.together, tid / LPR);
  const int nq = p.q.p != nullptr ? p.hq : 0, n = nq + p.hkv;
  stage_weights<D>(p, wt);
  const int64_t tok = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * p.together + sh.sub;
  bool live = tok < p.tokens;
  const T* q = static_cast<const T*>(p.q.p) + tok * p.q.stride;
  const T* k = static_cast<const T*>(p.k.p) + tok * p.k.stride;
  Runs<T> in[kRows];
  auto request = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int h = h0 + i * sh.rows;
      if (live && h < n) in[i] = lane.load(h < nq ? q + h * D : k + (h - nq) * D);
    }
  };
  request(sh.row);
  int64_t t = 0;
  T* kd = nullptr;  // the token's place in the cache (head 0)
  T* vd = nullptr;
  if constexpr (kAppend) {
    const int b = sequence_of(p.cu_q, p.num_seqs, tok);
    const int64_t first = p.cu_q[b], end = p.cu_q[b + 1];
    live = live && tok >= first && tok < end;  // (no token, or behind the last sequence)
    t = p.kv_lens[b] - end + tok;
    const int64_t pg = t >> p.page_shift;
    if (live && t >= 0 && pg < p.max_pages) {
      const int64_t page = p.table[b * p.table_stride + pg];
      if (page >= 0 && page < p.num_pages) {
        const int64_t at = page * p.page_stride + (t - (pg << p.page_shift)) * p.token_stride;
        kd = reinterpret_cast<T*>(p.kc) + at;
        vd = reinterpret_cast<T*>(p.vc) + at;
      }
    }
  } else if (live) {
    t = p.pos[tok];
  }
  if (sh.first) angles<D>(p, t, cs[sh.sub], sn[sh.sub]);
  __syncthreads();
  f32x4 c = f32x4{}, s = f32x4{};
  if (lane.turned) {
    c = *reinterpret_cast<const f32x4*>(cs[sh.sub] + lane.f0);
    s = *reinterpret_cast<const f32x4*>(sn[sh.sub] + lane.f0);
  }
  for (int h0 = sh.row; live && h0 < n; h0 += kRows * sh.rows) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int h = h0 + i * sh.rows;
      if (h >= n) break;
      const bool is_q = h < nq;
      T* dst = is_q ? static_cast<T*>(p.q_out) + (tok * p.hq + h) * D
                    : (kAppend ? (kd != nullptr ? kd + (h - nq) * p.head_stride : nullptr)
                               : static_cast<T*>(p.k_out) + (tok * p.hkv + h - nq) * D);
      if (kAppend && dst == nullptr) break;
      Pairs x = lane.pairs(in[i]);
      if ((is_q ? p.wq : p.wk) != nullptr) {
        const float r = rsqrtf(row_sum<LPR>(dot(x, x)) * (1.f / D) + p.eps);
        const float* w = wt + (is_q ? 0 : D);
        const Pairs g = lane.pairs(lane.load(w));
        x.a *= g.a * r;
        x.b *= g.b * r;
      }
      if (lane.turned) turn(x, c, s);
      lane.template store<kOnce>(dst, x);
    }
    request(h0 + kRows * sh.rows);
  }
  if constexpr (kAppend) {
    if (vd == nullptr) return;
    const T* v = static_cast<const T*>(p.v.p) + tok * p.v.stride;
    const int mine = 256 / p.together;
    for (int u = tid & (mine - 1); u < p.hkv * (D / E); u += mine) {  // bits as they are
      const int h = u / (D / E), e = u % (D / E) * E;
      put<kOnce>(reinterpret_cast<u32x4*>(vd + h * p.head_stride + e), *reinterpret_cast<const u32x4*>(v + h * D + e));
    }
  }
}

template <typename T, int D, bool kInter, bool kOnce>
__global__ __launch_bounds__(256) void rope_bwd_kernel(const RopeParams p) {
  constexpr int LPR = D / 8, ROWS = 256 / LPR;
  __shared__ __attribute__((aligned(16))) float cs[2][4][D / 2], sn[2][4][D / 2];
  __shared__ __attribute__((aligned(16))) float wt[2 * D];
  __shared__ __attribute__((aligned(16))) float acc[ROWS][D];
  const int tid = threadIdx.x, l = tid % LPR, row = tid / LPR;
  const Lane<D, kInter> lane(l, p.rot);
  const Share sh = Share::of<ROWS>(p.together, row);
  const int n = p.hq + p.hkv;
  Pairs dwq = {f32x4{}, f32x4{}}, dwk = {f32x4{}, f32x4{}};
  stage_weights<D>(p, wt);
  int buf = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * p.together; t0 < p.tokens; t0 += (int64_t)gridDim.x * p.together, buf ^= 1) {
    const int64_t tok = t0 + sh.sub;
    const bool live = tok < p.tokens;
    Runs<T> gi, xi;  // (one head at a time: two at once cost registers, and so waves, 541 -> 531 us)
    auto request = [&](int h) {
      if (!live || h >= n) return;
      const bool is_q = h < p.hq;
      const int hh = is_q ? h : h - p.hq;
      gi = lane.load(static_cast<const T*>(is_q ? p.gq : p.gk) + (tok * (is_q ? p.hq : p.hkv) + hh) * D);
      if ((is_q ? p.wq : p.wk) != nullptr) {
        const Heads& x = is_q ? p.q : p.k;
        xi = lane.load(static_cast<const T*>(x.p) + tok * x.stride + hh * D);
      }
    };
    request(sh.row);
    if (sh.first && live) angles<D>(p, p.pos[tok], cs[buf][sh.sub], sn[buf][sh.sub]);
    __syncthreads();
    f32x4 c = f32x4{}, s = f32x4{};
    if (lane.turned) {
      c = *reinterpret_cast<const f32x4*>(cs[buf][sh.sub] + lane.f0);
      s = *reinterpret_cast<const f32x4*>(sn[buf][sh.sub] + lane.f0);
    }
    for (int h = sh.row; live && h < n; h += sh.rows) {
      const bool is_q = h < p.hq;
      Pairs y = lane.pairs(gi), xx = lane.pairs(xi);
      request(h + sh.rows);
      if (lane.turned) turn(y, c, -s);
      if ((is_q ? p.wq : p.wk) != nullptr) {
        const float r = rsqrtf(row_sum<LPR>(dot(xx, xx)) * (1.f / D) + p.eps);
        xx.a *= r;
        xx.b *= r;
        if (is_q) {
          dwq.a += y.a * xx.a;
          dwq.b += y.b * xx.b;
        } else {
          dwk.a += y.a * xx.a;
          dwk.b += y.b * xx.b;
        }
        const Pairs wg = lane.pairs(lane.load(static_cast<const float*>(wt + (is_q ? 0 : D))));
        y.a *= wg.a;
        y.b *= wg.b;
        const float m = row_sum<LPR>(dot(y, xx)) * (1.f / D);
        y.a = (y.a - xx.a * m) * r;
        y.b = (y.b - xx.b * m) * r;
      }
      const Heads& dx = is_q ? p.dq : p.dk;
      lane.template store<kOnce>(static_cast<T*>(dx.p) + tok * dx.stride + (is_q ? h : h - p.hq) * D, y);
    }
  }
  if (p.part == nullptr) return;
  for (int i = 0; i < 2; ++i) {
    __syncthreads();
    lane.template store<false>(acc[row], i == 0 ? dwq : dwk);
    __syncthreads();
    for (int e = tid; e < D; e += 256) {
      float s = 0.f;
      for (int j = 0; j < ROWS; ++j) s += acc[j][e];
      p.part[((int64_t)blockIdx.x * 2 + i) * D + e] = s;
    }
  }
}

// dw[i][e] = sum over blocks of part[block][i][e]; one workgroup per 16 of the 2 D columns, four of them to a lane
// and the blocks dealt to its 256 rows of four lanes.
__global__ __launch_bounds__(1024) void rope_dw_kernel(const float* __restrict__ part, int blocks, int D,
                                                       float* dwq, float* dwk) {
  __shared__ __attribute__((aligned(16))) f32x4 acc[256][4];
  const int e = threadIdx.x & 3, j = threadIdx.x >> 2;
  const float* src = part + blockIdx.x * 16 + e * 4;
  f32x4 s = f32x4{};
#pragma unroll
  for (int i = 0; i < kRopeBwdBlocks / 256; ++i)
    if (j + i * 256 < blocks) s += *reinterpret_cast<const f32x4*>(src + (int64_t)(j + i * 256) * 2 * D);
  acc[j][e] = s;
  for (int half = 128; half > 0; half >>= 1) {
    __syncthreads();
    if (j < half) acc[j][e] += acc[j + half][e];
  }
  if (j != 0) return;
  const int col = blockIdx.x * 16 + e * 4;
  float* out = col < D ? dwq : dwk;
  if (out == nullptr) return;
  for (int i = 0; i < 4; ++i) out[(col < D ? col : col - D) + i] = acc[0][e][i];
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

// Tokens that a workgroup takes at a time: as many (1, 2 or 4) as give each row of lanes up to `heads` heads, and no
// more than leave every CU eight workgroups.
int together_of(const bs_dims& d, int heads, int n) {
  const int rows = 256 / (d.head_dim / 8) * heads;
  int t = 1;
  while (t < 4 && 2 * t * n <= rows && d.total_q >= 2048 * 2 * t) t *= 2;
  return t;
}

// n workgroups, and some more in the last row (a dimension of a grid has less than 2^32 threads).
dim3 grid_of(int64_t n) {
  const int64_t x = n < (1 << 23) ? n : 1 << 23;
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

// Whether a call writes more than the eight L2s hold: then past them, since nothing would be found there
// (32,768 tokens, 32/32 heads, forward + backward 541 / 524 us; appending 10,000 tokens 46 / 43).
bool writes_once(const bs_dims& d) {
  return d.total_q * (d.hq + d.hkv) * d.head_dim * (d.dtype == BS_BF16 ? 2 : 4) > (int64_t(32) << 20);
}

// CALL(T, D, kInter, kOnce) with the types of the call.
#define BS_ROPE_TYPE(CALL, T, D)                                                                     \
  do {                                                                                               \
    if (P.interleaved != 0) { if (once) CALL(T, D, true, true); else CALL(T, D, true, false); }      \
    else { if (once) CALL(T, D, false, true); else CALL(T, D, false, false); }                       \
  } while (0)
#define BS_ROPE_DISPATCH(CALL)                                                                           \
  do {                                                                                                   \
    const bool once = writes_once(d);                                                                    \
    if (d.dtype == BS_BF16) {                                                                            \
      if (d.head_dim == 128) BS_ROPE_TYPE(CALL, bf16, 128); else BS_ROPE_TYPE(CALL, bf16, 64);           \
    } else {                                                                                             \
      if (d.head_dim == 128) BS_ROPE_TYPE(CALL, float, 128); else BS_ROPE_TYPE(CALL, float, 64);         \
    }                                                                                                    \
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
  p.together = together_of(d, kRows, d.hq + d.hkv);
  const dim3 grid = grid_of((d.total_q + p.together - 1) / p.together);
#define BS_CALL(T, D, I, O) hipLaunchKernelGGL((rope_fwd_kernel<T, D, I, false, O>), grid, dim3(256), 0, stream, p)
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
  p.together = together_of(d, kRows, (q.p != nullptr ? d.hq : 0) + d.hkv);
  const dim3 grid = grid_of((d.total_q + p.together - 1) / p.together);
#define BS_CALL(T, D, I, O) hipLaunchKernelGGL((rope_fwd_kernel<T, D, I, true, O>), grid, dim3(256), 0, stream, p)
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
  p.together = together_of(d, 1, d.hq + d.hkv);
  const int64_t need = (d.total_q + p.together - 1) / p.together;
  const int blocks = (int)(need < kRopeBwdBlocks ? need : kRopeBwdBlocks);
  const dim3 grid((unsigned)blocks);
  if (blocks > 0) {
#define BS_CALL(T, D, I, O) hipLaunchKernelGGL((rope_bwd_kernel<T, D, I, O>), grid, dim3(256), 0, stream, p)
    BS_ROPE_DISPATCH(BS_CALL);
#undef BS_CALL
  }
  if (sums)
    hipLaunchKernelGGL(rope_dw_kernel, dim3((unsigned)(2 * d.head_dim / 16)), dim3(1024), 0, stream, part, blocks,
                       d.head_dim, dwq, dwk);
  return hipGetLastError();
}

}  // namespace bs
