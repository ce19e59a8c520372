// Attention of new tokens over a paged key/value cache (gfx950).
//
// bf16: rows of 32x32x16 MFMA blocks are (query, head of the KV group) pairs, row qi * group + hg, so
// that a group's heads share the keys they read, for one query of many heads as for many queries of
// one.  A workgroup takes 128 rows over blocks of 64 keys, 4 waves of 32 rows, in the orientation,
// with the swizzled tiles and the softmax of fwd_bf16.hip.  The work of all sequences is one line
// cut into equal ranges (paged_plan.hpp); a row block that several workgroups share leaves (O, max,
// sum) of each in float32, and paged_merge_kernel combines them.  Every workgroup lays out the line
// from the lengths itself: nothing but the shapes is known on the host, so that a captured call can be
// replayed with other lengths.
//
// Pages.  A wave copies 16 neighbouring keys of each tile, which lie in one page (page_size is a
// multiple of 16), so a page's place is scalar work, one number of the table per wave and tile, read
// a tile ahead.  Keys behind the sequence's end repeat its last one, as in fwd_bf16.hip; 16 keys of
// which none exists, or whose page is not there, are copied from a row of zeros: the probability of a
// hidden key is 0, but 0 times what the cache may hold there need not be.
//
// float32: a wave per token and query head, a lane per key for the scores of 64 keys, then a lane per
// D/64 elements of the head.
#include <type_traits>

#include "attn.hpp"
#include "paged_plan.hpp"
#include "qkv.hpp"

namespace bs {
namespace {

// A row of keys that are not there (never written).
__device__ __attribute__((aligned(256))) uint32_t g_zero_row[64];

// What the first workgroup of a shared row block leaves for the merge.
struct PagedShare {
  int32_t pieces;  // 0: none
  int32_t range;   // of its first workgroup
  int32_t hk, rows;
  int32_t row0;    // first row (of the group's rows of this segment)
  int32_t q_start;
  int32_t pad[2];
};

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
  PagedShare* share;  // [grid]
  float2* stat;       // [grid][2][BM] (max in log2 units, sum)
  float* part;        // [grid][2][BM][D]
  int64_t total_q;
  int32_t num_seqs, max_pages, page_shift, max_len;
  int32_t hq, hkv, group;
  int32_t causal;
  float scale_log2;
};

constexpr int kTileBM = 128, kTileBN = 64, kPagedGrid = 512;

struct PagedLds {
  int64_t pre[257];  // slots before the segments of each thread, per KV head
  int64_t wsum[4];
  int32_t bad;
};

__device__ __forceinline__ int32_t seqs_per_thread(int32_t n) { return (n + 255) >> 8; }

__device__ __forceinline__ PagedSeg paged_seg(const PagedParams& p, int32_t b) {
  return PagedSeg{p.cu_q[b + 1] - p.cu_q[b], p.kv_lens[b], p.group, p.causal};
}

__device__ __forceinline__ int64_t shfl_up64(int64_t x, int off) {
  const uint32_t lo = __shfl_up((uint32_t)x, off), hi = __shfl_up((uint32_t)((uint64_t)x >> 32), off);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Lays out the line (256 threads): pre[], and the slots per KV head; negative when the lengths are
// refused.  Block 0 writes the header.
template <int BM, int BLK>
__device__ __forceinline__ int64_t paged_line(const PagedParams& p, PagedLds& L) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  if (tid == 0) L.bad = BS_DEV_OK;
  __syncthreads();
  const int32_t pt = seqs_per_thread(p.num_seqs);
  int64_t sum = 0;
  int32_t code = BS_DEV_OK;
  for (int32_t i = 0; i < pt; ++i) {
    const int32_t b = tid * pt + i;
    if (b >= p.num_seqs) break;
    const int64_t n = (int64_t)p.cu_q[b + 1] - p.cu_q[b];
    const int32_t len = p.kv_lens[b];
    if (n < 0 || len < 0) code = BS_DEV_NOT_MONOTONE;
    else if (len > p.max_len) code = code == BS_DEV_OK ? BS_DEV_TOO_LONG : code;
    else if (n > p.total_q) code = BS_DEV_BAD_TOTAL;
    else if (n > 0) {
      const PagedCost c = paged_cost(PagedSeg{(int32_t)n, len, p.group, p.causal}, BM, BLK);
      sum += c.start(c.n);
    }
  }
  if (code != BS_DEV_OK) atomicCAS(&L.bad, BS_DEV_OK, code);
  int64_t run = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t x = shfl_up64(run, off);
    if (lane >= off) run += x;
  }
  if (lane == 63) L.wsum[w] = run;
  __syncthreads();
  if (tid == 0) {
    if (p.cu_q[0] != 0) L.bad = BS_DEV_BAD_FIRST;
    else if (L.bad == BS_DEV_OK && p.cu_q[p.num_seqs] > p.total_q) L.bad = BS_DEV_BAD_TOTAL;
  }
  int64_t at = run - sum;
  for (int i = 0; i < w; ++i) at += L.wsum[i];
  L.pre[tid] = at;
  if (tid == 255) L.pre[256] = at + sum;
  __syncthreads();
  const int32_t bad = L.bad;
  if (blockIdx.x == 0 && tid == 0) {
    p.hdr->status = bad;
    p.hdr->n_items = 0;
  }
  return bad == BS_DEV_OK ? L.pre[256] : -1;
}

// The piece that starts at slot x.  All of it is the same in every lane.
struct Piece {
  int32_t hk, seg, q_start, lq, lk;
  int32_t rb;      // row block
  int32_t kb, n;   // key blocks [kb, kb + n) of the row block's v; n <= 0: slots behind them
  int32_t v;
  int64_t xs;      // the row block's first slot
  int64_t next;    // the next row block's
};

template <int BM, int BLK>
__device__ __forceinline__ Piece paged_piece(const PagedParams& p, const PagedLds& L, int64_t line,
                                             int64_t x, int64_t x_end) {
  const int lane = threadIdx.x & 63;
  Piece c;
  int32_t hk = (int32_t)((double)x / (double)line);
  if (hk * line > x) --hk;
  if ((hk + 1) * line <= x) ++hk;
  const int64_t y = x - hk * line;
  int t = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) t += __popcll(__ballot(L.pre[i * 64 + lane] <= y));
  const int32_t pt = seqs_per_thread(p.num_seqs);
  int64_t before = L.pre[t];
  int32_t b = t;
  if (pt > 1) {  // (at most 64 segments per thread)
    const int32_t mine = t * pt + lane;
    int64_t cost = 0;
    if (lane < pt && mine < p.num_seqs) {
      const PagedSeg s = paged_seg(p, mine);
      if (s.lq > 0) {
        const PagedCost k = paged_cost(s, BM, BLK);
        cost = k.start(k.n);
      }
    }
    int64_t run = cost;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t z = shfl_up64(run, off);
      if (lane >= off) run += z;
    }
    const int64_t at = before + run - cost;
    const int k = __ffsll((unsigned long long)__ballot(cost > 0 && at <= y && y < at + cost)) - 1;
    b = t * pt + k;
    const uint32_t lo = __shfl((uint32_t)at, k), hi = __shfl((uint32_t)((uint64_t)at >> 32), k);
    before = (int64_t)(((uint64_t)hi << 32) | lo);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  c.hk = __builtin_amdgcn_readfirstlane(hk);
  c.seg = b;
  c.q_start = p.cu_q[b];
  const PagedSeg s = paged_seg(p, b);
  c.lq = s.lq;
  c.lk = s.lk;
  const PagedCost k = paged_cost(s, BM, BLK);
  c.rb = __builtin_amdgcn_readfirstlane(k.find(y - before));
  const int64_t first = before + k.start(c.rb);
  c.xs = hk * line + first;
  c.next = hk * line + before + k.start(c.rb + 1);
  c.kb = __builtin_amdgcn_readfirstlane((int32_t)(y - first));
  c.v = __builtin_amdgcn_readfirstlane(paged_blocks(s, BM, BLK, c.rb));
  const int64_t left = x_end - x;
  const int32_t rest = c.v - c.kb;
  c.n = __builtin_amdgcn_readfirstlane(rest < left ? rest : (int32_t)left);
  return c;
}

// One wave's copy of 16 rows (row r from src + min(r, last) * stride bytes) into 16 rows of a swizzled
// tile, as dma_tile copies them.
template <int D>
__device__ __forceinline__ void copy16(bf16* lds, const char* src, int stride, int last, int lane) {
  constexpr int CPR = D / 8, PER = 16 / (64 / CPR);
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)(src - 4096), 0, 0x7fffffff, 0x00020000);
  DmaRun<0, PER, D, 0>::issue(rs, lds, 0, lane / CPR, lane % CPR, stride >> 1, last);
}

constexpr float kRescaleBy = 8.0f;  // log2 units (fwd_bf16.hip)

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_tile_kernel(const PagedParams p) {
  constexpr int BM = kTileBM, BN = kTileBN, TILE = BN * D, KK = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) bf16 K0[TILE];
  __shared__ __attribute__((aligned(16))) bf16 K1[TILE];
  __shared__ __attribute__((aligned(16))) bf16 V0[TILE];
  __shared__ __attribute__((aligned(16))) bf16 V1[TILE];
  __shared__ PagedLds L;
  __shared__ __attribute__((aligned(16))) int32_t Miss[2][4];  // per buffer and 16 keys: the page is not there

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
  const int64_t line = paged_line<BM, BN>(p, L);
  PagedShare* share = p.share + blockIdx.x;
  if (line < 0) return;
  const PagedRanges R = paged_ranges(line * p.hkv, gridDim.x);
  const int32_t range = paged_range_of(blockIdx.x, R.active);
  if (range < 0) {
    if (tid == 0) share->pieces = 0;
    return;
  }
  int64_t x = range * R.per;
  const int64_t x_end = min(R.all, x + R.per);
  bool left_share = false;
  const int group = p.group;
  const float c2 = p.scale_log2;
  const int tstride = (int)p.token_stride;

  while (x < x_end) {
    const Piece e = paged_piece<BM, BN>(p, L, line, x, x_end);
    if (e.n <= 0) {
      x = e.next;
      continue;
    }
    x = e.kb + e.n == e.v ? e.next : x_end;
    const int rows = min((int)(e.lq * group - e.rb * BM), BM);
    const int qrow = w * 32 + c;
    const bool qvalid = qrow < rows;
    const uint32_t r_lane = (uint32_t)(e.rb * BM + (qvalid ? qrow : 0));
    const int qi = (int)(r_lane / (uint32_t)group), head = e.hk * group + (int)r_lane - qi * group;
    const int64_t orow = ((int64_t)e.q_start + qi) * p.hq + head;
    bf16x8 qf[KK];
    {
      const bf16* qp = static_cast<const bf16*>(p.q) + orow * D + hh * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);
    }
    const int diag = e.lk - e.lq;
    // keys below lim_base are visible to this lane's query (less the lane half's offset)
    const int lim_base = (p.causal ? min(e.lk, qi + diag + 1) : e.lk) - hh * 4;
    int full = e.lk;
    if (p.causal) full = min(full, (int)((uint32_t)(e.rb * BM) / (uint32_t)group) + diag + 1);
    const int n_full = full > 0 ? full / BN : 0;
    const int t0 = e.kb, n_tiles = e.kb + e.n;
    const int keys = e.lk;

    const int32_t* table = p.table + e.seg * p.table_stride;
    const int64_t hoff = e.hk * p.head_stride;
    // page of this wave's 16 keys of tile t (-1: behind the sequence's end)
    auto page_of = [&](int t) {
      const int key = t * BN + w * 16;
      return key < keys ? table[key >> p.page_shift] : -1;
    };
    auto copy = [&](int t, int page, bf16* Kd, bf16* Vd, int32_t* miss) {
      const int key = t * BN + w * 16;
      page = __builtin_amdgcn_readfirstlane(page);
      const bool there = page >= 0 && page < p.num_pages;
      const int64_t off = page * p.page_stride + (int64_t)(key & ((1 << p.page_shift) - 1)) * tstride + hoff;
      const char* ks = there ? p.kc + off : reinterpret_cast<const char*>(g_zero_row);
      const char* vs = there ? p.vc + off : reinterpret_cast<const char*>(g_zero_row);
      const int stride = there ? tstride : 0, last = min(15, keys - 1 - key);
      copy16<D>(Kd + w * 16 * D, ks, stride, last < 0 ? 0 : last, lane);
      copy16<D>(Vd + w * 16 * D, vs, stride, last < 0 ? 0 : last, lane);
      if (lane == 0) miss[w] = !there && key < keys;
    };

    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
    float m2 = -INFINITY, l_run = 0.f;

    copy(t0, page_of(t0), K0, V0, Miss[0]);
    int page = page_of(t0 + 1);
    wait_vmem_all();
    __syncthreads();

    auto step = [&](auto more, int t, const bf16* Kb, const bf16* Vb, const int32_t* miss, bf16* Kn,
                    bf16* Vn, int32_t* miss_n) {
      if constexpr (more()) {
        copy(t + 1, page, Kn, Vn, miss_n);
        page = page_of(t + 2);
      }
      f32x16 sacc[2] = {f32x16{}, f32x16{}};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const bf16x8 a = *reinterpret_cast<const bf16x8*>(&Kb[swz_off<D>(kb * 32 + c, kk * 2 + hh)]);
          sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kk], sacc[kb], 0, 0, 0);
        }
      }
      if (t >= n_full) {
        const int lim = lim_base - t * BN;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            sacc[kb][r] = (kb * 32 + (r >> 2) * 8 + (r & 3)) < lim ? sacc[kb][r] : -INFINITY;
      }
      if (__builtin_amdgcn_readfirstlane(miss[0] | miss[1] | miss[2] | miss[3])) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[kb][r] = miss[kb * 2 + (r >> 3)] ? -INFINITY : sacc[kb][r];
      }
      float mx = sacc[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[kb][r]);
      mx = half_max(mx) * c2;
      if (__any(mx > m2 + kRescaleBy)) {
        const float m_new = fmaxf(m2, mx);
        const float alpha = fast_exp2(m2 - (m_new == -INFINITY ? 0.f : m_new));
        m2 = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      }
      const float base = m2 == -INFINITY ? 0.f : m2;
      bf16x8 pb[4];  // P rounded to bf16 for the product; the sum takes it in float32
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float ex = fast_exp2(fmaf(sacc[kb][r], c2, -base));
          l_run += ex;
          pb[kb * 2 + (r >> 3)][r & 7] = f2bf(ex);
        }
      }
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const bf16x8 a = lds_read_tr2(Vb + swz_tr_off<D>(ks * 16, db * 32, 0, lane),
                                        Vb + swz_tr_off<D>(ks * 16, db * 32, 1, lane));
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[ks], oacc[db], 0, 0, 0);
        }
      }
      wait_vmem_all();
      __syncthreads();
    };
    for (int t = t0;; t += 2) {
      if (t + 1 == n_tiles) {
        step(std::false_type{}, t, K0, V0, Miss[0], K1, V1, Miss[1]);
        break;
      }
      step(std::true_type{}, t, K0, V0, Miss[0], K1, V1, Miss[1]);
      if (t + 2 == n_tiles) {
        step(std::false_type{}, t + 1, K1, V1, Miss[1], K0, V0, Miss[0]);
        break;
      }
      step(std::true_type{}, t + 1, K1, V1, Miss[1], K0, V0, Miss[0]);
    }

    const float l_tot = half_sum(l_run);
    const bool whole = e.n == e.v;
    // a range has at most one piece that goes on from the range before (slot 0) and one that another
    // range goes on with (slot 1)
    const int slot = e.kb == 0;
    if (!whole && slot) {
      left_share = true;
      if (tid == 0) {
        share->pieces = (int32_t)((e.xs + e.v - 1) / R.per - e.xs / R.per) + 1;
        share->range = range;
        share->hk = e.hk;
        share->rows = rows;
        share->row0 = e.rb * BM;
        share->q_start = e.q_start;
      }
    }
    if (qvalid && whole) {
      const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
      bf16* op = static_cast<bf16*>(p.o) + orow * D + hh * 4;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *reinterpret_cast<bf16x4*>(op + db * 32 + a * 8) =
              bf16x4{f2bf(oacc[db][a * 4 + 0] * inv), f2bf(oacc[db][a * 4 + 1] * inv),
                     f2bf(oacc[db][a * 4 + 2] * inv), f2bf(oacc[db][a * 4 + 3] * inv)};
      if (hh == 0)
        p.lse[head * p.total_q + e.q_start + qi] = l_tot > 0.f ? (m2 + log2f(l_tot)) * kLn2 : -INFINITY;
    } else if (qvalid) {
      const int64_t at = ((int64_t)range * 2 + slot) * BM + qrow;
      float* op = p.part + at * D + hh * 4;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *reinterpret_cast<f32x4*>(op + db * 32 + a * 8) =
              f32x4{oacc[db][a * 4 + 0], oacc[db][a * 4 + 1], oacc[db][a * 4 + 2], oacc[db][a * 4 + 3]};
      if (hh == 0) p.stat[at] = make_float2(m2, l_tot);
    }
  }
  if (!left_share && tid == 0) share->pieces = 0;
}

// Row blocks of several pieces: O = sum 2^(M_i - M) O_i / L, L = sum 2^(M_i - M) L_i, D/4 lanes per
// row.  The pieces are those of consecutive ranges: the first's slot 1, then slots 0.
template <int D, int BM>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedParams p) {
  constexpr int LPR = D / 4;
  if (p.hdr->status != BS_DEV_OK) return;
  const PagedShare s = p.share[blockIdx.x];
  if (s.pieces == 0) return;
  const int row = blockIdx.y * (256 / LPR) + threadIdx.x / LPR, ch = threadIdx.x % LPR;
  if (row >= s.rows) return;
  auto at = [&](int i) { return (((int64_t)s.range + i) * 2 + (i == 0)) * BM + row; };
  float M = -INFINITY;
  for (int i = 0; i < s.pieces; ++i) M = fmaxf(M, p.stat[at(i)].x);
  const float base = M == -INFINITY ? 0.f : M;
  float l = 0.f;
  f32x4 o = f32x4{};
  for (int i = 0; i < s.pieces; ++i) {
    const float2 st = p.stat[at(i)];
    const float wgt = fast_exp2(st.x - base);
    l += wgt * st.y;
    o += wgt * *reinterpret_cast<const f32x4*>(p.part + at(i) * D + ch * 4);
  }
  o *= l > 0.f ? 1.f / l : 0.f;
  const uint32_t r = (uint32_t)(s.row0 + row);
  const int qi = (int)(r / (uint32_t)p.group), head = s.hk * p.group + (int)r - qi * p.group;
  const int64_t tok = (int64_t)s.q_start + qi;
  *reinterpret_cast<bf16x4*>(static_cast<bf16*>(p.o) + (tok * p.hq + head) * D + ch * 4) =
      bf16x4{f2bf(o[0]), f2bf(o[1]), f2bf(o[2]), f2bf(o[3])};
  if (ch == 0) p.lse[head * p.total_q + tok] = l > 0.f ? (M + log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_row_kernel(const PagedParams p) {
  constexpr int E = D / 64;
  __shared__ float Q[4][D];
  __shared__ PagedLds L;
  if (paged_line<kTileBM, kTileBN>(p, L) < 0) return;
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

// Workspace: header, shares, statistics and sums of the ranges' pieces.
struct PagedLayout {
  int32_t grid;
  size_t share, stat, part, bytes;
};
PagedLayout paged_layout(const bs_dims& d) {
  PagedLayout L = {};
  if (d.dtype == BS_F32) {
    L.bytes = sizeof(WsHeader);
    return L;
  }
  L.grid = kPagedGrid;
  L.share = sizeof(WsHeader);
  L.stat = L.share + align256(sizeof(PagedShare) * (size_t)L.grid);
  L.part = L.stat + align256(sizeof(float2) * 2 * kTileBM * (size_t)L.grid);
  L.bytes = L.part + sizeof(float) * 2 * kTileBM * (size_t)L.grid * d.head_dim;
  return L;
}

}  // namespace

size_t paged_bytes(const bs_dims& d, int32_t, int32_t) { return paged_layout(d).bytes; }

hipError_t launch_paged_fwd(const bs_dims& d, const void* q, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, int32_t max_seqlen_k, int causal,
                            float scale, void* out, float* lse, void* ws, hipStream_t stream) {
  const int es = d.dtype == BS_BF16 ? 2 : 4;
  const PagedLayout W = paged_layout(d);
  char* base = static_cast<char*>(ws);
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
  p.share = reinterpret_cast<PagedShare*>(base + W.share);
  p.stat = reinterpret_cast<float2*>(base + W.stat);
  p.part = reinterpret_cast<float*>(base + W.part);
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
  if (d.dtype == BS_BF16) {
    const dim3 grid((unsigned)W.grid), mgrid((unsigned)W.grid, (unsigned)(kTileBM * d.head_dim / 1024));
#define BS_CALL(D)                                                                            \
  do {                                                                                        \
    hipLaunchKernelGGL((paged_tile_kernel<D>), grid, dim3(256), 0, stream, p);                \
    hipLaunchKernelGGL((paged_merge_kernel<D, kTileBM>), mgrid, dim3(256), 0, stream, p);     \
  } while (0)
    if (d.head_dim == 128) BS_CALL(128); else BS_CALL(64);
#undef BS_CALL
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((d.total_q * d.hq + 3) / 4 + (d.total_q == 0)));
  if (d.head_dim == 128) hipLaunchKernelGGL((paged_row_kernel<float, 128>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((paged_row_kernel<float, 64>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace bs
