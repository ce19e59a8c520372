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

// What the first workgroup of a shared row block leaves for the merge: its pieces lie at `first` and
// then at next + i * step, i = 1 .. pieces - 1.
struct PagedShare {
  int32_t pieces;  // 0: none
  int32_t first, next, step;
  int32_t hk, rows;
  int32_t row0;    // first row (of the group's rows of this segment)
  int32_t q_start;
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
  PagedShare* share;  // [ranges], or [row blocks]
  float2* stat;       // [pieces][BM] (max in log2 units, sum)
  float* part;        // [pieces][BM][D]
  int32_t parts;      // kItems: workgroups of a row block at most
  int64_t total_q;
  int32_t num_seqs, max_pages, page_shift, max_len;
  int32_t hq, hkv, group;
  int32_t causal;
  float scale_log2;
};

constexpr int kTileBM = 128, kTileBN = 64, kFewBM = 32, kPagedGrid = 512;
constexpr int kPartTiles = 4;  // key tiles of a part at least

struct PagedLds {
  int64_t pre[257];  // slots before the segments of each thread, per KV head
  int64_t wsum[4];
  int32_t bad;
};

__device__ __forceinline__ int32_t seqs_per_thread(int32_t n) { return (n + 255) >> 8; }

__device__ __forceinline__ PagedSeg paged_seg(const PagedParams& p, int32_t b) {
  return PagedSeg{p.cu_q[b + 1] - p.cu_q[b], p.kv_lens[b], p.group, p.causal};
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int64_t shfl_up64(int64_t x, int off) {
  const uint32_t lo = __shfl_up((uint32_t)x, off), hi = __shfl_up((uint32_t)((uint64_t)x >> 32), off);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Lays out the line (256 threads): pre[], and the slots per KV head; negative when the lengths are
// refused.  Block 0 writes the header.  BLK == 0: row blocks are counted instead.
template <int BM, int BLK>
__device__ __forceinline__ int64_t segment_cost(const PagedSeg& s) {
  if constexpr (BLK == 0) {
    return paged_row_blocks(s, BM);
  } else {
    const PagedCost c = paged_cost(s, BM, BLK);
    return c.start(c.n);
  }
}
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
    else if (n > 0) sum += segment_cost<BM, BLK>(PagedSeg{(int32_t)n, len, p.group, p.causal});
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
    p.hdr->n_items = BLK == 0 && bad == BS_DEV_OK ? (int32_t)L.pre[256] : 0;  // row blocks per KV head
  }
  return uniform64(bad == BS_DEV_OK ? L.pre[256] : -1);
}

// The segment that holds place y of the line, and the places before it.  The same in every lane.
template <int BM, int BLK>
__device__ __forceinline__ int32_t find_segment(const PagedParams& p, const PagedLds& L, int64_t y,
                                                int64_t& before) {
  const int lane = threadIdx.x & 63;
  int t = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) t += __popcll(__ballot(L.pre[i * 64 + lane] <= y));
  const int32_t pt = seqs_per_thread(p.num_seqs);
  before = L.pre[t];
  int32_t b = t;
  if (pt > 1) {  // (at most 64 segments per thread)
    const int32_t mine = t * pt + lane;
    int64_t cost = 0;
    if (lane < pt && mine < p.num_seqs) {
      const PagedSeg s = paged_seg(p, mine);
      if (s.lq > 0) cost = segment_cost<BM, BLK>(s);
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
  return __builtin_amdgcn_readfirstlane(b);
}

// A part of a row block.  All of it is the same in every lane.
struct Piece {
  int32_t hk, seg, q_start, lq, lk;
  int32_t rb;      // row block
  int32_t kb, n;   // key blocks [kb, kb + n) of the row block's v; n <= 0: slots behind them
  int32_t v;
  int32_t at;      // its place among the pieces, where the row block is shared
  int64_t xs;      // kLine: the row block's first slot
  int64_t next;    // and the next row block's
};

// The piece that starts at slot x.
template <int BM, int BLK>
__device__ __forceinline__ Piece paged_piece(const PagedParams& p, const PagedLds& L, int64_t line,
                                             int64_t x, int64_t x_end, int32_t range) {
  Piece c;
  int32_t hk = (int32_t)((double)x / (double)line);
  if (hk * line > x) --hk;
  if ((hk + 1) * line <= x) ++hk;
  const int64_t y = x - hk * line;
  int64_t before;
  c.seg = find_segment<BM, BLK>(p, L, y, before);
  c.hk = __builtin_amdgcn_readfirstlane(hk);
  const PagedSeg s = paged_seg(p, c.seg);
  c.q_start = __builtin_amdgcn_readfirstlane(p.cu_q[c.seg]);
  c.lq = __builtin_amdgcn_readfirstlane(s.lq);
  c.lk = __builtin_amdgcn_readfirstlane(s.lk);
  const PagedCost k = paged_cost(s, BM, BLK);
  c.rb = __builtin_amdgcn_readfirstlane(k.find(y - before));
  const int64_t first = before + k.start(c.rb);
  c.xs = uniform64(hk * line + first);
  c.next = uniform64(hk * line + before + k.start(c.rb + 1));
  c.kb = __builtin_amdgcn_readfirstlane((int32_t)(y - first));
  c.v = __builtin_amdgcn_readfirstlane(paged_blocks(s, BM, BLK, c.rb));
  const int64_t left = x_end - x;
  const int32_t rest = c.v - c.kb;
  c.n = __builtin_amdgcn_readfirstlane(rest < left ? rest : (int32_t)left);
  // a range has at most one piece that goes on from the range before (place 0 of its two) and one that
  // another range goes on with (place 1)
  c.at = range * 2 + (c.kb == 0);
  return c;
}

// The piece of workgroup b: a part of a row block, the row blocks of one segment and head side by side on one
// XCD (b % 8), the longest first; line: row blocks per KV head.  false: none.
template <int BM, int BLK>
__device__ __forceinline__ bool paged_item(const PagedParams& p, const PagedLds& L, int64_t line, int32_t b,
                                           Piece& c) {
  const bool own = (p.hkv & 7) == 0;  // each XCD owns an eighth of the heads
  const int32_t hx = own ? p.hkv >> 3 : p.hkv, j = own ? b >> 3 : b;
  const int32_t i = j / (hx * p.parts);  // a row block's place, if all heads took turns
  if (i >= line) return false;
  int64_t before;
  c.seg = find_segment<BM, 0>(p, L, i, before);
  const PagedSeg s = paged_seg(p, c.seg);
  c.q_start = __builtin_amdgcn_readfirstlane(p.cu_q[c.seg]);
  c.lq = __builtin_amdgcn_readfirstlane(s.lq);
  c.lk = __builtin_amdgcn_readfirstlane(s.lk);
  const int32_t nrb = paged_row_blocks(s, BM);
  const int32_t r = j - (int32_t)before * hx * p.parts;  // of the segment's nrb * hx * parts
  int32_t hl, u;  // head; row block and part
  if (own) {
    hl = r / (nrb * p.parts);
    u = r - hl * nrb * p.parts;
  } else {
    u = r / hx;
    hl = r - u * hx;
  }
  const int32_t back = u / p.parts, part = u - back * p.parts;
  c.hk = __builtin_amdgcn_readfirstlane(own ? (b & 7) * hx + hl : hl);
  c.rb = __builtin_amdgcn_readfirstlane(nrb - 1 - back);
  c.v = __builtin_amdgcn_readfirstlane(paged_blocks(s, BM, BLK, c.rb));
  const int32_t parts = min(p.parts, max(1, c.v / kPartTiles));
  if (part >= parts) {
    c.n = 0;
    return true;
  }
  c.kb = part * c.v / parts;
  c.n = (part + 1) * c.v / parts - c.kb;
  // pieces and shares are numbered by head and row block
  c.at = __builtin_amdgcn_readfirstlane((c.hk * (int32_t)line + (int32_t)before + c.rb) * p.parts + part);
  return true;
}

// One wave's copy of 16 rows (row r from src + min(r, last) * stride bytes) into 16 rows of a swizzled
// tile, as dma_tile copies them.
template <int D, int AUX = 0>
__device__ __forceinline__ void copy16(bf16* lds, const char* src, int stride, int last, int lane) {
  constexpr int CPR = D / 8, PER = 16 / (64 / CPR);
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)(src - 4096), 0, 0x7fffffff, 0x00020000);
  DmaRun<0, PER, D, AUX>::issue(rs, lds, 0, lane / CPR, lane % CPR, stride >> 1, last);
}

constexpr float kRescaleBy = 8.0f;  // log2 units (fwd_bf16.hip)

// kLine: a workgroup per range of the line; otherwise per part of a row block.
template <int D, bool kLine>
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
  const int64_t line = paged_line<BM, kLine ? BN : 0>(p, L);
  if (line < 0) return;
  PagedShare* share = nullptr;
  PagedRanges R;
  int32_t range = 0;
  int64_t x = 0, x_end = 1;
  if constexpr (kLine) {
    share = p.share + blockIdx.x;
    R = paged_ranges(line * p.hkv, gridDim.x);
    R.per = uniform64(R.per);
    R.active = __builtin_amdgcn_readfirstlane(R.active);
    range = paged_range_of(blockIdx.x, R.active);
    if (range < 0) {
      if (tid == 0) share->pieces = 0;
      return;
    }
    x = range * R.per;
    x_end = min(R.all, x + R.per);
  }
  bool left_share = false;
  const int group = p.group;
  const float c2 = p.scale_log2;
  const int tstride = (int)p.token_stride;
  const int rbase = swz_row_base<D>(lane), tbase = swz_tr_base<D>(lane);

  while (x < x_end) {
    Piece e;
    if constexpr (kLine) {
      e = paged_piece<BM, BN>(p, L, line, x, x_end, range);
      if (e.n <= 0) {
        x = e.next;
        continue;
      }
      x = e.kb + e.n == e.v ? e.next : x_end;
    } else {
      if (!paged_item<BM, BN>(p, L, line, blockIdx.x, e) || e.n == 0) return;
      x = x_end;
    }
    const int rows = min((int)(e.lq * group - e.rb * BM), BM);
    const int qrow = w * 32 + c;
    const bool qvalid = qrow < rows;
    const uint32_t r_lane = (uint32_t)(e.rb * BM + (qvalid ? qrow : 0));
    bf16x8 qf[KK];
    int lim_base;  // keys below it are visible to this lane's query (less the lane half's offset)
    {
      const int qi = (int)(r_lane / (uint32_t)group), head = e.hk * group + (int)r_lane - qi * group;
      const int64_t orow = ((int64_t)e.q_start + qi) * p.hq + head;
      lim_base = (p.causal ? min(e.lk, qi + e.lk - e.lq + 1) : e.lk) - hh * 4;
      const bf16* qp = static_cast<const bf16*>(p.q) + orow * D + hh * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);
    }
    int full = e.lk;
    if (p.causal) full = min(full, (int)((uint32_t)(e.rb * BM) / (uint32_t)group) + e.lk - e.lq + 1);
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
          const bf16x8 a = lds_row16(Kb, (rbase ^ (kk << 5)) + kb * 64 * D);
          sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kk], sacc[kb], 0, 0, 0);
        }
      }
      // K reads two contraction steps ahead of the products, copies spread among them (fwd_bf16.hip)
      __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 4, 0);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        __builtin_amdgcn_sched_group_barrier(kSchedMfma, 2, 0);
        if constexpr (more()) __builtin_amdgcn_sched_group_barrier(kSchedVmem, 1, 0);
        if (kk + 2 < KK) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 2, 0);
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
          const bf16x8 a = lds_tr16(Vb, (tbase ^ (db << 6)) + ks * 32 * D,
                                    (tbase ^ ((db << 6) | 32)) + ks * 32 * D + 16 * D);
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
    if constexpr (kLine) {
      if (!whole && e.kb == 0) {
        left_share = true;
        if (tid == 0)
          *share = PagedShare{(int32_t)((e.xs + e.v - 1) / R.per - e.xs / R.per) + 1, e.at, range * 2, 2, e.hk, rows,
                              e.rb * BM, e.q_start};
      }
    } else if (p.parts > 1 && e.kb == 0) {
      const int32_t parts = whole ? 0 : min(p.parts, e.v / kPartTiles);
      if (tid == 0)
        p.share[e.at / p.parts] = PagedShare{parts, e.at, e.at, 1, e.hk, rows, e.rb * BM, e.q_start};
    }
    if (qvalid && whole) {
      uint32_t r = r_lane;
      asm volatile("" : "+v"(r));  // the row's place is worked out again: held over the loop, registers spill
      const int qi = (int)(r / (uint32_t)group), head = e.hk * group + (int)r - qi * group;
      const int64_t orow = ((int64_t)e.q_start + qi) * p.hq + head;
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
      const int64_t at = (int64_t)e.at * BM + qrow;
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
  if constexpr (kLine)
    if (!left_share && tid == 0) share->pieces = 0;
}

// Waits until at most N of this wave's copies are under way; until its LDS reads have returned (few_bf16.hip).
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | N);  // vmcnt(N), N < 16
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Few rows: 32 of them, and the four waves take the key tiles of a block of 4 KT keys, each with LDS buffers,
// page numbers and a softmax of its own; the layout is that of few_bf16.hip.  Per tile a wave reads the
// numbers of its KT / 16 pages in one load, a tile ahead of the copies that need them.
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_few_kernel(const PagedParams p) {
  constexpr int BM = kFewBM, KT = D == 128 ? 32 : 64, BLK = 4 * KT, NC = KT / 16;
  constexpr int KB = KT / 32, KK = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) bf16 Kt[4][KT * D];
  __shared__ __attribute__((aligned(16))) bf16 Vt[4][KT * D];
  __shared__ PagedLds L;
  __shared__ float Ms[4][32], Ls[4][32];

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
  const int64_t line = paged_line<BM, BLK>(p, L);
  if (line < 0) return;
  PagedShare* share = p.share + blockIdx.x;
  PagedRanges R = paged_ranges(line * p.hkv, gridDim.x);
  R.per = uniform64(R.per);
  R.active = __builtin_amdgcn_readfirstlane(R.active);
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
  const int rbase = swz_row_base<D>(lane), tbase = swz_tr_base<D>(lane);
  bf16* Kw = Kt[w];
  bf16* Vw = Vt[w];

  while (x < x_end) {
    const Piece e = paged_piece<BM, BLK>(p, L, line, x, x_end, range);
    if (e.n <= 0) {
      x = e.next;
      continue;
    }
    x = e.kb + e.n == e.v ? e.next : x_end;
    const int rows = min((int)(e.lq * group - e.rb * BM), BM);
    const uint32_t r_lane = (uint32_t)(e.rb * BM + min(c, rows - 1));
    const int qi = (int)(r_lane / (uint32_t)group), hg = (int)r_lane - qi * group;
    bf16x8 qf[KK];
    {
      const bf16* qp = static_cast<const bf16*>(p.q) +
                       (((int64_t)e.q_start + qi) * p.hq + e.hk * group + hg) * D + hh * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);
    }
    const int keys = e.lk;
    const int lim_lane = (p.causal ? min(keys, qi + keys - e.lq + 1) : keys) - hh * 4;
    // keys some row sees, and this piece's end
    int k_end = keys;
    if (p.causal) k_end = min(k_end, (int)((uint32_t)(e.rb * BM + rows - 1) / (uint32_t)group) + keys - e.lq + 1);
    if (e.kb + e.n < e.v) k_end = min(k_end, (e.kb + e.n) * BLK);

    const int32_t* table = p.table + e.seg * p.table_stride;
    const int64_t hoff = e.hk * p.head_stride;
    // lane i < NC: page of keys k .. k + 15 of its part of the tile at k0 (-1: behind the sequence's end)
    auto pages_of = [&](int k0) {
      const int key = k0 + lane * 16;
      return lane < NC && key < keys ? table[key >> p.page_shift] : -1;
    };
    // what a tile's copies need: place and stride of each 16 keys, their last row; the missing ones
    struct Place {
      int64_t off[NC];
      int there, miss;
    };
    auto place_of = [&](int pages, int k0) {
      Place a;
      a.there = a.miss = 0;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int page = __builtin_amdgcn_readlane(pages, i), key = k0 + i * 16;
        const bool there = page >= 0 && page < p.num_pages;
        a.off[i] = page * p.page_stride + (int64_t)(key & ((1 << p.page_shift) - 1)) * tstride + hoff;
        a.there |= there << i;
        a.miss |= (!there && key < keys) << i;
      }
      return a;
    };
    auto copy = [&](bf16* dst, const char* cache, const Place& a, int k0) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const bool there = (a.there >> i) & 1;
        const char* src = there ? cache + a.off[i] : reinterpret_cast<const char*>(g_zero_row);
        const int last = min(15, keys - 1 - k0 - i * 16);
        copy16<D, 2>(dst + i * 16 * D, src, there ? tstride : 0, last < 0 ? 0 : last, lane);
      }
    };

    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
    float m2 = -INFINITY, l_run = 0.f;

    int k0 = (e.kb * 4 + w) * KT;
    Place now;
    int ahead = -1;  // pages of the next tile
    // one tile; `more`: another follows (straight-line forms, so that the copies under way can be counted)
    auto step = [&](auto more) {
      wait_copies<8>();  // K has landed (V's eight copies may be under way)
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const bf16x8 a = lds_row16(Kw, (rbase ^ (kk << 5)) + kb * 64 * D);
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kk], s[kb], 0, 0, 0);
        }
      const int next = k0 + BLK, miss = now.miss;
      wait_reads();
      if constexpr (more()) {
        now = place_of(ahead, next);
        ahead = pages_of(next + BLK);
        copy(Kw, p.kc, now, next);
      }
      const int lim = lim_lane - k0;
      if (k0 + KT > keys || p.causal) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[kb][r] = (kb * 32 + (r >> 2) * 8 + (r & 3)) < lim ? s[kb][r] : -INFINITY;
      }
      if (miss) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[kb][r] = (miss >> (kb * 2 + (r >> 3))) & 1 ? -INFINITY : s[kb][r];
      }
      float mx = s[0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
      mx = half_max(mx) * c2;
      if (__any(mx > m2)) {
        const float m_new = fmaxf(m2, mx);
        const float alpha = fast_exp2(m2 - (m_new == -INFINITY ? 0.f : m_new));
        m2 = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      }
      const float base = m2 == -INFINITY ? 0.f : m2;
      bf16x8 pb[2 * KB];  // P rounded to bf16 for the product; the sum takes it in float32
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float ex = fast_exp2(fmaf(s[kb][r], c2, -base));
          l_run += ex;
          pb[kb * 2 + (r >> 3)][r & 7] = f2bf(ex);
        }
      // V has landed.  (At most K's eight copies and the pages' load come after it; where the load is
      // moved, waiting for one operation more than needed is all that happens.)
      wait_copies<more() ? 8 : 0>();
#pragma unroll
      for (int ks = 0; ks < 2 * KB; ++ks)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const bf16x8 a = lds_tr16(Vw, (tbase ^ (db << 6)) + ks * 32 * D,
                                    (tbase ^ ((db << 6) | 32)) + ks * 32 * D + 16 * D);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[ks], oacc[db], 0, 0, 0);
        }
      wait_reads();
      if constexpr (more()) copy(Vw, p.vc, now, next);
      k0 = next;
    };
    if (k0 < k_end) {
      now = place_of(pages_of(k0), k0);
      ahead = pages_of(k0 + BLK);
      copy(Kw, p.kc, now, k0);
      copy(Vw, p.vc, now, k0);
      // Q is waited for here: left to the loop, the compiler would wait for every copy there
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[kk]));
      while (k0 + BLK < k_end) step(std::true_type{});
      step(std::false_type{});
    }

    // combine the four waves' (max, sum, O) through their own buffers (as few_bf16.hip)
    const float l_tot = half_sum(l_run);
    if (hh == 0) {
      Ms[w][c] = m2;
      Ls[w][c] = l_tot;
    }
    __syncthreads();
    float M = -INFINITY, Lt = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) M = fmaxf(M, Ms[i][c]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float mi = Ms[i][c];
      Lt += Ls[i][c] * (mi == -INFINITY ? 0.f : fast_exp2(mi - M));
    }
    const bool whole = e.n == e.v;
    float wgt = m2 == -INFINITY ? 0.f : fast_exp2(m2 - M);
    if (whole) wgt *= Lt > 0.f ? 1.f / Lt : 0.f;
    auto area = [&](int wv, int ch) {  // chunk ch (head_dim 4 ch ..) of row 0
      return reinterpret_cast<char*>(ch < 16 ? Kt[wv] : Vt[wv]);
    };
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int ch = db * 8 + a * 2 + hh;
        const f32x4 o4 = {oacc[db][a * 4] * wgt, oacc[db][a * 4 + 1] * wgt,
                          oacc[db][a * 4 + 2] * wgt, oacc[db][a * 4 + 3] * wgt};
        *reinterpret_cast<f32x4*>(area(w, db * 8) + c * 256 + (((ch & 15) ^ (c & 15)) << 4)) = o4;
      }
    if (!whole && e.kb == 0) {
      left_share = true;
      if (tid == 0)
        *share = PagedShare{(int32_t)((e.xs + e.v - 1) / R.per - e.xs / R.per) + 1, e.at, range * 2, 2, e.hk, rows,
                            e.rb * BM, e.q_start};
    }
    if (w == 0 && hh == 0 && c < rows) {
      if (whole)
        p.lse[(e.hk * group + hg) * p.total_q + e.q_start + qi] = Lt > 0.f ? (M + log2f(Lt)) * kLn2 : -INFINITY;
      else p.stat[(int64_t)e.at * BM + c] = make_float2(M, Lt);
    }
    __syncthreads();
    for (int u = tid; u < rows * (D / 4); u += 256) {
      const int r = u / (D / 4), ch = u % (D / 4);
      const int at = r * 256 + (((ch & 15) ^ (r & 15)) << 4);
      f32x4 o4 = *reinterpret_cast<const f32x4*>(area(0, ch) + at);
#pragma unroll
      for (int i = 1; i < 4; ++i) o4 += *reinterpret_cast<const f32x4*>(area(i, ch) + at);
      if (whole) {
        const uint32_t rr = (uint32_t)(e.rb * BM + r);
        const int ri = (int)(rr / (uint32_t)group);
        const int64_t row = ((int64_t)e.q_start + ri) * p.hq + e.hk * group + (int)rr - ri * group;
        *reinterpret_cast<bf16x4*>(static_cast<bf16*>(p.o) + row * D + ch * 4) =
            bf16x4{f2bf(o4[0]), f2bf(o4[1]), f2bf(o4[2]), f2bf(o4[3])};
      } else {
        *reinterpret_cast<f32x4*>(p.part + ((int64_t)e.at * BM + r) * D + ch * 4) = o4;
      }
    }
    __syncthreads();  // the buffers are free
  }
  if (!left_share && tid == 0) share->pieces = 0;
}

// Row blocks of several pieces: O = sum 2^(M_i - M) O_i / L, L = sum 2^(M_i - M) L_i, D/4 lanes per
// row.  kLine: by ranges, otherwise by row blocks.
template <int D, int BM, bool kLine>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedParams p) {
  constexpr int LPR = D / 4;
  if (p.hdr->status != BS_DEV_OK) return;
  if (!kLine && blockIdx.x >= p.hdr->n_items * (unsigned)p.hkv) return;
  const PagedShare s = p.share[blockIdx.x];
  if (s.pieces == 0) return;
  const int row = blockIdx.y * (256 / LPR) + threadIdx.x / LPR, ch = threadIdx.x % LPR;
  if (row >= s.rows) return;
  auto at = [&](int i) { return (int64_t)(i == 0 ? s.first : s.next + i * s.step) * BM + row; };
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

// What a call launches, from its shapes alone, and its workspace: header, shares, statistics and sums
// of the pieces.
struct PagedLayout {
  bool few, line;
  int32_t bm;      // rows of a block
  int32_t grid;    // workgroups
  int32_t parts;   // !line: of a row block
  int32_t shares;  // shares, and so workgroups in x of the merge (0: no merge)
  size_t share, stat, part, bytes;
};
PagedLayout paged_layout(const bs_dims& d, int32_t num_seqs) {
  PagedLayout L = {};
  L.share = L.stat = L.part = L.bytes = sizeof(WsHeader);
  if (d.dtype == BS_F32) return L;
  const int64_t rows = d.total_q * (d.hq / d.hkv);
  const int64_t blocks = num_seqs == 0 ? 0 : rows / kTileBM + (rows < num_seqs ? rows : num_seqs);  // per KV head at most
  int64_t pieces;
  L.few = rows <= kFewBM * (int64_t)num_seqs;
  L.bm = L.few ? kFewBM : kTileBM;
  L.line = num_seqs == 0 || rows <= 2 * kTileBM * (int64_t)num_seqs;
  if (L.line) {
    L.grid = L.shares = kPagedGrid;
    pieces = 2 * kPagedGrid;
  } else {
    const int64_t items = blocks * d.hkv;
    L.parts = items >= kPagedGrid ? 1 : (int32_t)(2 * kPagedGrid / items < 8 ? 2 * kPagedGrid / items : 8);
    L.grid = (int32_t)(items * L.parts);
    L.shares = L.parts > 1 ? (int32_t)items : 0;
    pieces = L.parts > 1 ? items * L.parts : 0;
  }
  if (L.shares == 0) return L;
  L.stat = L.share + align256(sizeof(PagedShare) * (size_t)L.shares);
  L.part = L.stat + align256(sizeof(float2) * L.bm * (size_t)pieces);
  L.bytes = L.part + sizeof(float) * L.bm * (size_t)pieces * d.head_dim;
  return L;
}

}  // namespace

size_t paged_bytes(const bs_dims& d, int32_t num_seqs, int32_t) { return paged_layout(d, num_seqs).bytes; }

hipError_t launch_paged_fwd(const bs_dims& d, const void* q, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, int32_t max_seqlen_k, int causal,
                            float scale, void* out, float* lse, void* ws, hipStream_t stream) {
  const int es = d.dtype == BS_BF16 ? 2 : 4;
  const PagedLayout W = paged_layout(d, num_seqs);
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
  p.parts = W.parts;
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
    const dim3 grid((unsigned)W.grid), mgrid((unsigned)W.shares, (unsigned)(W.bm * d.head_dim / 1024));
#define BS_LAUNCH(D, LINE)                                                                         \
  do {                                                                                             \
    hipLaunchKernelGGL((paged_tile_kernel<D, LINE>), grid, dim3(256), 0, stream, p);               \
    if (W.shares > 0)                                                                              \
      hipLaunchKernelGGL((paged_merge_kernel<D, kTileBM, LINE>), mgrid, dim3(256), 0, stream, p);  \
  } while (0)
#define BS_CALL(D)                                                                                  \
  do {                                                                                              \
    if (W.few) {                                                                                    \
      hipLaunchKernelGGL((paged_few_kernel<D>), grid, dim3(256), 0, stream, p);                     \
      hipLaunchKernelGGL((paged_merge_kernel<D, kFewBM, true>), mgrid, dim3(256), 0, stream, p);    \
    } else if (W.line) {                                                                            \
      BS_LAUNCH(D, true);                                                                           \
    } else {                                                                                        \
      BS_LAUNCH(D, false);                                                                          \
    }                                                                                               \
  } while (0)
    if (d.head_dim == 128) BS_CALL(128); else BS_CALL(64);
#undef BS_CALL
#undef BS_LAUNCH
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((d.total_q * d.hq + 3) / 4 + (d.total_q == 0)));
  if (d.head_dim == 128) hipLaunchKernelGGL((paged_row_kernel<float, 128>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((paged_row_kernel<float, 64>), grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace bs
