// Attention of new tokens over a paged key/value cache (gfx950).
//
// Rows of a matrix product's block are (query, head of the KV group) pairs, row qi * group + hg, so
// that a group's heads share the keys they read, for one query of many heads as for many queries of
// one.  A workgroup of four waves takes one of two forms for a block of rows:
//   few   32 rows; the waves take 32 (bf16, head_dim 64: 64) keys in turn, each with LDS buffers, page
//         numbers and a softmax of its own, joined at the end: bound by reading the keys, no barrier
//         between copies (the layout of few_bf16.hip).  Sequences of up to 32 rows; in float32, on that
//         type's matrix instruction, longer ones too where there are not enough for tiles;
//   tile  128 rows over tiles of 64 keys (float32: 32) that the waves share, 32 rows each: bound by the
//         matrix core (the layout of fwd_bf16.hip).
// Both side by side in one launch, so that a step of decoding and prompt chunks uses memory and matrix
// core at once.  How the work is shared:
//   line  the blocks of all sequences form one line cut into equal ranges (paged_plan.hpp): decoding,
//         where row blocks are few and their lengths differ;
//   items where sequences have many rows, or few keys: a workgroup per block of rows, or per part of its
//         keys when there are too few; those of a sequence and head run next to one another on one XCD
//         and walk the same keys in step, which then come into its L2 once.
// A block of rows that several workgroups share leaves (O, max, sum) of each part in float32, and
// paged_merge_kernel combines them.  Every workgroup lays out the line from the lengths itself: only
// shapes are known on the host, so a captured call can be replayed with other lengths.
//
// Measured: 32 single queries over up to 8K keys, 64/8 heads of 128, bf16: 80 us, 5.4 TB/s (the merge 4 of it), float32,
// 32/8: 173 us, 5.3 TB/s; 256 over up to 4K, 32/8, bf16: 302 us, 6.0 TB/s; one over 3K, 32/8: 12 us, two launches that
// leave the chip empty.  8 chunks of up to 1,024 queries over up to 16K keys, 64/8: 1.53 to 1.60 ms, 1,000 to 1,040
// TFLOP/s of visible pairs, within 4 % of the contiguous forward.  A chunk of 509 among 16 single queries over 8K, 48/8:
// 93 us, of which the keys' bytes alone are 56.  float32, 3 x up to 200 queries over 700, 8/4 heads of 64: 18 us, a chain
// of key blocks and a merge.
//
// Pages.  A wave copies 16 neighbouring keys at a time, which lie in one page (page_size is a multiple
// of 16), so a page's place is scalar work, one number of the table per 16 keys, read a tile ahead.
// Keys behind the sequence's end repeat its last one, as in fwd_bf16.hip; 16 keys of which none exists,
// or whose page is not there, are copied from a row of zeros: the probability of a hidden key is 0, but
// 0 times what the cache may hold there need not be.
#include <type_traits>

#include "attn.hpp"
#include "f32_tiles.hpp"
#include "paged_plan.hpp"
#include "qkv.hpp"

namespace bs {
namespace {

// A row of keys that are not there (never written).
__device__ __attribute__((aligned(256))) uint32_t g_zero_row[128];

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
  int32_t parts;      // items: whether row blocks may be shared (> 1)
  int32_t bm;         // rows of a piece's room in stat and part
  int64_t total_q;
  int32_t num_seqs, page_shift, max_len;  // max_len: no more than the table holds
  int32_t hq, hkv, group;
  int32_t causal;
  float scale_log2;
};

constexpr int kTileBM = 128, kTileBN = 64, kTileBN32 = 32, kFewBM = 32;
constexpr int kShortKeys = 1024, kFewWhole = 8;

// Time of a key with its row block, two workgroups on a CU, us (at head_dim 128 and 64: a tile of 64 keys 2.1 and 1.2;
// 128 keys in float32 5.8 and 4.6), and of a part's sums, written and read at 4 TB/s.
__host__ __device__ constexpr float key_us(bool bf, int d) {
  return bf ? (d == 128 ? 0.033f : 0.018f) : (d == 128 ? 0.045f : 0.036f);
}
__host__ __device__ constexpr float piece_us(bool bf, int d) { return (bf ? kTileBM : kFewBM) * d * 2e-6f; }

// How the work of a call is shared: a line, or items in the tile or in the few form.
enum Mode { kLine = 0, kTileItems = 1, kFewItems = 2 };

template <typename T, int D>
constexpr int few_keys() { return sizeof(T) == 2 && D == 64 ? 64 : 32; }  // of a wave's tile

// Block of rows and block of keys of a segment of so many rows per KV head.  (Both blocks of keys, 128 or 256 for
// few rows and 64 for a tile, take a workgroup about as long: weights of 3 : 2 and 2 : 3 were within 5 % and on
// average slower.)
struct Shape {
  int bm, blk;
};
template <typename T, int D, int kMode>
__device__ __forceinline__ Shape shape_of(const PagedSeg& s) {
  if (kMode == kFewItems || (sizeof(T) == 4 ? kMode != kTileItems : (int64_t)s.lq * s.group <= kFewBM))
    return Shape{kFewBM, 4 * few_keys<T, D>()};
  return Shape{kTileBM, sizeof(T) == 4 ? kTileBN32 : kTileBN};
}

// What a workgroup knows of the segments: thread t takes segments t * n .. of n = ceil(num_seqs / 256), or with n = 1
// the t-th in the order of the walk.
struct PagedLds {
  int32_t pre[257];  // places on the line before each thread's segments, per KV head
  int32_t sum[4];
  int32_t bad;
  __attribute__((aligned(16))) int32_t seg[256], q0[256], lq[256], lk[256];  // n = 1: the segment, its first query and lengths
};

__device__ __forceinline__ int32_t seqs_per_thread(int32_t n) { return (n + 255) >> 8; }

__device__ __forceinline__ PagedSeg paged_seg(const PagedParams& p, int32_t b) {
  return PagedSeg{p.cu_q[b + 1] - p.cu_q[b], p.kv_lens[b], p.group, p.causal};
}

// Inclusive sum over the lanes of a wave (moves inside rows of 16 lanes, then from row to row, as operands of the
// additions).
template <int kCtrl, int kRows>
__device__ __forceinline__ int32_t lane_move(int32_t x) {
  return __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xf, true);
}
__device__ __forceinline__ int32_t wave_scan(int32_t x) {
  x += lane_move<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
  x += lane_move<0x112, 0xf>(x);
  x += lane_move<0x114, 0xf>(x);
  x += lane_move<0x118, 0xf>(x);
  x += lane_move<0x142, 0xa>(x);  // the last lane of row 0 to row 1, of row 2 to row 3
  x += lane_move<0x143, 0xc>(x);  // lane 31 to rows 2 and 3
  return x;
}

// Places of a segment on the line, or its blocks of rows.
template <typename T, int D, int kMode>
__device__ __forceinline__ int32_t segment_cost(const PagedSeg& s) {
  const Shape f = shape_of<T, D, kMode>(s);
  if constexpr (kMode != kLine) return paged_row_blocks(s, f.bm);
  const PagedCost c = paged_cost(s, f.bm, f.blk);
  return c.start(c.n);
}

// Lays out the line (256 threads); the places per KV head, negative when the lengths are refused.  Block 0
// writes the header.
template <typename T, int D, int kMode>
__device__ __forceinline__ int32_t paged_line(const PagedParams& p, PagedLds& L) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int32_t pt = seqs_per_thread(p.num_seqs);
  if (tid == 0) L.bad = BS_DEV_OK;
  int32_t code = BS_DEV_OK;
  if (tid == 0) {
    const int32_t first = p.cu_q[0], end = p.cu_q[p.num_seqs];
    code = first != 0 ? BS_DEV_BAD_FIRST : end > p.total_q ? BS_DEV_BAD_TOTAL : BS_DEV_OK;
  }
  // the lengths of segment b, which are checked (refused ones count as empty)
  auto check = [&](int32_t b, int32_t& q0) {
    q0 = p.cu_q[b];
    const int64_t n = (int64_t)p.cu_q[b + 1] - q0;
    const int32_t len = p.kv_lens[b];
    int32_t c = BS_DEV_OK;
    if (n < 0 || len < 0) c = BS_DEV_NOT_MONOTONE;
    else if (len > p.max_len) c = BS_DEV_TOO_LONG;
    else if (n > p.total_q) c = BS_DEV_BAD_TOTAL;
    if (code == BS_DEV_OK) code = c;
    return c == BS_DEV_OK ? PagedSeg{(int32_t)n, len, p.group, p.causal} : PagedSeg{0, 0, p.group, p.causal};
  };
  int32_t sum = 0;
  auto count = [&](const PagedSeg& s) {
    if (s.lq > 0) sum += segment_cost<T, D, kMode>(s);
  };
  if (pt > 1) {
    for (int32_t b = tid * pt; b < min(tid * pt + pt, p.num_seqs); ++b) {
      int32_t q0;
      count(check(b, q0));
    }
  } else {
    int32_t q0 = 0, at = tid;
    PagedSeg s = PagedSeg{0, -1, p.group, p.causal};
    if (tid < p.num_seqs) s = check(tid, q0);
    constexpr bool kRanked = kMode == kTileItems || (kMode == kFewItems && sizeof(T) == 4);
    if constexpr (kRanked) {
      // the longest chains first, so that the last workgroups to start are short ones
      L.lk[tid] = s.lk;
      __syncthreads();
      at = 0;
      const int4* all = reinterpret_cast<const int4*>(L.lk);
#pragma unroll 4
      for (int i = 0; i < p.num_seqs; i += 4) {  // (entries past num_seqs are -1)
        const int4 k = all[i >> 2];
        at += k.x > s.lk || (k.x == s.lk && i < tid);
        at += k.y > s.lk || (k.y == s.lk && i + 1 < tid);
        at += k.z > s.lk || (k.z == s.lk && i + 2 < tid);
        at += k.w > s.lk || (k.w == s.lk && i + 3 < tid);
      }
      if (tid >= p.num_seqs) at = tid;
      __syncthreads();
    }
    L.seg[at] = tid;
    L.q0[at] = q0;
    L.lq[at] = s.lq;
    L.lk[at] = s.lk;
    if constexpr (kRanked) __syncthreads();
    count(PagedSeg{L.lq[tid], L.lk[tid], p.group, p.causal});
  }
  const int32_t run = wave_scan(sum);
  if (lane == 63) L.sum[w] = run;
  __syncthreads();
  if (code != BS_DEV_OK) {  // (the first thread's comes first)
    if (tid == 0) L.bad = code;
    else atomicCAS(&L.bad, BS_DEV_OK, code);
  }
  int32_t at = run - sum;
  for (int i = 0; i < w; ++i) at += L.sum[i];
  L.pre[tid] = at;
  if (tid == 255) L.pre[256] = at + sum;
  __syncthreads();
  const int32_t bad = L.bad, all = __builtin_amdgcn_readfirstlane(L.pre[256]);
  if (blockIdx.x == 0 && tid == 0) {
    p.hdr->status = bad;
    p.hdr->n_items = kMode != kLine && bad == BS_DEV_OK ? all : 0;  // row blocks per KV head
  }
  return bad == BS_DEV_OK ? all : -1;
}

// The segment that holds place y of the line, and the places before it.  The same in every lane.
struct Found {
  int32_t seg, q_start, lq, lk, before;
};
template <typename T, int D, int kMode>
__device__ __forceinline__ Found find_segment(const PagedParams& p, const PagedLds& L, int32_t y) {
  const int lane = threadIdx.x & 63;
  int t = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) t += __popcll(__ballot(L.pre[i * 64 + lane] <= y));
  const int32_t pt = seqs_per_thread(p.num_seqs);
  Found f;
  if (pt <= 1) {
    f = Found{L.seg[t], L.q0[t], L.lq[t], L.lk[t], L.pre[t]};
  } else {  // (at most 64 segments per thread)
    const int32_t mine = t * pt + lane;
    int32_t cost = 0;
    if (lane < pt && mine < p.num_seqs) {
      const PagedSeg s = paged_seg(p, mine);
      if (s.lq > 0) cost = segment_cost<T, D, kMode>(s);
    }
    const int32_t at = L.pre[t] + wave_scan(cost) - cost;
    const int k = __ffsll((unsigned long long)__ballot(cost > 0 && at <= y && y - at < cost)) - 1;
    const int32_t b = t * pt + k;
    f = Found{b, p.cu_q[b], p.cu_q[b + 1] - p.cu_q[b], p.kv_lens[b], __builtin_amdgcn_readlane(at, k)};
  }
  f.seg = __builtin_amdgcn_readfirstlane(f.seg);
  f.q_start = __builtin_amdgcn_readfirstlane(f.q_start);
  f.lq = __builtin_amdgcn_readfirstlane(f.lq);
  f.lk = __builtin_amdgcn_readfirstlane(f.lk);
  f.before = __builtin_amdgcn_readfirstlane(f.before);
  return f;
}

// A part of a block of rows.  All of it is the same in every lane.
struct Piece {
  int32_t hk, seg, q_start, lq, lk;
  int32_t rb, rows;  // block of rows, and how many it has
  int32_t kb, n, v;  // key blocks [kb, kb + n) of v
  int32_t at;        // its place among the pieces, where the row block is shared
  int32_t pieces;    // of the row block
};

// Line: the piece that starts at place x (n <= 0: none); next: where the next row block starts.
template <typename T, int D>
__device__ __forceinline__ Piece line_piece(const PagedParams& p, const PagedLds& L, int32_t line,
                                            const PagedRanges& R, int64_t x, int64_t x_end, int32_t range, Shape& f,
                                            int64_t& next) {
  Piece c;
  c.hk = __builtin_amdgcn_readfirstlane(paged_head(x, line));
  const int32_t y = (int32_t)(x - c.hk * (int64_t)line);
  const Found s = find_segment<T, D, kLine>(p, L, y);
  c.seg = s.seg;
  c.q_start = s.q_start;
  c.lq = s.lq;
  c.lk = s.lk;
  const PagedSeg g = PagedSeg{s.lq, s.lk, p.group, p.causal};
  f = shape_of<T, D, kLine>(g);
  if (s.lq * p.group <= f.bm) {  // one row block: its places are its blocks
    c.rb = 0;
    c.kb = y - s.before;
    c.v = paged_blocks(g, f.bm, f.blk, 0);
    next = x + c.v - c.kb;
  } else {
    const PagedCost k = paged_cost(g, f.bm, f.blk);
    c.rb = __builtin_amdgcn_readfirstlane(k.find(y - s.before));
    c.kb = __builtin_amdgcn_readfirstlane(y - s.before - k.start(c.rb));
    next = x + __builtin_amdgcn_readfirstlane(s.before + k.start(c.rb + 1) - y);
    c.v = __builtin_amdgcn_readfirstlane(paged_blocks(g, f.bm, f.blk, c.rb));
  }
  c.n = (int32_t)min((int64_t)(c.v - c.kb), x_end - x);
  c.rows = min((int)(c.lq * p.group - c.rb * f.bm), f.bm);
  // (the number of pieces is wanted where the row block starts only)
  c.pieces = c.n == c.v ? 1 : c.kb > 0 ? 2 : __builtin_amdgcn_readfirstlane(R.of(x + c.v - 1)) - range + 1;
  // a range has at most one piece that goes on from the range before (place 0 of its two) and one that
  // another range goes on with (place 1)
  c.at = range * 2 + (c.kb == 0);
  return c;
}

// paged_parts, one number of parts per lane (one after another they take 5 us).
__device__ __forceinline__ int32_t best_parts(int32_t n, float chain, float piece) {
  static_assert(kPagedMaxParts <= 64, "a lane for each");
  const int32_t lane = threadIdx.x & 63;
  const float mine = lane < kPagedMaxParts ? paged_part_cost(n, lane + 1, chain, piece) : 1e30f;
  float least = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) least = fminf(least, __shfl_xor(least, off));
  return __ffsll((unsigned long long)__ballot(mine == least));
}

// The piece of workgroup b: a part of a row block, the row blocks of one segment and head side by side on one
// XCD (b % 8), the longest first; line: row blocks per KV head.  false: none.
template <typename T, int D, int kMode>
__device__ __forceinline__ bool item_piece(const PagedParams& p, const PagedLds& L, int32_t line, int32_t b,
                                           int32_t max_parts, Piece& c) {
  const bool own = (p.hkv & 7) == 0;  // each XCD owns an eighth of the heads
  const int32_t hx = own ? p.hkv >> 3 : p.hkv, j = own ? b >> 3 : b;
  const int32_t i = j / (hx * max_parts);  // a row block's place, if all heads took turns
  if (i >= line) return false;
  const Found g = find_segment<T, D, kMode>(p, L, i);
  c.seg = g.seg;
  c.q_start = g.q_start;
  c.lq = g.lq;
  c.lk = g.lk;
  const PagedSeg s = PagedSeg{g.lq, g.lk, p.group, p.causal};
  const Shape f = shape_of<T, D, kMode>(s);
  const int32_t nrb = paged_row_blocks(s, f.bm);
  const int32_t r = j - g.before * hx * max_parts;  // of the segment's nrb * hx * parts
  int32_t hl, u;  // head; row block and part
  if (own) {
    hl = r / (nrb * max_parts);
    u = r - hl * nrb * max_parts;
  } else {
    u = r / hx;
    hl = r - u * hx;
  }
  const int32_t back = u / max_parts, part = u - back * max_parts;
  c.hk = __builtin_amdgcn_readfirstlane(own ? (b & 7) * hx + hl : hl);
  c.rb = __builtin_amdgcn_readfirstlane(nrb - 1 - back);
  c.v = __builtin_amdgcn_readfirstlane(paged_blocks(s, f.bm, f.blk, c.rb));
  c.rows = min((int)(c.lq * p.group - c.rb * f.bm), f.bm);
  c.pieces = min(max_parts, c.v);  // (a part may be one block; with four at least 3 x 200 over 700, float32, took 31 us for 21)
  if (part >= c.pieces) return false;
  c.kb = __builtin_amdgcn_readfirstlane(part * c.v / c.pieces);
  c.n = __builtin_amdgcn_readfirstlane((part + 1) * c.v / c.pieces) - c.kb;
  // pieces and shares are numbered by head and row block
  c.at = __builtin_amdgcn_readfirstlane((c.hk * line + g.before + c.rb) * max_parts + part);
  return true;
}

// One wave's copy of 16 rows (row r from src + min(r, last) * stride bytes) into 16 rows of a swizzled
// tile, as dma_tile (bf16) and copy_rows (float32) copy them.
template <int D, int AUX>
__device__ __forceinline__ void copy16(bf16* lds, const char* src, int stride, int last, int lane) {
  constexpr int CPR = D / 8, PER = 16 / (64 / CPR);
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)(src - 4096), 0, 0x7fffffff, 0x00020000);
  DmaRun<0, PER, D, AUX>::issue(rs, lds, 0, lane / CPR, lane % CPR, stride >> 1, last);
}
template <int D, int AUX>
__device__ __forceinline__ void copy16(float* lds, const char* src, int stride, int last, int lane) {
  constexpr int RPI = 256 / D, CPR = D / 4;
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)(src - 4096), 0, 0x7fffffff, 0x00020000);
#pragma unroll
  for (int r0 = 0; r0 < 16; r0 += 4 * RPI)
    CopyRun<0, 4, D>::issue(rs, lds + r0 * D, r0, lane / CPR, lane % CPR, stride >> 2, last);
}

// Waits until at most N of this wave's copies are under way; until its LDS reads have returned (few_bf16.hip).
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);  // vmcnt(N)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ void store_o(bf16* p, f32x4 x) {
  *reinterpret_cast<bf16x4*>(p) = bf16x4{f2bf(x[0]), f2bf(x[1]), f2bf(x[2]), f2bf(x[3])};
}
__device__ __forceinline__ void store_o(float* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }

// A row of the group's rows of a segment: its query, and place of (query, head) among all.
struct Row {
  int qi, head;
  int64_t at;
};
__device__ __forceinline__ Row row_of(const PagedParams& p, const Piece& e, uint32_t r) {
  Row x;
  x.qi = (int)(r / (uint32_t)p.group);
  x.head = e.hk * p.group + (int)r - x.qi * p.group;
  x.at = ((int64_t)e.q_start + x.qi) * p.hq + x.head;
  return x;
}
// (a NaN among the scores is one in the sum; -inf says that no key is seen)
__device__ __forceinline__ float lse_of(float m2, float l) { return l == 0.f ? -INFINITY : (m2 + log2f(l)) * kLn2; }
// Keys that the row's query sees.
__device__ __forceinline__ int seen_by(const PagedParams& p, const Piece& e, int qi) {
  return p.causal ? min(e.lk, qi + e.lk - e.lq + 1) : e.lk;
}

constexpr float kRescaleBy = 8.0f;  // log2 units (fwd_bf16.hip)

// A lane's sum of weights, of which there may be millions of nearly one size: added one after another to a sum far above
// them, all would be rounded the same way (131,072 keys 3 to 7 below a first one, in one chain: LSE off by 8.5e-4; so by
// 1.9e-6).  A tile's weights make four sums, which are one addition, whose rounding the next one takes back.
struct WeightSum {
  float sum = 0.f, over = 0.f;  // over: what the last addition was rounded up by
  float tile[4];
  // weight i of a tile, in order
  __device__ __forceinline__ void take(int i, float w) {
    if (i == 0) tile[0] = w - over;
    else if (i < 4) tile[i] = w;
    else tile[i & 3] += w;
  }
  __device__ __forceinline__ void finish() {
    const float x = (tile[0] + tile[1]) + (tile[2] + tile[3]), s = sum + x;
    over = (s - sum) - x;
    sum = s;
  }
  __device__ __forceinline__ void scale(float by) {
    sum *= by;
    over *= by;
  }
};

// The thread's number, which the compiler does not know to be the same for every piece: what depends on it is
// worked out in each (held over the loop of pieces, 46 registers of the line kernel spill).
__device__ __forceinline__ int own_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// LDS of a workgroup: two arrays X and Y, so that the compiler can tell copies into one from reads of the other.
// Tile form: X and Y are the two buffers, K then V in each; few form: X holds the waves' K, Y their V.
template <typename T, int D, int kMode>
constexpr int buf_elems() { return sizeof(T) == 2 ? 128 * 128 : kMode == kTileItems ? 2 * kTileBN32 * D : 128 * D; }
struct FewLds {
  float m[4][32], l[4][32];
};
struct TileLds {
  __attribute__((aligned(16))) int32_t miss[2][4];  // per buffer and 16 keys: the page is not there
};

// Tile form of bf16.
template <int D>
__device__ __forceinline__ void tile_piece(const PagedParams& p, const Piece& e, bf16 (&X)[128 * 128],
                                           bf16 (&Y)[128 * 128], TileLds& S) {
  constexpr int BM = kTileBM, BN = kTileBN, TILE = BN * D, KK = D / 16, DB = D / 32;
  const int tid = own_thread();
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
  const float c2 = p.scale_log2;
  const int tstride = (int)p.token_stride;
  const int rbase = swz_row_base<D>(lane), tbase = swz_tr_base<D>(lane);
  const int qrow = w * 32 + c;
  const bool qvalid = qrow < e.rows;
  const uint32_t r_lane = (uint32_t)(e.rb * BM + (qvalid ? qrow : 0));
  bf16x8 qf[KK];
  int lim_base;  // keys below it are visible to this lane's query (less the lane half's offset)
  {
    const Row r = row_of(p, e, r_lane);
    lim_base = seen_by(p, e, r.qi) - hh * 4;
    const bf16* qp = static_cast<const bf16*>(p.q) + r.at * D + hh * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);
  }
  const int full = seen_by(p, e, (int)((uint32_t)(e.rb * BM) / (uint32_t)p.group));
  const int n_full = __builtin_amdgcn_readfirstlane(full > 0 ? full / BN : 0);  // tiles that all rows see whole
  const int t0 = e.kb, n_tiles = e.kb + e.n, keys = e.lk;

  const int32_t* table = p.table + e.seg * p.table_stride;
  const int64_t hoff = e.hk * p.head_stride;
  // page of this wave's 16 keys of tile t (-1: behind the end of the sequence, which has a key)
  auto page_of = [&](int t) {
    const int key = t * BN + w * 16, page = table[min(key, keys - 1) >> p.page_shift];
    return key < keys ? page : -1;
  };
  auto copy = [&](int t, int page, bf16* Kd, bf16* Vd, int32_t* miss) {
    const int key = t * BN + w * 16;
    page = __builtin_amdgcn_readfirstlane(page);
    const bool there = page >= 0 && page < p.num_pages;
    const int64_t off = page * p.page_stride + (int64_t)(key & ((1 << p.page_shift) - 1)) * tstride + hoff;
    const char* ks = there ? p.kc + off : reinterpret_cast<const char*>(g_zero_row);
    const char* vs = there ? p.vc + off : reinterpret_cast<const char*>(g_zero_row);
    const int stride = there ? tstride : 0, last = min(15, keys - 1 - key);
    copy16<D, 0>(Kd + w * 16 * D, ks, stride, last < 0 ? 0 : last, lane);
    copy16<D, 0>(Vd + w * 16 * D, vs, stride, last < 0 ? 0 : last, lane);
    if (lane == 0) miss[w] = !there && key < keys;
  };

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m2 = -INFINITY;
  WeightSum l_run;

  copy(t0, keys > 0 ? page_of(t0) : -1, X, X + TILE, S.miss[0]);
  int page = e.n > 1 ? page_of(t0 + 1) : -1;
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
      l_run.scale(alpha);
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
    }
    const float base = m2 == -INFINITY ? 0.f : m2;
    // P rounded to bf16 for the product, as in the contiguous forward (the sum takes it in float32): a second product for
    // what the rounding loses, as the few form has it, takes 37 % more (8 chunks of up to 1,024 queries over up to 16K keys,
    // 64/8 heads 1,547 -> 2,111 us) for a relative error of 2.3e-3 -> 1.66e-3, of which the result's own rounding is 1.65e-3
    bf16x8 pb[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float ex = fast_exp2(fmaf(sacc[kb][r], c2, -base));
        l_run.take(kb * 16 + r, ex);
        pb[kb * 2 + (r >> 3)][r & 7] = f2bf(ex);
      }
    }
    l_run.finish();
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
  if (w * 32 >= e.rows) {  // a wave without rows copies its keys, and leaves the matrix core to the others
    for (int t = t0; t < n_tiles; ++t) {
      if (t + 1 < n_tiles) {
        const int odd = (t + 1 - t0) & 1;
        bf16* Z = odd ? Y : X;
        copy(t + 1, page, Z, Z + TILE, S.miss[odd]);
        page = page_of(t + 2);
      }
      wait_vmem_all();
      __syncthreads();
    }
    return;
  }
  int t = t0;
  for (; t + 2 < n_tiles; t += 2) {
    step(std::true_type{}, t, X, X + TILE, S.miss[0], Y, Y + TILE, S.miss[1]);
    step(std::true_type{}, t + 1, Y, Y + TILE, S.miss[1], X, X + TILE, S.miss[0]);
  }
  const bool two = t + 2 == n_tiles;
  if (two) step(std::true_type{}, t, X, X + TILE, S.miss[0], Y, Y + TILE, S.miss[1]);
  const bf16* Z = two ? Y : X;
  step(std::false_type{}, n_tiles - 1, Z, Z + TILE, S.miss[two], nullptr, nullptr, nullptr);

  const float l_tot = half_sum(l_run.sum);
  if (!qvalid) return;
  uint32_t r1 = r_lane;
  asm volatile("" : "+v"(r1));  // the row's place is worked out again: held over the loop, registers spill
  const Row r = row_of(p, e, r1);
  if (e.pieces == 1) {
    const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
    bf16* op = static_cast<bf16*>(p.o) + r.at * D + hh * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *reinterpret_cast<bf16x4*>(op + db * 32 + a * 8) =
            bf16x4{f2bf(oacc[db][a * 4 + 0] * inv), f2bf(oacc[db][a * 4 + 1] * inv),
                   f2bf(oacc[db][a * 4 + 2] * inv), f2bf(oacc[db][a * 4 + 3] * inv)};
    if (hh == 0) p.lse[r.head * p.total_q + e.q_start + r.qi] = lse_of(m2, l_tot);
    return;
  }
  const int64_t at = (int64_t)e.at * p.bm + qrow;
  float* op = p.part + at * D + hh * 4;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      *reinterpret_cast<f32x4*>(op + db * 32 + a * 8) =
          f32x4{oacc[db][a * 4 + 0], oacc[db][a * 4 + 1], oacc[db][a * 4 + 2], oacc[db][a * 4 + 3]};
  if (hh == 0) p.stat[at] = make_float2(m2, l_tot);
}

// The types of the few form.  A wave's block of rows in LDS, for the sum over the waves: row r's chunk
// ch of 16 bytes; bf16 keeps 64 columns in the K and 64 in the V buffer, float32 all in the K buffer.
template <typename T, int D>
struct FewOps;
template <int D>
struct FewOps<bf16, D> {
  static constexpr int KT = few_keys<bf16, D>(), KB = KT / 32, KK = D / 16, DB = D / 32, COPIES = 8;
  typedef bf16x8 Q;
  static constexpr int NQ = KK;
  const int rbase, tbase;
  __device__ __forceinline__ FewOps(int lane) : rbase(swz_row_base<D>(lane)), tbase(swz_tr_base<D>(lane)) {}
  static __device__ __forceinline__ void load(Q (&q)[NQ], const bf16* row, int hh) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = *reinterpret_cast<const bf16x8*>(row + hh * 8 + kk * 16);
  }
  __device__ __forceinline__ void scores(const bf16* K, const Q (&q)[NQ], f32x16 (&s)[KB]) const {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) s[kb] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const bf16x8 a = lds_row16(K, (rbase ^ (kk << 5)) + kb * 64 * D);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[kk], s[kb], 0, 0, 0);
      }
  }
  // P as two bf16 numbers, what the first loses by its rounding being the second: within 2^-17 of float32.  The few form
  // waits for keys, so the second product costs little (32 single queries over up to 8K keys, 64/8 heads 78.3 -> 79.1 us;
  // 256 over up to 4K, 32/8 300 -> 304; head_dim 64, 32 over 8K 51.1 -> 52.3), and the result's own rounding is all that
  // is left of bf16 (relative error of those 32 2.1e-3 -> 1.65e-3).
  struct P {
    bf16x8 x[2 * KB], y[2 * KB];
  };
  static __device__ __forceinline__ void put(P& p, int kb, int r, float v) {
    const bf16 x = f2bf(v);
    p.x[kb * 2 + (r >> 3)][r & 7] = x;
    p.y[kb * 2 + (r >> 3)][r & 7] = f2bf(v - bf2f(x));
  }
  __device__ __forceinline__ void values(const bf16* V, const P& p, f32x16 (&o)[DB]) const {
#pragma unroll
    for (int ks = 0; ks < 2 * KB; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 a = lds_tr16(V, (tbase ^ (db << 6)) + ks * 32 * D, (tbase ^ ((db << 6) | 32)) + ks * 32 * D + 16 * D);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p.x[ks], o[db], 0, 0, 0);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p.y[ks], o[db], 0, 0, 0);
      }
  }
  static __device__ __forceinline__ void put_rows(bf16* K, bf16* V, int lane, const f32x16 (&o)[DB]) {
    const int c = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int ch = db * 8 + a * 2 + hh;
        *reinterpret_cast<f32x4*>(reinterpret_cast<char*>(db < 2 ? K : V) + c * 256 + (((ch & 15) ^ (c & 15)) << 4)) =
            f32x4{o[db][a * 4], o[db][a * 4 + 1], o[db][a * 4 + 2], o[db][a * 4 + 3]};
      }
  }
  static __device__ __forceinline__ f32x4 get(const bf16* K, const bf16* V, int r, int ch) {
    return *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(ch < 16 ? K : V) + r * 256 +
                                           (((ch & 15) ^ (r & 15)) << 4));
  }
};
template <int D>
struct FewOps<float, D> {
  static constexpr int KT = 32, KB = 1, DB = D / 32, COPIES = D / 8;
  typedef f32x4 Q;
  static constexpr int NQ = D / 8;
  const int rbase, cbase;
  __device__ __forceinline__ FewOps(int lane) : rbase(row_base<D>(lane)), cbase(col_base<D>(lane)) {}
  static __device__ __forceinline__ void load(Q (&q)[NQ], const float* row, int hh) { load_frag<D>(q, row, hh); }
  __device__ __forceinline__ void scores(const float* K, const Q (&q)[NQ], f32x16 (&s)[1]) const {
    s[0] = row_products<D>(reinterpret_cast<const char*>(K), rbase, q);
  }
  struct P {
    f32x16 x;
  };
  static __device__ __forceinline__ void put(P& p, int, int r, float v) { p.x[r] = v; }
  __device__ __forceinline__ void values(const float* V, const P& p, f32x16 (&o)[DB]) const {
    // a tile's products have sums of their own, which are one addition to O's: two keys a step would be as many roundings
    // as keys / 2, all one way over values of one size (131,072 keys of one value, in one chain: 1.9e-3 of O; so 6e-5, for
    // 1 to 4 % of the time of prompts, one of 4,096, 32/8 heads 1.12 -> 1.14 ms, 64 x up to 60, head_dim 64, 49 -> 51 us)
    f32x16 t[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) t[db] = f32x16{};
    col_products<D>(reinterpret_cast<const char*>(V), cbase, p.x, t);
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] += t[db];
  }
  static __device__ __forceinline__ void put_rows(float* K, float*, int lane, const f32x16 (&o)[DB]) {
    put_acc<D>(reinterpret_cast<char*>(K), lane, o);
  }
  static __device__ __forceinline__ f32x4 get(const float* K, const float*, int r, int ch) {
    return get_chunk<D>(reinterpret_cast<const char*>(K), r, ch);
  }
};

// Tile form of float32: tiles of 32 keys, of which two waves copy K and two V, 16 keys each.  Half the LDS of the few
// form, so that two workgroups share a CU at head_dim 128 too, and no sum over waves at the end.
template <int D>
__device__ __forceinline__ void tile_piece(const PagedParams& p, const Piece& e, float (&X)[2 * kTileBN32 * D],
                                           float (&Y)[2 * kTileBN32 * D], TileLds& S) {
  typedef FewOps<float, D> Ops;
  constexpr int BM = kTileBM, BN = kTileBN32, TILE = BN * D, DB = D / 32;
  const int tid = own_thread();
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
  const float c2 = p.scale_log2;
  const int tstride = (int)p.token_stride;
  const Ops ops(lane);
  const int qrow = w * 32 + c;
  const bool qvalid = qrow < e.rows;
  const uint32_t r_lane = (uint32_t)(e.rb * BM + (qvalid ? qrow : 0));
  typename Ops::Q qf[Ops::NQ];
  int lim_base;
  {
    const Row r = row_of(p, e, r_lane);
    Ops::load(qf, static_cast<const float*>(p.q) + r.at * D, hh);
    lim_base = seen_by(p, e, r.qi) - hh * 4;
  }
  const int full = seen_by(p, e, (int)((uint32_t)(e.rb * BM) / (uint32_t)p.group));
  const int n_full = __builtin_amdgcn_readfirstlane(full > 0 ? full / BN : 0);  // tiles that all rows see whole
  const int t0 = e.kb, n_tiles = e.kb + e.n, keys = e.lk;

  const int32_t* table = p.table + e.seg * p.table_stride;
  const int64_t hoff = e.hk * p.head_stride;
  const int half = w & 1;
  const char* cache = w < 2 ? p.kc : p.vc;
  auto page_of = [&](int t) {
    const int key = t * BN + half * 16, page = table[min(key, keys - 1) >> p.page_shift];
    return key < keys ? page : -1;
  };
  auto copy = [&](int t, int page, float* buf, int32_t* miss) {
    const int key = t * BN + half * 16;
    page = __builtin_amdgcn_readfirstlane(page);
    const bool there = page >= 0 && page < p.num_pages;
    const int64_t off = page * p.page_stride + (int64_t)(key & ((1 << p.page_shift) - 1)) * tstride + hoff;
    const char* src = there ? cache + off : reinterpret_cast<const char*>(g_zero_row);
    const int last = min(15, keys - 1 - key);
    copy16<D, 0>(buf + (w >> 1) * TILE + half * 16 * D, src, there ? tstride : 0, last < 0 ? 0 : last, lane);
    if (w < 2 && lane == 0) miss[half] = !there && key < keys;
  };

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m2 = -INFINITY;
  WeightSum l_run;
  copy(t0, keys > 0 ? page_of(t0) : -1, X, S.miss[0]);
  int page = e.n > 1 ? page_of(t0 + 1) : -1;
  wait_vmem_all();
  __syncthreads();

  const bool idle = w * 32 >= e.rows;  // a wave without rows copies only
  auto step = [&](int t, const float* B, const int32_t* miss, float* Bn, int32_t* miss_n) {
    if (t + 1 < n_tiles) {
      copy(t + 1, page, Bn, miss_n);
      page = page_of(t + 2);
    }
    if (!idle) {
      f32x16 s[1];
      ops.scores(B, qf, s);
      if (t >= n_full) {
        const int lim = lim_base - t * BN;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[0][r] = ((r >> 2) * 8 + (r & 3)) < lim ? s[0][r] : -INFINITY;
      }
      if (__builtin_amdgcn_readfirstlane(miss[0] | miss[1])) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[0][r] = miss[r >> 3] ? -INFINITY : s[0][r];
      }
      float mx = s[0][0];
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[0][r]);
      mx = half_max(mx) * c2;
      if (__any(mx > m2)) {
        const float m_new = fmaxf(m2, mx);
        const float alpha = fast_exp2(m2 - (m_new == -INFINITY ? 0.f : m_new));
        m2 = m_new;
        l_run.scale(alpha);
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      }
      const float base = m2 == -INFINITY ? 0.f : m2;
      typename Ops::P pr;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float ex = fast_exp2(fmaf(s[0][r], c2, -base));
        l_run.take(r, ex);
        Ops::put(pr, 0, r, ex);
      }
      l_run.finish();
      ops.values(B + TILE, pr, oacc);
    }
    wait_vmem_all();
    __syncthreads();
  };
  for (int t = t0; t < n_tiles; t += 2) {
    step(t, X, S.miss[0], Y, S.miss[1]);
    if (t + 1 < n_tiles) step(t + 1, Y, S.miss[1], X, S.miss[0]);
  }

  // (whole row blocks only: a call of this form has enough of them)
  const float l_tot = half_sum(l_run.sum);
  if (!qvalid) return;
  const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  uint32_t r1 = r_lane;
  asm volatile("" : "+v"(r1));  // worked out again, as in the form of bf16
  const Row row = row_of(p, e, r1);
  float* op = static_cast<float*>(p.o) + row.at * D;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int i = (r >> 2) * 8 + hh * 4 + (r & 3);  // acc[.][r]: elements DB i ..
    if constexpr (D == 128) {
      *reinterpret_cast<f32x4*>(op + i * 4) = f32x4{oacc[0][r], oacc[1][r], oacc[2][r], oacc[3][r]} * inv;
    } else if (r % 2 == 0) {
      *reinterpret_cast<f32x4*>(op + i * 2) = f32x4{oacc[0][r], oacc[1][r], oacc[0][r + 1], oacc[1][r + 1]} * inv;
    }
  }
  if (hh == 0) p.lse[row.head * p.total_q + e.q_start + row.qi] = lse_of(m2, l_tot);
}

// Few form.  kAux: cache policy of the copies (2: non-temporal).
template <typename T, int D, int kAux, int N>
__device__ __forceinline__ void few_piece(const PagedParams& p, const Piece& e, T (&X)[N], T (&Y)[N], FewLds& S) {
  typedef FewOps<T, D> Ops;
  constexpr int BM = kFewBM, KT = Ops::KT, BLK = 4 * KT, NC = KT / 16, KB = Ops::KB, DB = Ops::DB;
  static_assert(4 * KT * D <= N, "four waves' tiles per array");
  const int tid = own_thread();
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
  const float c2 = p.scale_log2;
  const int tstride = (int)p.token_stride;
  const Ops ops(lane);
  T* Kw = X + w * KT * D;
  T* Vw = Y + w * KT * D;
  const Row row = row_of(p, e, (uint32_t)(e.rb * BM + min(c, e.rows - 1)));
  typename Ops::Q qf[Ops::NQ];
  Ops::load(qf, static_cast<const T*>(p.q) + row.at * D, hh);
  const int keys = e.lk;
  const int lim_lane = seen_by(p, e, row.qi) - hh * 4;
  // keys that all rows see; keys some row sees, and this piece's end
  const int full = __builtin_amdgcn_readfirstlane(seen_by(p, e, (int)((uint32_t)(e.rb * BM) / (uint32_t)p.group)));
  int k_end = seen_by(p, e, (int)((uint32_t)(e.rb * BM + e.rows - 1) / (uint32_t)p.group));
  if (e.kb + e.n < e.v) k_end = min(k_end, (e.kb + e.n) * BLK);

  const int32_t* table = p.table + e.seg * p.table_stride;
  const int64_t hoff = e.hk * p.head_stride;
  // lane i < NC: page of keys 16 i .. of the tile at k0 (-1: behind the sequence's end)
  auto pages_of = [&](int k0) {
    const int key = k0 + lane * 16, page = table[min(key, keys - 1) >> p.page_shift];
    return key < keys ? page : -1;
  };
  // what a tile's copies need: place of each 16 keys, which are there, which are missing
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
  auto copy = [&](T* dst, const char* cache, const Place& a, int k0) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const bool there = (a.there >> i) & 1;
      const char* src = there ? cache + a.off[i] : reinterpret_cast<const char*>(g_zero_row);
      const int last = min(15, keys - 1 - k0 - i * 16);
      copy16<D, kAux>(dst + i * 16 * D, src, there ? tstride : 0, last < 0 ? 0 : last, lane);
    }
  };

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m2 = -INFINITY;
  WeightSum l_run;

  int k0 = (e.kb * 4 + w) * KT;
  Place now;
  int ahead = -1;  // pages of the next tile
  // one tile; `more`: another follows (straight-line forms, so that the copies under way can be counted)
  auto step = [&](auto more) {
    wait_copies<Ops::COPIES>();  // K has landed (V's copies may be under way)
    f32x16 s[KB];
    ops.scores(Kw, qf, s);
    const int next = k0 + BLK, miss = now.miss;
    wait_reads();
    if constexpr (more()) {
      now = place_of(ahead, next);
      ahead = pages_of(next + BLK);
      copy(Kw, p.kc, now, next);
    }
    if (k0 + KT > full) {
      const int lim = lim_lane - k0;
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
      l_run.scale(alpha);
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
    }
    const float base = m2 == -INFINITY ? 0.f : m2;
    typename Ops::P pr;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float ex = fast_exp2(fmaf(s[kb][r], c2, -base));
        l_run.take(kb * 16 + r, ex);
        Ops::put(pr, kb, r, ex);
      }
    l_run.finish();
    // V has landed.  (K's copies and the pages' load come after it; where the load is moved, waiting for
    // one operation more than needed is all that happens.)
    wait_copies<more() ? Ops::COPIES : 0>();
    ops.values(Vw, pr, oacc);
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
    for (int i = 0; i < Ops::NQ; ++i) asm volatile("" : "+v"(qf[i]));
    while (k0 + BLK < k_end) step(std::true_type{});
    step(std::false_type{});
  }

  // the four waves' (max, sum, O), through their own buffers
  const float l_tot = half_sum(l_run.sum);
  if (hh == 0) {
    S.m[w][c] = m2;
    S.l[w][c] = l_tot;
  }
  __syncthreads();
  float M = -INFINITY, Lt = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) M = fmaxf(M, S.m[i][c]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float mi = S.m[i][c];
    Lt += S.l[i][c] * (mi == -INFINITY ? 0.f : fast_exp2(mi - M));
  }
  const bool whole = e.pieces == 1;
  float wgt = m2 == -INFINITY ? 0.f : fast_exp2(m2 - M);
  if (whole) wgt *= Lt > 0.f ? 1.f / Lt : 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] *= wgt;
  Ops::put_rows(Kw, Vw, lane, oacc);
  if (w == 0 && hh == 0 && c < e.rows) {
    if (whole) p.lse[row.head * p.total_q + e.q_start + row.qi] = lse_of(M, Lt);
    else p.stat[(int64_t)e.at * p.bm + c] = make_float2(M, Lt);
  }
  __syncthreads();
  for (int u = tid; u < e.rows * (D / 4); u += 256) {
    const int r = u / (D / 4), ch = u % (D / 4);
    f32x4 o4 = Ops::get(X, Y, r, ch);
#pragma unroll
    for (int i = 1; i < 4; ++i) o4 += Ops::get(X + i * KT * D, Y + i * KT * D, r, ch);
    if (whole) store_o(static_cast<T*>(p.o) + row_of(p, e, (uint32_t)(e.rb * BM + r)).at * D + ch * 4, o4);
    else *reinterpret_cast<f32x4*>(p.part + ((int64_t)e.at * p.bm + r) * D + ch * 4) = o4;
  }
  __syncthreads();  // the buffers are free
}

template <typename T, int D, int kMode>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_kernel(const PagedParams p) {
  constexpr int N = buf_elems<T, D, kMode>();
  __shared__ __attribute__((aligned(16))) T X[N];
  __shared__ __attribute__((aligned(16))) T Y[N];
  __shared__ PagedLds L;
  __shared__ FewLds F;
  __shared__ TileLds S;

  const int32_t line = paged_line<T, D, kMode>(p, L);
  if (line < 0) {  // nothing is written
    if (kMode == kLine && threadIdx.x == 0) p.share[blockIdx.x].pieces = 0;
    return;
  }
  // non-temporal copies where a sequence's keys are read once
  auto few = [&](const Piece& e) {
    if constexpr (sizeof(T) == 2 || kMode != kTileItems) few_piece<T, D, sizeof(T) == 2 ? 2 : 0>(p, e, X, Y, F);
  };
  if constexpr (kMode != kLine) {
    Piece e;
    int32_t parts = 1;
    if (p.parts > 1) {
      const int32_t keys = p.num_seqs <= 256 ? L.lk[0] : p.max_len;  // (the longest comes first)
      parts = __builtin_amdgcn_readfirstlane(best_parts(line * p.hkv, (float)keys * key_us(sizeof(T) == 2, D), piece_us(sizeof(T) == 2, D)));
    }
    if (!item_piece<T, D, kMode>(p, L, line, blockIdx.x, parts, e)) return;
    if (p.parts > 1 && e.kb == 0 && threadIdx.x == 0)
      p.share[e.at / parts] = PagedShare{e.pieces > 1 ? e.pieces : 0, e.at, e.at, 1, e.hk, e.rows,
                                           e.rb * (kMode == kFewItems ? kFewBM : kTileBM), e.q_start};
    if (kMode == kFewItems || (sizeof(T) == 2 && e.lq * p.group <= kFewBM)) {
      few(e);
    } else {
      if constexpr (kMode != kFewItems) tile_piece<D>(p, e, X, Y, S);
    }
  } else {
    PagedShare* share = p.share + blockIdx.x;
    const PagedRanges R((int64_t)line * p.hkv);
    const int32_t range = paged_range_of(blockIdx.x, R.n);
    bool left_share = false;
    if (range >= 0) {
      int64_t x = R.start(range);
      const int64_t x_end = R.start(range + 1);
      while (x < x_end) {
        Shape f;
        int64_t next;
        const Piece e = line_piece<T, D>(p, L, line, R, x, x_end, range, f, next);
        x = e.kb + e.n >= e.v || e.n <= 0 ? next : x_end;
        if (e.n <= 0) continue;
        if (e.pieces > 1 && e.kb == 0) {
          left_share = true;
          if (threadIdx.x == 0)
            *share = PagedShare{e.pieces, e.at, range * 2, 2, e.hk, e.rows, e.rb * f.bm, e.q_start};
        }
        if constexpr (sizeof(T) == 2) {
          if (f.bm != kFewBM) {
            tile_piece<D>(p, e, X, Y, S);
            continue;
          }
        }
        few(e);
      }
    }
    if (!left_share && threadIdx.x == 0) share->pieces = 0;
  }
}

// Row blocks of several pieces: O = sum 2^(M_i - M) O_i / L, L = sum 2^(M_i - M) L_i, by ranges of the line, or by
// row blocks.  D/4 lanes hold a row, as `per` groups that share its pieces where there are many pieces and few rows.
// A launch is a chain of loads (share, maxima, sums): a lane weighs every D/4-th piece of its group, so that no lane
// waits for the pieces one after another, and sums are requested four at a time (eight: 1 us more where row blocks have two or three), the first before the maxima are known.
template <typename T, int D, int kMode>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedParams p) {
  constexpr int LPR = D / 4, G = 256 / LPR, AT_ONCE = 4;
  __shared__ __attribute__((aligned(16))) f32x4 acc[256];
  __shared__ float sums[G];
  const PagedShare s = p.share[blockIdx.x];
  if (kMode != kLine && blockIdx.x >= p.hdr->n_items * (unsigned)p.hkv) return;  // (0 items if lengths are refused)
  if (s.pieces == 0) return;
  const int ch = threadIdx.x % LPR, lane0 = threadIdx.x & 63 & ~(LPR - 1);
  int rows = G;  // at a time
  if (s.pieces > 2 * AT_ONCE)  // (one query over 30K, 16 heads of one group: 47 -> 33 us)
    while (rows > 1 && (rows >> 1) * (int)gridDim.y >= s.rows) rows >>= 1;
  const int per = G / rows, grp = threadIdx.x / LPR / rows, sub = threadIdx.x / LPR % rows;
  for (int r0 = blockIdx.y * rows; r0 < s.rows; r0 += gridDim.y * rows) {
    const int row = min(r0 + sub, s.rows - 1);
    // (2 kPagedSlots pieces of 128 rows: byte offsets of 32 bits, which take half the registers of pointers)
    auto at = [&](int i) { return (uint32_t)(i == 0 ? s.first : s.next + i * s.step) * (uint32_t)p.bm + (uint32_t)row; };
    auto part = [&](int j) {
      const uint32_t off = (at(grp + j * per) * D + ch * 4) * 4u;
      return *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(p.part) + off);
    };
    auto stat = [&](int i) { return *reinterpret_cast<const float2*>(reinterpret_cast<const char*>(p.stat) + at(i) * 8u); };
    const int mine = grp < s.pieces ? (s.pieces - grp + per - 1) / per : 0;  // pieces of this group
    f32x4 x[AT_ONCE];
    auto request = [&](int j0) {
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) x[j] = j0 + j < mine ? part(j0 + j) : f32x4{};
    };
    request(0);
    float M = -INFINITY;
    for (int i = ch; i < s.pieces; i += LPR) M = fmaxf(M, stat(i).x);
#pragma unroll
    for (int off = 1; off < LPR; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
    const float base = M == -INFINITY ? 0.f : M;
    float l = 0.f;
    f32x4 o = f32x4{};
    float wgt = 0.f;  // of piece ch of LPR
    for (int j0 = 0; j0 < mine; j0 += AT_ONCE) {
      if (j0 % LPR == 0) {
        wgt = 0.f;
        if (j0 + ch < mine) {
          const float2 st = stat(grp + (j0 + ch) * per);
          wgt = fast_exp2(st.x - base);
          l += wgt * st.y;
        }
      }
      if (j0 > 0) request(j0);
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) o += __shfl(wgt, lane0 + j0 % LPR + j) * x[j];
    }
#pragma unroll
    for (int off = 1; off < LPR; off <<= 1) l += __shfl_xor(l, off);
    if (per > 1) {  // the groups' sums, in order
      __syncthreads();
      acc[threadIdx.x] = o;
      if (ch == 0) sums[threadIdx.x / LPR] = l;
      __syncthreads();
      if (grp == 0)
        for (int g = 1; g < per; ++g) {
          o += acc[threadIdx.x + g * rows * LPR];
          l += sums[sub + g * rows];
        }
    }
    if (grp > 0 || r0 + sub >= s.rows) continue;
    o *= l > 0.f ? 1.f / l : 0.f;
    const uint32_t r = (uint32_t)(s.row0 + row);
    const int qi = (int)(r / (uint32_t)p.group), head = s.hk * p.group + (int)r - qi * p.group;
    const int64_t tok = (int64_t)s.q_start + qi;
    store_o(static_cast<T*>(p.o) + (tok * p.hq + head) * D + ch * 4, o);
    if (ch == 0) p.lse[head * p.total_q + tok] = lse_of(M, l);
  }
}

// What a call launches, from its shapes alone, and its workspace: header, shares, statistics and sums
// of the pieces.
struct PagedLayout {
  Mode mode;
  int32_t bm;      // rows of a piece's room
  int32_t grid;    // workgroups
  int32_t parts;   // items: of a row block at most
  int32_t shares;  // shares, and so workgroups in x of the merge (0: no merge)
  size_t share, stat, part, bytes;
};
PagedLayout paged_layout(const bs_dims& d, int32_t num_seqs, int32_t max_seqlen_k) {
  PagedLayout L = {};
  L.share = L.stat = L.part = L.bytes = sizeof(WsHeader);
  const int64_t rows = d.total_q * (d.hq / d.hkv), seqs = num_seqs;
  const bool bf = d.dtype == BS_BF16;
  auto blocks = [&](int bm) { return (rows / bm + (rows < seqs ? rows : seqs)) * d.hkv; };  // at most
  const int few_block = 4 * (bf && d.head_dim == 64 ? 64 : 32);
  // Up to 32 rows per sequence on average: where all sequences are short (kFewWhole key blocks), whole row blocks in
  // the few form, since what a workgroup saves by an equal share is less than the merge's launch; the line for decoding
  // (up to two new tokens per sequence on average; in bf16 more are ahead as items, measured in us, line / items: a
  // chunk of 200 and 16 single queries over 3K, 32/32 heads 84 / 73; of 100 and 16 over 2K, 8/2 26 / 16; 6 queries of
  // one sequence over 16K, 32/8 22 / 17; but 16 x 8 over 8K 54 / 56).  More rows: items (a chunk of 500 and 32 single
  // queries over 8K, 64/8 heads 167 / 151; of 900 and 64 over 4K, 32/8 148 / 113; 8 x 30 over 4K, 64/8 44 / 38; but
  // 32 x 30 over 8K 164 / 207, where chains are uneven).  In float32 up to 256 rows per sequence take the line where
  // there are fewer row blocks than workgroups (a chunk of 300 and 32 single queries over 4K, 32/4, head_dim 64: 72 /
  // 104) or keys are many.
  const bool few = rows <= kFewBM * seqs, short_keys = max_seqlen_k <= kFewWhole * few_block;
  const bool line32 = few || (rows <= 2 * kTileBM * seqs && (blocks(kFewBM) < kPagedSlots || max_seqlen_k > kShortKeys));
  if (seqs == 0) L.mode = kLine;
  else if (few && short_keys) L.mode = kFewItems;
  else if (bf) L.mode = few && d.total_q <= 2 * seqs ? kLine : kTileItems;
  else L.mode = line32 ? kLine : kFewItems;
  // Float32 tiles, where those fill the chip.  At head_dim 128 the few form has a CU's LDS to itself, and all it does
  // before and after its products counts: 36 prompts of up to 154 tokens, 32/4 heads 160 -> 76 us, one of 4,096, 32/8
  // 1.27 -> 1.14 ms.  A single query's chain of many keys is four times as long, though (a chunk of 2,000 among 32
  // single queries over 4K, 32/8: 818 us without tiles, 1,015 with).  At head_dim 64 two workgroups of the few form
  // share a CU, and tiles are ahead over few keys only: 36 x 154 73 -> 45 us, 64 x 60 over 200 69 -> 51, but over 500 49 -> 63.
  const bool short_chains = d.head_dim == 64 ? max_seqlen_k <= 256
                                             : max_seqlen_k <= 2048 || rows >= 8 * kTileBM * seqs;
  if (!bf && seqs > 0 && !few && blocks(kTileBM) >= kPagedSlots && short_chains) L.mode = kTileItems;
  L.bm = L.mode == kTileItems || (L.mode == kLine && bf && rows > kFewBM) ? kTileBM : kFewBM;
  int64_t pieces;
  if (L.mode == kLine) {
    L.grid = L.shares = kPagedSlots;
    pieces = 2 * kPagedSlots;
  } else {
    const int64_t n = blocks(L.bm);
    // (where about so many row blocks of the longest chains would not be cut, the merge need not be launched)
    const int64_t about = (rows / L.bm > seqs ? rows / L.bm : rows < seqs ? rows : seqs) * d.hkv;
    const bool whole = n >= kPagedSlots || (few && short_keys) ||
                       paged_parts((int32_t)about, max_seqlen_k * key_us(bf, d.head_dim), piece_us(bf, d.head_dim)) == 1;
    L.parts = whole ? 1 : kPagedMaxParts;
    pieces = n * L.parts < 2 * kPagedSlots ? n * L.parts : 2 * kPagedSlots;  // (what paged_parts keeps to)
    L.grid = L.parts == 1 ? (int32_t)(n > 0 ? n : 1) : (int32_t)pieces;      // (one workgroup checks the lengths)
    L.shares = L.parts > 1 ? (int32_t)n : 0;
    if (L.shares == 0) pieces = 0;
  }
  if (L.shares == 0) return L;
  L.stat = L.share + align256(sizeof(PagedShare) * (size_t)L.shares);
  L.part = L.stat + align256(sizeof(float2) * L.bm * (size_t)pieces);
  L.bytes = L.part + sizeof(float) * L.bm * (size_t)pieces * d.head_dim;
  return L;
}

}  // namespace

size_t paged_bytes(const bs_dims& d, int32_t num_seqs, int32_t max_seqlen_k) {
  return paged_layout(d, num_seqs, max_seqlen_k).bytes;
}

bool paged_fits(const bs_dims& d, int32_t num_seqs, int32_t max_seqlen_k, int64_t keys) {
  const PagedLayout L = paged_layout(d, num_seqs, max_seqlen_k);
  if (L.mode != kLine) return L.grid < (1 << 24);  // (a grid has less than 2^32 threads)
  const int64_t rows = d.total_q * (d.hq / d.hkv);
  const int64_t places = d.dtype == BS_BF16 ? paged_places(rows, num_seqs, keys, kTileBM, kTileBN)
                                            : paged_places(rows, num_seqs, keys, kFewBM, 4 * few_keys<float, 64>());
  return places < INT32_MAX && places * d.hkv < int64_t(1) << 39;
}

hipError_t launch_paged_fwd(const bs_dims& d, const void* q, const bs_paged_cache& C,
                            const int32_t* cu_q, int32_t num_seqs, int32_t max_seqlen_k, int causal,
                            float scale, void* out, float* lse, void* ws, hipStream_t stream) {
  const int es = d.dtype == BS_BF16 ? 2 : 4;
  const PagedLayout W = paged_layout(d, num_seqs, max_seqlen_k);
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
  p.bm = W.bm;
  p.total_q = d.total_q;
  p.num_seqs = num_seqs;
  p.page_shift = __builtin_ctz((unsigned)C.page_size);
  const int64_t room = (int64_t)C.max_pages * C.page_size;
  p.max_len = (int32_t)(max_seqlen_k < room ? max_seqlen_k : room);
  p.hq = d.hq;
  p.hkv = d.hkv;
  p.group = d.hq / d.hkv;
  p.causal = causal;
  p.scale_log2 = scale * kLog2e;
  // (4 or 16 workgroups share a block of rows in the merge)
  const dim3 grid((unsigned)W.grid), mgrid((unsigned)W.shares, W.bm == kFewBM ? 4 : 16);
#define BS_LAUNCH(T, D, MODE)                                                               \
  do {                                                                                      \
    hipLaunchKernelGGL((paged_kernel<T, D, MODE>), grid, dim3(256), 0, stream, p);          \
    if (W.shares > 0)                                                                       \
      hipLaunchKernelGGL((paged_merge_kernel<T, D, MODE>), mgrid, dim3(256), 0, stream, p); \
  } while (0)
#define BS_CALL(T, D)                                                                                   \
  do {                                                                                                  \
    if (W.mode == kLine) BS_LAUNCH(T, D, kLine);                                                        \
    else if (W.mode == kFewItems) BS_LAUNCH(T, D, kFewItems);                                           \
    else BS_LAUNCH(T, D, kTileItems);                                                                   \
  } while (0)
  if (d.dtype == BS_BF16) {
    if (d.head_dim == 128) BS_CALL(bf16, 128); else BS_CALL(bf16, 64);
  } else {
    if (d.head_dim == 128) BS_CALL(float, 128); else BS_CALL(float, 64);
  }
#undef BS_CALL
#undef BS_LAUNCH
  return hipGetLastError();
}

}  // namespace bs
