// How the work of a paged attention call is shared, as plain functions for host and device.
//
// A segment's rows (lq queries x the `group` heads of a KV head) form blocks of BM; row block i sees
// the first keys(i) keys, in v(i) blocks of BLK, at least one.  All blocks of all row blocks, segments and
// KV heads form one line that is cut into equal ranges, one per workgroup, so that a workgroup's
// range may begin and end inside a row block, whatever the lengths.
//
// With a causal mask v(i) grows with i, and its sum has no closed form because of the rounding.  The
// line therefore gives row block i the slots [S(i), S(i + 1)) of
//   S(i) = floor(i (A + i B)),  A + B (2 i + 1) >= v(i) + 1 / BLK
// a sum of the unrounded counts: S(i + 1) - S(i) >= floor(A + B (2 i + 1)) >= v(i), about one slot
// more than needed on average.  The slots behind the v(i)-th are skipped.  The one row block of a
// short segment has its v exactly.  Where a segment has more queries than keys, its first row blocks see none: they
// have a slot each, and i counts from the first block that may see a key.
#pragma once

#include <stdint.h>

#if defined(__HIP__)
#define BS_HD __host__ __device__ __forceinline__
#else
#define BS_HD inline
#endif

namespace bs {

struct PagedSeg {
  int32_t lq, lk, group, causal;
};

BS_HD int32_t paged_row_blocks(const PagedSeg& s, int BM) {
  return (int32_t)(((int64_t)s.lq * s.group + BM - 1) / BM);
}

// Keys that some row of block i sees, and their blocks.
BS_HD int32_t paged_keys(const PagedSeg& s, int BM, int32_t i) {
  if (!s.causal) return s.lk;
  const uint32_t last = ((uint32_t)(i + 1) * (uint32_t)BM - 1) / (uint32_t)s.group;
  const int32_t q = last < (uint32_t)s.lq ? (int32_t)last : s.lq - 1;
  const int32_t k = s.lk - s.lq + q + 1;  // at most lk
  return k > 0 ? k : 0;
}
BS_HD int32_t paged_blocks(const PagedSeg& s, int BM, int BLK, int32_t i) {
  const int32_t k = paged_keys(s, BM, i);
  return k > BLK ? (k + BLK - 1) / BLK : 1;
}

// The slots of a segment.
struct PagedCost {
  double a, b;
  int32_t n, none;  // row blocks, and how many of them, the first, are known to see no key
  // (a product of one rounding, so that every caller gets the same number)
  BS_HD int32_t start(int32_t i) const {
    const int32_t j = i - none;
    return j <= 0 ? i : none + (int32_t)(j * __builtin_fma((double)j, b, a));
  }
  // The row block that slot y of the segment belongs to.
  BS_HD int32_t find(int32_t y) const {
    if (n == 1) return 0;
    if (y < none) return y;
    double g = b > 0 ? (__builtin_sqrt(a * a + 4 * b * (double)(y - none)) - a) / (2 * b) : (double)y / a;
    int32_t i = none + g < n ? none + (int32_t)g : n - 1;
    while (i > none && start(i) > y) --i;
    while (i + 1 < n && start(i + 1) <= y) ++i;
    return i;
  }
};
BS_HD PagedCost paged_cost(const PagedSeg& s, int BM, int BLK) {
  PagedCost c;
  c.n = paged_row_blocks(s, BM);
  c.none = 0;
  c.b = 0;
  c.a = s.lk > BLK ? (s.lk + BLK - 1) / BLK : 1;
  if (s.causal && c.n > 1) {
    const double step = (double)BM / s.group / BLK;
    int32_t first = s.lk - s.lq + 1;  // keys of the first query
    if (first < 1) {
      c.none = (int32_t)((int64_t)(s.lq - s.lk) * s.group / BM);
      first = 1;  // (of the query that sees one, and not before row block `none`)
    }
    c.b = step * 0.5;
    c.a = (double)(first + BLK) / BLK + c.b;
  }
  return c;
}

// Slots of sequences of so many rows and at most so many keys each, at most: S(n) is n times at most
// lk / BLK + 1 + 1 / BLK + 3 B, and B <= 1 (128 rows of as many queries, 64 keys).
BS_HD int64_t paged_places(int64_t rows, int64_t seqs, int64_t keys, int BM, int BLK) {
  return (rows / BM + seqs) * (keys / BLK + 5);
}

// Workgroups that run at a time (two per CU), the ranges of a line at most, and parts of a row block's keys at most.
constexpr int32_t kPagedSlots = 512, kPagedMaxParts = 64;

// The n <= kPagedSlots ranges of a line of `all` places, as equal as can be.  A line has less than 2^31 places per KV
// head and less than 2^39 in all: the entry point refuses more.
struct PagedRanges {
  int64_t all;
  int32_t n;
  BS_HD explicit PagedRanges(int64_t places) : all(places), n(places < kPagedSlots ? (int32_t)places : kPagedSlots) {}
  BS_HD int64_t start(int32_t w) const { return n == kPagedSlots ? w * all / kPagedSlots : w; }  // (a shift)
  // The range that place x lies in (a float quotient is off by one at most).
  BS_HD int32_t of(int64_t x) const {
    int32_t w = (int32_t)((float)(x + 1) * (float)n / (float)all);
    if (w > n - 1) w = n - 1;
    while (start(w) > x) --w;
    while (start(w + 1) <= x) ++w;
    return w;
  }
};
// Floor of x / line, below 2^12.
BS_HD int32_t paged_head(int64_t x, int32_t line) {
  int32_t h = (int32_t)((float)x / (float)line);
  while (h * (int64_t)line > x) --h;
  while ((h + 1) * (int64_t)line <= x) ++h;
  return h;
}
// Into how many parts the keys of n < kPagedSlots row blocks are cut, n times that at most 2 kPagedSlots: the
// smallest estimate, in microseconds, of
//   chain x rounds of workgroups / parts  +  3 for the merge's launch, 0.2 for each of a row block's parts, which it
//   reads one after another, and `piece` for each part's sums,
// the rounds between the whole number that equal chains take and what uneven ones, the longest first, take on
// average; a workgroup that has its CU to itself takes two thirds of the time.  chain: time of the longest.  Measured,
// us: one sequence of 512 new tokens over 14K, 64/8 heads (256 row blocks): 2 parts 166, 4 parts 177; 700 over 9K,
// 48/8 (264): 1 part 160, 3 parts 134; 900 over 1K, 64/8 (450): 1 part 65, 2 parts 83; 128 over 16K, 64/8 (64): 4
// parts 57, 8 parts 55; 300 over 60K, 8/2 (20): 8 parts 86, 45 63; a prompt of 700, 16/4 (88): 1 part 22, 2 parts 25.
BS_HD float paged_part_cost(int32_t n, int32_t p, float chain, float piece) {
  if (p > 1 && n * p > 2 * kPagedSlots) return 1e30f;
  const float x = (float)(n * p) / kPagedSlots + 0.4f, even = x > 1.f ? x : 1.f;
  const float whole = (float)((n * p + kPagedSlots - 1) / kPagedSlots);
  const float rate = n * p <= kPagedSlots / 2 ? 0.66f : 1.f;
  return chain * rate * (0.7f * whole + 0.3f * even) / (float)p + (p > 1 ? 3.f + 0.2f * (float)p + piece * (float)(n * p) : 0.f);
}
BS_HD int32_t paged_parts(int32_t n, float chain, float piece) {
  int32_t best = 1;
  float least = paged_part_cost(n, 1, chain, piece);
  for (int32_t p = 2; p <= kPagedMaxParts && n * p <= 2 * kPagedSlots; ++p) {
    const float cost = paged_part_cost(n, p, chain, piece);
    if (cost < least) {
      least = cost;
      best = p;
    }
  }
  return best;
}

// Range, of n, of block b of the grid: blocks are dealt to the 8 XCDs in turn, and each XCD takes neighbouring
// ranges, which read the same keys.  -1: none.
BS_HD int32_t paged_range_of(int32_t b, int32_t n) {
  const int32_t each = (n + 7) >> 3, at = b >> 3, w = (b & 7) * each + at;
  return at < each && w < n ? w : -1;
}

}  // namespace bs
