// The line of a paged attention call (csrc/paged_plan.hpp), walked on the host: every key block of
// every row block is taken by exactly one range, the ranges of a shared row block follow one another, and
// every row of a block sees no key behind its blocks.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <vector>

#include "../../paper_2502_21231_amd/csrc/paged_plan.hpp"

using namespace bs;

#define CHECK(c)                                                     \
  do {                                                               \
    if (!(c)) {                                                      \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #c);           \
      std::exit(1);                                                  \
    }                                                                \
  } while (0)

static void segment(const PagedSeg& s, int BM, int BLK) {
  if ((double)paged_row_blocks(s, BM) * (s.lk / BLK + 3) >= 2147483648.0) return;  // (no line)
  const PagedCost c = paged_cost(s, BM, BLK);
  CHECK(c.n == paged_row_blocks(s, BM));
  CHECK(c.start(0) == 0);
  int64_t need = 0;
  for (int32_t i = 0; i < c.n; ++i) {
    const int32_t v = paged_blocks(s, BM, BLK, i);
    const int64_t at = c.start(i), room = c.start(i + 1) - at;
    need += v;
    CHECK(v >= 1 && room >= v && room <= v + 2 + (s.lk < s.lq ? s.lq / BLK + 1 : 0) + BM / BLK + 1);
    CHECK(c.find(at) == i && c.find(at + room - 1) == i && c.find(at + room / 2) == i);
    // the keys of the block's last row, by the definition
    const int64_t last = std::min<int64_t>((int64_t)s.lq * s.group, (int64_t)(i + 1) * BM) - 1;
    const int64_t seen = s.causal ? std::min<int64_t>(s.lk, std::max<int64_t>(0, s.lk - s.lq + last / s.group + 1)) : s.lk;
    CHECK(paged_keys(s, BM, i) == seen);
    CHECK((int64_t)v * BLK >= seen && (v == 1 || (int64_t)(v - 1) * BLK < seen));
  }
  if (c.n == 1) CHECK(c.start(1) == need);
}

static void ranges(const PagedRanges& R) {
  CHECK(R.n <= kPagedSlots && (R.n > 0) == (R.all > 0) && R.start(0) == 0 && (R.n == 0 || R.start(R.n) == R.all));
  for (int32_t w = 0; w < R.n; ++w) {
    const int64_t a = R.start(w), b = R.start(w + 1);
    CHECK(b > a && b - a <= R.all / R.n + 1);
    CHECK(R.of(a) == w && R.of(b - 1) == w);
  }
}

// Segments of up to 32 rows take the first shape, others the second.
static void line(const std::vector<PagedSeg>& segs, int hkv) {
  const int bm[2] = {32, 128}, blk[2] = {128, 64};
  auto kind = [&](const PagedSeg& s) { return (int64_t)s.lq * s.group <= 32 ? 0 : 1; };
  int64_t per_head = 0;
  std::vector<int64_t> pre;
  for (const PagedSeg& s : segs) {
    pre.push_back(per_head);
    const int t = kind(s);
    if (s.lq > 0) per_head += paged_cost(s, bm[t], blk[t]).start(paged_row_blocks(s, bm[t]));
  }
  const PagedRanges R(per_head * hkv);
  ranges(R);
  std::vector<int> taken(kPagedSlots, 0);
  for (int32_t b = 0; b < kPagedSlots; ++b) {
    const int32_t w = paged_range_of(b, R.n);
    CHECK(w >= -1 && w < R.n);
    if (w >= 0) CHECK(++taken[w] == 1);
  }
  for (int32_t w = 0; w < R.n; ++w) CHECK(taken[w] == 1);
  std::vector<int> heads_of(R.n, 0), tails_of(R.n, 0);  // pieces that leave sums: one of each at most
  for (int h = 0; h < hkv; ++h)
    for (size_t b = 0; b < segs.size(); ++b) {
      if (segs[b].lq == 0) continue;
      const int t = kind(segs[b]);
      const PagedCost c = paged_cost(segs[b], bm[t], blk[t]);
      for (int32_t i = 0; i < c.n; ++i) {
        const int64_t xs = h * per_head + pre[b] + c.start(i);
        CHECK(c.n > 1 || c.start(1) == paged_blocks(segs[b], bm[t], blk[t], 0));
        const int32_t v = paged_blocks(segs[b], bm[t], blk[t], i), first = R.of(xs), pieces = R.of(xs + v - 1) - first + 1;
        int64_t done = 0;
        for (int32_t k = 0; k < pieces; ++k) {
          const int32_t w = first + k;
          const int64_t lo = std::max(R.start(w), xs), hi = std::min(R.start(w + 1), xs + v);
          CHECK(w < R.n && lo - xs == done && hi > lo);
          done += hi - lo;
          if (pieces > 1) CHECK(++(lo == xs ? heads_of : tails_of)[w] == 1);
        }
        CHECK(done == v);
      }
    }
}

int main() {
  std::mt19937 rng(1);
  auto pick = [&](int64_t lo, int64_t hi) {
    const double x = std::uniform_real_distribution<double>(std::log((double)lo), std::log((double)hi + 1))(rng);
    return (int32_t)std::min<int64_t>(hi, (int64_t)std::exp(x));
  };
  const int tiles[][2] = {{128, 64}, {32, 128}, {32, 256}, {32, 64}};
  for (int n = 0; n < 30000; ++n) {
    const int32_t group = n % 3 == 0 ? 1 << (rng() % 8) : pick(1, n % 5 == 0 ? 4096 : 16);
    PagedSeg s{pick(1, n % 7 == 0 ? 40000 : 700), pick(1, n % 11 == 0 ? 2000000 : 9000) - 1, group, (int32_t)(rng() % 4 != 0)};
    if ((int64_t)s.lq * group > 400000) s.lq = 400000 / group;
    if (s.lq < 1) s.lq = 1;
    const int* t = tiles[n % 4];
    segment(s, t[0], t[1]);
  }
  for (int64_t lk : {0, 1, 63, 64, 65, 128, 1 << 20, (1 << 30) - 1})
    for (int64_t lq : {1, 2, 127, 128, 129, 4096})
      for (int group : {1, 3, 8, 128, 4096})
        for (int causal : {0, 1})
          for (const int* t : tiles) segment(PagedSeg{(int32_t)lq, (int32_t)lk, group, causal}, t[0], t[1]);
  for (int n = 0; n < 3000; ++n) {
    std::vector<PagedSeg> segs(rng() % 20);
    const int32_t group = pick(1, 16), causal = rng() % 4 != 0;
    for (PagedSeg& s : segs) s = PagedSeg{(int32_t)(rng() % 5 ? pick(1, 300) : 0), pick(1, 3000) - 1, group, causal};
    line(segs, 1 + rng() % 9);
  }
  for (int64_t all : {(int64_t)0, (int64_t)1, (int64_t)511, (int64_t)512, (int64_t)513, ((int64_t)1 << 39) - 1})
    for (int n = 0; n < 2000; ++n) {
      const PagedRanges R(all - n * (all >> 12));
      ranges(R);
    }
  for (int n = 0; n < 300000; ++n) {
    const int32_t len = pick(1, (1 << 30)), h = rng() % 4096;
    const int64_t x = h * (int64_t)len + rng() % len;
    CHECK(paged_head(x, len) == h && paged_head(h * (int64_t)len, len) == h && paged_head((h + 1) * (int64_t)len - 1, len) == h);
  }
  for (int32_t n = 0; n < kPagedSlots; ++n) {
    for (float chain : {0.f, 2.f, 100.f, 1e6f}) {
      const int32_t parts = paged_parts(n, chain, 0.033f);
      CHECK(parts >= 1 && parts <= kPagedMaxParts && n * parts <= 2 * kPagedSlots);
    }
  }
  std::puts("ok");
}
