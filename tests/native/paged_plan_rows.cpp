// The line of a paged attention call (csrc/paged_plan.hpp) where sequences have more new tokens than keys, so that
// their first rows see none: the slots of a segment are within the bound that the host accepts a call by, every row
// block has room for its blocks of keys, and is found from its slots.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

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
  const int64_t bound = paged_places((int64_t)s.lq * s.group, 1, s.lk, BM, BLK);
  if (bound >= INT32_MAX) return;  // (no line)
  const PagedCost c = paged_cost(s, BM, BLK);
  CHECK(c.n == paged_row_blocks(s, BM) && c.start(0) == 0);
  const double most = c.n == 1 ? c.start(1) : (c.n - c.none) * (c.a + c.b * (c.n - c.none)) + c.none;
  CHECK(most <= (double)bound);
  int64_t at = 0;
  for (int32_t i = 0; i < c.n; ++i) {
    const int32_t v = paged_blocks(s, BM, BLK, i);
    const int64_t next = c.start(i + 1);
    CHECK(c.start(i) == at && next - at >= v);
    CHECK(!s.causal || paged_keys(s, BM, i) > 0 || next - at <= 5);
    if (i < 300 || i > c.n - 300 || i % 97 == 0) CHECK(c.find((int32_t)at) == i && c.find((int32_t)next - 1) == i);
    at = next;
  }
  CHECK(at <= bound);
}

int main() {
  const int tiles[][2] = {{128, 64}, {32, 128}, {32, 256}};
  for (const int* t : tiles)
    for (int causal = 0; causal < 2; ++causal) {
      // the largest that a call of 16,384 sequences takes as a line
      for (int lk : {0, 1, 31, 63, 64, 127, 2000, 65536}) segment(PagedSeg{1 << 22, lk, 1, causal}, t[0], t[1]);
      for (int lq : {1, 31, 32, 33, 127, 128, 129, 130, 1000, 4096, 100001})
        for (int group : {1, 2, 3, 7, 8, 33, 128, 4096})
          for (int less : {-1000, -129, -1, 0, 1, 2, 31, 32, 33, 63, 64, 127, 128, 129, 500, 4000, 100000})
            if (lq - less >= 0 && (int64_t)lq * group < 3000000) segment(PagedSeg{lq, lq - less, group, causal}, t[0], t[1]);
    }
  std::puts("ok");
}
