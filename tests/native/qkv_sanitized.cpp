// Host-side argument checks of bs_qkv.h under the address and undefined-behaviour sanitizers: every call
// below fails validation, or has nothing to do, before the library touches a device (the pointers are
// placeholders that are never dereferenced).  Built by tests/test_qkv_sanitized.py with capi_qkv.hip
// instrumented on the host side only.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "../../include/bs_qkv.h"

#define CHECK(cond)                                                                            \
  do {                                                                                         \
    if (!(cond)) {                                                                             \
      std::fprintf(stderr, "line %d: %s (last error: %s)\n", __LINE__, #cond, bs_last_error()); \
      std::exit(1);                                                                            \
    }                                                                                          \
  } while (0)

static char* const AT = reinterpret_cast<char*>((uintptr_t)1 << 40);
static const int64_t G = (int64_t)1 << 32;

static bs_dims dims(int64_t T = 128, int32_t hq = 4, int32_t hkv = 2, int32_t d = 128, int32_t dtype = BS_BF16) {
  return bs_dims{T, 0, hq, hkv, d, dtype};
}
static bs_qk_params params(int32_t rot = 128, float eps = 1e-6f) {
  return bs_qk_params{(const float*)AT, rot, 0, AT, AT, BS_F32, eps};
}
static bs_paged_cache cache() {
  return bs_paged_cache{AT, AT + (1 << 30), 8, 4096, 256, 128, (const int32_t*)AT, 4, 4, 16, (const int32_t*)AT};
}
static int fwd(const bs_dims& d, const bs_qk_params& p, int64_t qs = 512, char* qo = AT + 4 * G) {
  return bs_qk_norm_rope_fwd(&d, &p, AT + 2 * G, qs, AT + 3 * G, 256, (const int64_t*)AT, qo, AT + 5 * G, nullptr);
}
static int paged(const bs_dims& d, const bs_paged_cache& c, int32_t n = 2, int32_t most = 64, float scale = 0.1f,
                 size_t ws = (size_t)1 << 30) {
  return bs_attn_paged_fwd(&d, AT + 2 * G, &c, (const int32_t*)AT, n, most, 1, scale, AT + 4 * G, (float*)AT, AT, ws, nullptr);
}
static int append(const bs_dims& d, const bs_paged_cache& c, char* k = AT + 3 * G) {
  return bs_kv_append(&d, nullptr, &c, (const int32_t*)AT, 2, nullptr, 0, k, 256, AT + 6 * G, 256, nullptr, nullptr);
}

int main() {
  CHECK(fwd(dims(128, 4, 2, 96), params()) == BS_ERR_UNSUPPORTED);
  CHECK(fwd(dims(-5), params()) == BS_ERR_INVALID_ARG);
  CHECK(fwd(dims(), params(136)) == BS_ERR_INVALID_ARG);
  CHECK(fwd(dims(), params(INT32_MIN)) == BS_ERR_INVALID_ARG);
  CHECK(fwd(dims(), params(128, NAN)) == BS_ERR_INVALID_ARG);
  CHECK(fwd(dims(), params(128, INFINITY)) == BS_ERR_INVALID_ARG);
  for (int64_t s : {(int64_t)0, (int64_t)-512, (int64_t)504, INT64_MAX, INT64_MIN, INT64_MAX - 7})
    CHECK(fwd(dims(), params(), s) == BS_ERR_INVALID_ARG);
  CHECK(fwd(dims(), params(), 512, AT + 2 * G + 16) == BS_ERR_INVALID_ARG);
  CHECK(std::strstr(bs_last_error(), "overlaps") != nullptr);
  CHECK(fwd(dims(0), params()) == BS_OK);
  CHECK(bs_qk_norm_rope_fwd(nullptr, nullptr, nullptr, 0, nullptr, 0, nullptr, nullptr, nullptr, nullptr) == BS_ERR_INVALID_ARG);
  CHECK(bs_qk_norm_rope_workspace_size(nullptr) == 0);

  for (int64_t v : {(int64_t)0, (int64_t)-1, INT64_MAX, INT64_MIN}) {
    bs_paged_cache c = cache();
    c.num_pages = v;
    CHECK(paged(dims(), c) == BS_ERR_INVALID_ARG);
    c = cache();
    c.page_stride = v;
    CHECK(paged(dims(), c) != BS_OK && append(dims(), c) != BS_OK);
    c = cache();
    c.token_stride = v;
    CHECK(paged(dims(), c) != BS_OK && append(dims(), c) != BS_OK);
    c = cache();
    c.head_stride = v;
    CHECK(paged(dims(), c) != BS_OK && append(dims(), c) != BS_OK);
    c = cache();
    c.table_stride = v;
    CHECK(paged(dims(), c) == BS_ERR_INVALID_ARG);
  }
  bs_paged_cache big = cache();  // the largest strides that are not refused by themselves
  big.num_pages = INT32_MAX;
  big.page_stride = INT64_MAX / 64 / INT32_MAX / 8 * 8;
  big.head_stride = INT64_MAX / 64 / 4096 / 8 * 8;
  CHECK(paged(dims(), big) == BS_ERR_INVALID_ARG && std::strstr(bs_last_error(), "overlaps") != nullptr);
  for (int32_t s : {0, 1, 15, 17, 8192, INT32_MAX, INT32_MIN}) {
    bs_paged_cache c = cache();
    c.page_size = s;
    CHECK(paged(dims(), c) == BS_ERR_UNSUPPORTED);
  }
  CHECK(append(dims(), cache(), nullptr) == BS_ERR_INVALID_ARG);
  CHECK(append(dims(), cache(), AT + 4096) == BS_ERR_INVALID_ARG);
  CHECK(append(dims(0), cache()) == BS_OK);
  CHECK(paged(dims(), cache(), INT32_MAX) == BS_ERR_UNSUPPORTED);
  CHECK(paged(dims(), cache(), 2, INT32_MAX) == BS_ERR_INVALID_ARG);
  CHECK(paged(dims(), cache(), 2, 64, NAN) == BS_ERR_INVALID_ARG);
  CHECK(paged(dims(), cache(), 2, 64, 0.1f, 0) == BS_ERR_WORKSPACE);
  CHECK(paged(dims((1 << 30) - 1, 4096, 4096), cache()) == BS_ERR_UNSUPPORTED);
  // sizes at their limits: no overflow on the way to a workspace size
  for (int64_t T : {(int64_t)0, (int64_t)1, (int64_t)1 << 19, ((int64_t)1 << 30) - 1})
    for (int32_t hq : {1, 4096})
      for (int32_t n : {0, 1, 16384})
        for (int32_t most : {0, 1, (1 << 30) - 1})
          for (int32_t dt : {(int32_t)BS_F32, (int32_t)BS_BF16}) {
            const bs_dims d = dims(T, hq, hq, 64, dt);
            const size_t b = bs_attn_paged_workspace_size(&d, n, most);
            CHECK(b > 0 ? b < (size_t)1 << 32 : T * hq > INT32_MAX);
          }
  std::puts("ok");
  return 0;
}
