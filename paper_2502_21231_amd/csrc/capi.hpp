// What the C ABI's sources (capi.hip, capi_qkv.hip) share: error messages, argument checks, profiling.
#pragma once

#include "common.hpp"

namespace bs {

// Sets the thread's message and returns `code` / clears it and returns BS_OK.
int fail(int code, const char* fmt, ...);
int ok();
int hip_fail(hipError_t e, const char* what);

constexpr int64_t kMaxTokens = int64_t(1) << 30;
// query heads: keeps the byte offsets inside one tile of rows below 2^31
constexpr int32_t kMaxHeads = 4096;

int check_dims(const bs_dims* d, bool need_kv);
int check_ptr(const void* p, int64_t count, const char* name);
int check_scale(float s);

// Records an event pair around the launches made during its lifetime (none when an event
// cannot be had: the one that was is returned to the pool).
class ProfScope {
 public:
  ProfScope(int kind, hipStream_t s);
  ~ProfScope();

 private:
  int kind_;
  hipStream_t s_;
  hipEvent_t a_ = nullptr, b_ = nullptr;
};

// True when the byte ranges [a, a + na) and [b, b + nb) intersect.
inline bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

#define BS_TRY(x)                 \
  do {                            \
    int rc__ = (x);               \
    if (rc__ != BS_OK) return rc__; \
  } while (0)
#define BS_HIP(x, what)                        \
  do {                                         \
    hipError_t e__ = (x);                      \
    if (e__ != hipSuccess) return hip_fail(e__, what); \
  } while (0)

}  // namespace bs
