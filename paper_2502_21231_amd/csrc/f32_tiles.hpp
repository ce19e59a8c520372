// float32 tiles in LDS as operands of v_mfma_f32_32x32x2_f32, for the float32 attention kernels (the layout is
// described in f32.hip).
#pragma once

#include "common.hpp"

namespace bs {

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x16 mfma2(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// Copy instructions K .. N-1 of a run of N <= 4 (1 KB of LDS each, 256 / D rows).
template <int K, int N, int D>
struct CopyRun {
  static __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, float* lds, int row0,
                                               int sub, int phys, int gstride, int last) {
    constexpr int RPI = 256 / D;
    const int row = row0 + K * RPI + sub;
    const int r = row < last ? row : last;
    const int voff = (r * gstride + ((phys ^ (row & 15)) << 2)) * 4 + 4096 - K * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds, 16,
                                             voff, 0, K * 1024, 0);
    if constexpr (K + 1 < N) CopyRun<K + 1, N, D>::issue(rs, lds, row0, sub, phys, gstride, last);
  }
};

// One wave's share of copying rows 0..R-1 (row r from src + min(r, last) * gstride) into a
// swizzled [R][D] float tile, without staging registers; waited for with wait_vmem_all().
// The buffer starts 4 KB before `src` so that the offsets, which subtract the instruction
// offset, are not negative (only src + row offsets are accessed); R rows x gstride x 4 bytes
// stay below 2^31 for the head counts the C API accepts.
template <int D, int R, int NW>
__device__ __forceinline__ void copy_rows(float* tile, const float* src, int gstride, int last,
                                          int wave, int lane) {
  constexpr int RPI = 256 / D, PER = R / RPI / NW, CPR = D / 4;
  static_assert(PER >= 4 && PER % 4 == 0, "runs of four copy instructions");
  const int sub = lane / CPR, phys = lane % CPR;
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(reinterpret_cast<const char*>(src) - 4096), 0, 0x7fffffff, 0x00020000);
#pragma unroll
  for (int u = 0; u < PER; u += 4) {
    const int u0 = wave * PER + u;
    CopyRun<0, 4, D>::issue(rsrc, tile + u0 * 256, u0 * RPI, sub, phys, gstride, last);
  }
}

// Lane bases (bytes) of the two reads inside a 32-row block of a tile, and the reads.
template <int D>
__device__ __forceinline__ int row_base(int lane) {
  const int c = lane & 31, hh = lane >> 5;
  return c * D * 4 + ((hh ^ (c & 15)) << 4);
}
template <int D>
__device__ __forceinline__ f32x4 row_read(const char* block, int base, int kk) {
  return *reinterpret_cast<const f32x4*>(block + (base ^ (kk << 5)));
}
template <int D>
__device__ __forceinline__ int col_base(int lane) {
  const int c = lane & 31, hh = lane >> 5;
  if constexpr (D == 128) return hh * 4 * D * 4 + ((c ^ (hh * 4)) << 4);
  else return hh * 4 * D * 4 + (((c >> 1) ^ (hh * 4)) << 4) + (c & 1) * 8;
}
template <int D>
__device__ __forceinline__ void col_read(const char* block, int base, int r, float (&x)[D / 32]) {
  const char* p = block + (base ^ ((((r >> 2) & 1) * 8 + (r & 3)) << 4)) +
                  ((r >> 2) * 8 + (r & 3)) * D * 4;
  if constexpr (D == 128) {
    const f32x4 y = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = y[i];
  } else {
    const f32x2 y = *reinterpret_cast<const f32x2*>(p);
    x[0] = y[0];
    x[1] = y[1];
  }
}

// acc += A^T B over the 32 rows of `block`: B (P or dS) in registers, A's columns from LDS.
template <int D>
__device__ __forceinline__ void col_products(const char* block, int cbase, const f32x16& b,
                                             f32x16 (&acc)[D / 32]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float a[D / 32];
    col_read<D>(block, cbase, r, a);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = mfma2(a[db], b[r], acc[db]);
  }
}

// A wave's [32 lanes][D] accumulators (lane c = one query or key) into LDS as swizzled rows.
template <int D>
__device__ __forceinline__ void put_acc(char* block, int lane, const f32x16 (&acc)[D / 32]) {
  const int c = lane & 31, hh = lane >> 5;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int i = (r >> 2) * 8 + hh * 4 + (r & 3);
    char* row = block + c * D * 4;
    if constexpr (D == 128)
      *reinterpret_cast<f32x4*>(row + ((i ^ (c & 15)) << 4)) =
          f32x4{acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
    else
      *reinterpret_cast<f32x2*>(row + (((i >> 1) ^ (c & 15)) << 4) + (i & 1) * 8) =
          f32x2{acc[0][r], acc[1][r]};
  }
}
// Chunk ch (head_dim 4 ch ..) of row c of such a block.
template <int D>
__device__ __forceinline__ f32x4 get_chunk(const char* block, int c, int ch) {
  return *reinterpret_cast<const f32x4*>(block + c * D * 4 + ((ch ^ (c & 15)) << 4));
}

// Lane's row of a [*, heads, D] tensor as product operands: elements 8 kk + 4 hh .. + 3.
template <int D>
__device__ __forceinline__ void load_frag(f32x4 (&f)[D / 8], const float* row, int hh) {
#pragma unroll
  for (int kk = 0; kk < D / 8; ++kk)
    f[kk] = *reinterpret_cast<const f32x4*>(row + kk * 8 + hh * 4);
}
template <int D>
__device__ __forceinline__ f32x16 row_products(const char* block, int rbase, const f32x4 (&f)[D / 8]) {
  f32x16 s = f32x16{};
#pragma unroll
  for (int kk = 0; kk < D / 8; ++kk) {
    const f32x4 a = row_read<D>(block, rbase, kk);
#pragma unroll
    for (int e = 0; e < 4; ++e) s = mfma2(a[e], f[kk][e], s);
  }
  return s;
}

}  // namespace bs
