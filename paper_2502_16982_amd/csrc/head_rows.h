// Rows of hidden states and weights as the head's kernels read and write them (device code).
#pragma once
#include <hip/hip_runtime.h>

#include "head_gemm.h"

namespace muon {
namespace head {

// Global memory takes 16 (8) bytes at any address of an element.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

struct Row8 {
  float v[8];
};
// Elements [c, c + 8) of a row of `width` elements, zero behind its end.
template <bool F32>
__device__ __forceinline__ Row8 load_row8(const void* base, long long row_at, long long c, long long width) {
  Row8 r;
  if constexpr (F32) {
    const float* p = static_cast<const float*>(base) + row_at + c;
    if (c + 8 <= width) {
      const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.v[e] = a[e], r.v[4 + e] = b[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.v[e] = c + e < width ? p[e] : 0.f;
    }
  } else {
    const u16* p = static_cast<const u16*>(base) + row_at + c;
    if (c + 8 <= width) {
      const u32x4 a = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.v[2 * e] = bf16_lo(a[e]), r.v[2 * e + 1] = bf16_hi(a[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.v[e] = c + e < width ? bf16_value(p[e]) : 0.f;
    }
  }
  return r;
}
// Eight fp32 values as operand planes: each plane what the ones before it left, rounded to bf16.
template <bool F32>
__device__ __forceinline__ void store_planes8(const Row8& r, u16* dst, long long plane) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = r.v[e];
#pragma unroll
  for (int q = 0; q < (F32 ? 3 : 1); ++q) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
      v[2 * e] -= bf16_lo(w[e]);
      v[2 * e + 1] -= bf16_hi(w[e]);
    }
    *reinterpret_cast<u32x4*>(dst + q * plane) = w;
  }
}

}  // namespace head
}  // namespace muon
