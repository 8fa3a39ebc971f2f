// The products of the head's losses on the matrix cores: T = L R^T in tiles, 16-bit operands, fp32 accumulators (device code).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "head_launch.h"

namespace muon {
namespace head {

typedef unsigned short u16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned pack_bf16(float x, float y) {
  const f32x2 v = {x, y};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ unsigned pack_f16(float x, float y) {
  const f32x2 v = {x, y};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, f16x2));
}
__device__ __forceinline__ float bf16_lo(unsigned v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(unsigned v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ float bf16_value(u16 v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ u16 bf16_bits(float x) { return (u16)(pack_bf16(x, 0.f) & 0xffffu); }

constexpr float kLog2e = 1.44269504088896340736f;
// 2^15: the largest probability relative to its block's maximum lies high in f16's range, so that 2^-12 of relative precision holds
// down to 2^-29 of the maximum.
constexpr float kProbScale = 32768.f;

// The planes of the pair with that number, (0,0) (0,1) (1,0) (1,1) (0,2) (2,0): what is left out is below 2^-24.
__device__ __forceinline__ int pair_left(int pair) { return pair == 2 || pair == 3 ? 1 : pair == 5 ? 2 : 0; }
__device__ __forceinline__ int pair_right(int pair) { return pair == 1 || pair == 3 ? 1 : pair == 4 ? 2 : 0; }

// A 128 x 128 tile by four waves of 64 x 64: acc[i][j] of a wave holds, in lane (r, h), column 32 j + r and rows 32 i + 8 q + 4 h + e.
struct Tile128 {
  static constexpr int BM = 128, BN = 128, WM = 64, WN = 64, FM = 2, FN = 2, THREADS = 256;
  static constexpr int kLds = 2 * 128 * 64 * 2;

  f32x16 acc[FM][FN];
  int lane, wave, wm, wn;

  // One slab of an operand: 128 of its rows by 64 of K.
  template <bool KM>
  __device__ __forceinline__ void stage(const HeadOperand& o, const u16* p, long long row0, long long k0, long long k, u16* lds) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int c = threadIdx.x + 256 * n;
      const int major = KM ? c >> 4 : c >> 3, chunk = KM ? c & 15 : c & 7;     // row of 16 (K-major) or 8 chunks
      const long long a = KM ? k0 + major : row0 + major, b = KM ? row0 + 8 * chunk : k0 + 8 * chunk;
      const bool there = KM ? a < k && b < o.rows : a < o.rows && b < k;
      u32x4 v = {0u, 0u, 0u, 0u};
      if (there) v = *reinterpret_cast<const u32x4*>(p + a * o.ld + b);
      *reinterpret_cast<u32x4*>(lds + major * (KM ? 128 : 64) + 8 * chunk) = v;
    }
  }
  template <bool KM>
  __device__ __forceinline__ bf16x8 fragment(const u16* lds, int row, int k) {
    if constexpr (!KM) return *reinterpret_cast<const bf16x8*>(lds + row * 64 + k);
    unsigned short v[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = lds[(k + t) * 128 + row];
    return __builtin_bit_cast(bf16x8, v);
  }

  template <bool LKM, bool RKM>
  __device__ __forceinline__ void run(const HeadOperand& l, const HeadOperand& r, long long row0, long long col0, long long k, int first,
                                      int last, u16* lds) {
    lane = threadIdx.x & 63;
    wave = threadIdx.x >> 6;
    wm = wave >> 1;
    wn = wave & 1;
    for (int i = 0; i < FM; ++i)
      for (int j = 0; j < FN; ++j)
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    u16 *ls = lds, *rs = lds + 128 * 64;
    const int per_pair = (int)((k + kHeadSlab - 1) / kHeadSlab);
    for (int s = first; s < last; ++s) {
      const int pair = s / per_pair;
      const long long k0 = (long long)(s - pair * per_pair) * kHeadSlab;
      __syncthreads();
      stage<LKM>(l, l.p + pair_left(pair) * l.plane, row0, k0, k, ls);
      stage<RKM>(r, r.p + pair_right(pair) * r.plane, col0, k0, k, rs);
      __syncthreads();
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        bf16x8 a[FM], b[FN];
        const int at = 16 * kk + 8 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = fragment<LKM>(ls, wm * WM + 32 * i + (lane & 31), at);
#pragma unroll
        for (int j = 0; j < FN; ++j) b[j] = fragment<RKM>(rs, wn * WN + 32 * j + (lane & 31), at);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
      }
    }
  }
};

}  // namespace head
}  // namespace muon
