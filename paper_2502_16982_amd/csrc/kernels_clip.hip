// The norm of a list of gradients as one vector, and the gradients times a factor.
//
//   norm = sqrt(sum g^2)     scale = max_norm / norm where norm > max_norm, else 1     g <- scale g
//
// Bound by memory: the norm reads every element once, scaling reads and writes it.  Squares are summed in double: what fp32 gradients
// square to does not fit fp32, neither large (beyond 1.8e19) nor small (below 1e-19), and a sum of 10^10 of them keeps its digits.  A block
// leaves one partial sum; they are summed in a fixed order.
#include <hip/hip_runtime.h>

#include "clip_launch.h"

namespace muon {
namespace {

typedef unsigned short u16;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// global memory takes 16 bytes at any address of an element
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_lo(unsigned v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(unsigned v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ unsigned pack_bf16(float x, float y) {
  const f32x2 v = {x, y};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

template <typename T>
struct Chunk;                                    // 16 bytes
template <>
struct Chunk<u16> {
  static constexpr int N = 8;
  u32x4_any v;
  __device__ __forceinline__ void load(const u16* p) { v = *reinterpret_cast<const u32x4_any*>(p); }
  __device__ __forceinline__ void store(u16* p) const { *reinterpret_cast<u32x4_any*>(p) = v; }
  __device__ __forceinline__ void add_squares(double* sum) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double x = bf16_lo(v[e]), y = bf16_hi(v[e]);
      sum[0] = fma(x, x, sum[0]);
      sum[1] = fma(y, y, sum[1]);
    }
  }
  __device__ __forceinline__ void scale(float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack_bf16(s * bf16_lo(v[e]), s * bf16_hi(v[e]));
  }
};
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  f32x4_any v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x4_any*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<f32x4_any*>(p) = v; }
  __device__ __forceinline__ void add_squares(double* sum) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double x = v[e];
      sum[e & 1] = fma(x, x, sum[e & 1]);
    }
  }
  __device__ __forceinline__ void scale(float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = s * v[e];
  }
};
__device__ __forceinline__ float value(u16 v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ void put(u16* p, float v) { *p = (u16)(pack_bf16(v, 0.f) & 0xffffu); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

constexpr int kAhead = 8;                        // accesses of a thread on their way

// f(chunk's address) for the whole chunks of a block's span, kAhead at a time, g(element's address) for what is left.
template <typename T, typename F, typename G>
__device__ __forceinline__ void over_span(T* p, long long count, F&& many, G&& one) {
  constexpr int N = Chunk<std::remove_const_t<T>>::N, kStep = 256 * N;
  long long i = threadIdx.x * N;
  for (; i + (kAhead - 1) * kStep + N <= count; i += kAhead * kStep) many(p + i, std::integral_constant<int, kAhead>{});
  for (; i + N <= count; i += kStep) many(p + i, std::integral_constant<int, 1>{});
  for (long long k = 0; k < N && i + k < count; ++k) one(p + i + k);
}

template <typename T>
__device__ __forceinline__ double span_squares(const T* p, long long count) {
  double sum[2] = {0.0, 0.0};
  over_span(
      p, count,
      [&](const T* at, auto n) {
        constexpr int K = decltype(n)::value;
        Chunk<T> c[K];
#pragma unroll
        for (int u = 0; u < K; ++u) c[u].load(at + u * 256 * Chunk<T>::N);
#pragma unroll
        for (int u = 0; u < K; ++u) c[u].add_squares(sum);
      },
      [&](const T* at) {
        const double x = value(*at);
        sum[0] = fma(x, x, sum[0]);
      });
  return sum[0] + sum[1];
}
template <typename T>
__device__ __forceinline__ void span_scale(T* p, long long count, float s) {
  over_span(
      p, count,
      [&](T* at, auto n) {
        constexpr int K = decltype(n)::value;
        Chunk<T> c[K];
#pragma unroll
        for (int u = 0; u < K; ++u) c[u].load(at + u * 256 * Chunk<T>::N);
#pragma unroll
        for (int u = 0; u < K; ++u) {
          c[u].scale(s);
          c[u].store(at + u * 256 * Chunk<T>::N);
        }
      },
      [&](T* at) { put(at, s * value(*at)); });
}

struct Piece {
  void* g;
  long long begin, count;                        // of the block's elements
  bool f32;
};
__device__ __forceinline__ Piece piece_of(const GradBatch& b, int block) {
  int t = 0;
#pragma unroll
  for (int step = 128; step > 0; step /= 2)
    if (t + step < b.n && block >= b.block_start[t + step]) t += step;
  const uint64_t size = b.size[t];
  const long long numel = (long long)(size & ~kGradIsF32), begin = (long long)(block - b.block_start[t]) * kGradSpan;
  return {b.g[t], begin, numel - begin < kGradSpan ? numel - begin : kGradSpan, (size & kGradIsF32) != 0};
}

// Sum over a block's threads (up to 1024), in thread 0.
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double waves[16];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < (int)blockDim.x / 64; ++w) x += waves[w];
  return x;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(GradBatch b, double* __restrict__ partial) {
  const Piece p = piece_of(b, blockIdx.x);
  double x = p.f32 ? span_squares(static_cast<const float*>(p.g) + p.begin, p.count) : span_squares(static_cast<const u16*>(p.g) + p.begin, p.count);
  x = block_sum(x);
  if (threadIdx.x == 0) partial[blockIdx.x] = x;
}

__device__ __forceinline__ double sum_of(const double* __restrict__ v, long long n) {
  double x[4] = {0.0, 0.0, 0.0, 0.0};
  long long i = threadIdx.x;
  for (; i + 3 * 1024 < n; i += 4 * 1024)
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] += v[i + 1024 * u];
  for (; i < n; i += 1024) x[0] += v[i];
  return block_sum((x[0] + x[1]) + (x[2] + x[3]));
}
__global__ __launch_bounds__(1024) void grad_join_kernel(const double* __restrict__ partial, long long n, double* __restrict__ out) {
  const long long at = blockIdx.x * (long long)kGradJoin;
  const double x = sum_of(partial + at, n - at < kGradJoin ? n - at : kGradJoin);
  if (threadIdx.x == 0) out[blockIdx.x] = x;
}
__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* __restrict__ partial, long long n, double max_norm, double* __restrict__ norm,
                                                         float* __restrict__ scale) {
  const double x = sqrt(sum_of(partial, n));
  if (threadIdx.x) return;
  *norm = x;
  if (scale) *scale = x > max_norm && x < (double)INFINITY ? (float)(max_norm / x) : 1.f;
}

__global__ __launch_bounds__(256) void grad_scale_kernel(GradBatch b, const float* __restrict__ scale) {
  const float s = *scale;
  if (s == 1.f) return;
  const Piece p = piece_of(b, blockIdx.x);
  if (p.f32) span_scale(static_cast<float*>(p.g) + p.begin, p.count, s);
  else span_scale(static_cast<u16*>(p.g) + p.begin, p.count, s);
}

}  // namespace

hipError_t launch_grad_squares(const GradBatch& b, int blocks, double* partial, hipStream_t s) {
  grad_squares_kernel<<<blocks, 256, 0, s>>>(b, partial);
  return hipGetLastError();
}

hipError_t launch_grad_norm(double* partial, int64_t n, double max_norm, double* norm, float* scale, hipStream_t s) {
  if (n > kGradJoin) {
    const int64_t groups = (n + kGradJoin - 1) / kGradJoin;
    grad_join_kernel<<<(unsigned)groups, 1024, 0, s>>>(partial, n, partial + n);
    partial += n;
    n = groups;
  }
  grad_norm_kernel<<<1, 1024, 0, s>>>(partial, n, max_norm, norm, scale);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradBatch& b, int blocks, const float* scale, hipStream_t s) {
  grad_scale_kernel<<<blocks, 256, 0, s>>>(b, scale);
  return hipGetLastError();
}

}  // namespace muon
