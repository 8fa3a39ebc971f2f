// The norm of a list of gradients as one vector, and the gradients times a factor.
//
//   norm = sqrt(sum g^2)     scale = max_norm / norm where norm > max_norm, else 1     g <- scale g
//
// Bound by memory: the norm reads every element once, scaling reads and writes it.  Squares are summed in double: what fp32 gradients
// square to does not fit fp32, neither large (beyond 1.8e19) nor small (below 1e-19), and a sum of 10^10 of them keeps its digits; it costs
// nothing (sums of eight squares in fp32 instead: 82 us for 2^28 bf16 elements either way).  A block leaves one partial sum; they are summed in a
// fixed order.
// Accesses of a call that scales in place carry the streaming hint.  Without it a pass over the gradients has whatever a backward pass left dirty in the
// memory-side cache written back to make room: 2^28 bf16 elements, 537 MB, after 600 MB of writes, norm 148 us (3.6 TB/s) without, 82 us
// (6.5 TB/s) with; norm and scaling 241 -> 192 us at 403 MB, 69 -> 50 us at 101 MB; where nothing else came between, of up to 256 MB, 119 -> 125 at
// most.  A norm alone goes without: the step that follows reads and writes three times as much and has the write-backs to pay otherwise (184 M bf16
// elements, norm and AdamW 802 us without, 846 with).
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

#define MUON_GLOBAL __attribute__((address_space(1)))

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
  template <bool STREAM>
  __device__ __forceinline__ void load(const u16* p) {
    const MUON_GLOBAL u32x4_any* q = (const MUON_GLOBAL u32x4_any*)p;
    if constexpr (STREAM) v = __builtin_nontemporal_load(q);
    else v = *q;
  }
  __device__ __forceinline__ void store(u16* p) const { __builtin_nontemporal_store(v, (MUON_GLOBAL u32x4_any*)p); }
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
  template <bool STREAM>
  __device__ __forceinline__ void load(const float* p) {
    const MUON_GLOBAL f32x4_any* q = (const MUON_GLOBAL f32x4_any*)p;
    if constexpr (STREAM) v = __builtin_nontemporal_load(q);
    else v = *q;
  }
  __device__ __forceinline__ void store(float* p) const { __builtin_nontemporal_store(v, (MUON_GLOBAL f32x4_any*)p); }
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

// A block's span, kAhead chunks per thread on their way at a time, then element by element what is less than a chunk.  chunk(c): what is done with
// a chunk; back(c, address) and one(address) after it.
template <bool STREAM, typename T, typename F, typename B, typename G>
__device__ __forceinline__ void over_span(T* p, long long count, F&& chunk, B&& back, G&& one) {
  using C = Chunk<std::remove_const_t<T>>;
  constexpr int kStep = 256 * C::N;
  for (long long i = threadIdx.x * C::N; i < count; i += kAhead * kStep) {
    C c[kAhead];
    const long long left = count - i;                      // (from the thread's first chunk on)
    if (left >= (kAhead - 1) * kStep + C::N) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) c[u].template load<STREAM>(p + i + u * kStep);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        chunk(c[u]);
        back(c[u], p + i + u * kStep);
      }
      continue;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (left >= u * kStep + C::N) c[u].template load<STREAM>(p + i + u * kStep);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (left >= u * kStep + C::N) {
        chunk(c[u]);
        back(c[u], p + i + u * kStep);
      } else if (left > u * kStep) {
#pragma unroll
        for (int k = 0; k < C::N - 1; ++k)
          if (left > u * kStep + k) one(p + i + u * kStep + k);
      }
    }
  }
}

template <bool STREAM, typename T>
__device__ __forceinline__ double span_squares(const T* p, long long count) {
  double sum[2] = {0.0, 0.0};
  over_span<STREAM>(
      p, count, [&](const Chunk<T>& c) { c.add_squares(sum); }, [](const Chunk<T>&, const T*) {},
      [&](const T* at) {
        const double x = value(*at);
        sum[0] = fma(x, x, sum[0]);
      });
  return sum[0] + sum[1];
}
template <typename T>
__device__ __forceinline__ void span_scale(T* p, long long count, float s) {
  over_span<true>(
      p, count, [&](Chunk<T>& c) { c.scale(s); }, [](const Chunk<T>& c, T* at) { c.store(at); }, [&](T* at) { put(at, s * value(*at)); });
}

struct Piece {
  void* g;
  long long begin, count;                        // of the block's elements
  bool f32;
};
__device__ __forceinline__ Piece piece_of(const GradBatch& b, int block) {
  // the last tensor that starts at the block or before it: 192 comparisons at once (a search would be eight loads, one after the other)
  const int lane = threadIdx.x & 63;
  int t = -1;
#pragma unroll
  for (int k = 0; k < kGradSlots; k += 64) t += __popcll(__ballot(k + lane < b.n && b.block_start[k + lane] <= block));
  t = __builtin_amdgcn_readfirstlane(t);
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

template <bool STREAM>
__global__ __launch_bounds__(256) void grad_squares_kernel(GradBatch b, double* __restrict__ partial) {
  const Piece p = piece_of(b, blockIdx.x);
  double x = p.f32 ? span_squares<STREAM>(static_cast<const float*>(p.g) + p.begin, p.count) : span_squares<STREAM>(static_cast<const u16*>(p.g) + p.begin, p.count);
  x = block_sum(x);
  if (threadIdx.x == 0) partial[blockIdx.x] = x;
}

__device__ __forceinline__ float scale_of(double norm, double max_norm) {
  return norm > max_norm && norm < (double)INFINITY ? (float)(max_norm / norm) : 1.f;
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
  if (scale) *scale = scale_of(x, max_norm);
}

__global__ __launch_bounds__(256) void grad_scale_kernel(GradBatch b, const float* __restrict__ scale) {
  const float s = *scale;
  if (s == 1.f) return;
  const Piece p = piece_of(b, blockIdx.x);
  if (p.f32) span_scale(static_cast<float*>(p.g) + p.begin, p.count, s);
  else span_scale(static_cast<u16*>(p.g) + p.begin, p.count, s);
}

// Norm, scale and scaling of a short list: every block sums the partial sums itself, a launch less.
__global__ __launch_bounds__(256) void grad_norm_scale_kernel(GradBatch b, const double* __restrict__ partial, int n, double max_norm, double* __restrict__ norm,
                                                              float* __restrict__ scale) {
  __shared__ float factor;
  const Piece p = piece_of(b, blockIdx.x);
  const double x = sqrt(block_sum((int)threadIdx.x < n ? partial[threadIdx.x] : 0.0));
  if (threadIdx.x == 0) {
    factor = scale_of(x, max_norm);
    if (blockIdx.x == 0) {
      *norm = x;
      *scale = factor;
    }
  }
  __syncthreads();
  const float s = factor;
  if (s == 1.f) return;
  if (p.f32) span_scale(static_cast<float*>(p.g) + p.begin, p.count, s);
  else span_scale(static_cast<u16*>(p.g) + p.begin, p.count, s);
}

}  // namespace

hipError_t launch_grad_squares(const GradBatch& b, int blocks, bool stream, double* partial, hipStream_t s) {
  if (stream) grad_squares_kernel<true><<<blocks, 256, 0, s>>>(b, partial);
  else grad_squares_kernel<false><<<blocks, 256, 0, s>>>(b, partial);
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

hipError_t launch_grad_norm_scale(const GradBatch& b, int blocks, const double* partial, int n, double max_norm, double* norm, float* scale, hipStream_t s) {
  grad_norm_scale_kernel<<<blocks, 256, 0, s>>>(b, partial, n, max_norm, norm, scale);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradBatch& b, int blocks, const float* scale, hipStream_t s) {
  grad_scale_kernel<<<blocks, 256, 0, s>>>(b, scale);
  return hipGetLastError();
}

}  // namespace muon
