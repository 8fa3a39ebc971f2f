// Tokens to their experts and back: a stable sort of the pairs (token, choice) by expert, the tokens' rows copied into that order, the
// experts' rows summed back with weights, and the gradients.
//
//   position[t, j] = rank of (t, j) in the stable sort by expert        rows[position[t, j]] = x[t]
//   out[t] = sum_j w[t, j] rows[position[t, j]]                         d_x[t] = sum_j d_rows[position[t, j]]   (w = 1)
//   d_rows[position[t, j]] = w[t, j] d_out[t]                           d_w[t, j] = <d_out[t], rows[position[t, j]]>
//
// All of it is bound by memory.  Every kernel goes by token: a token's row is read once and kept in registers while its `top` rows are
// written or read, so that x, out and d_out cross once and not `top` times.  Nothing is atomic but the integer counts of the sort, whose
// order does not matter.
#include <hip/hip_runtime.h>

#include "experts_launch.h"

namespace muon {
namespace {

typedef unsigned short u16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---- sort ----
__device__ __forceinline__ int expert_at(const void* expert, int index64, long long i, int experts) {
  const long long e = index64 ? static_cast<const long long*>(expert)[i] : (long long)static_cast<const int*>(expert)[i];
  return e >= 0 && e < experts ? (int)e : -1;
}

__global__ __launch_bounds__(256) void expert_count_kernel(const void* __restrict__ expert, int index64, long long pairs, long long chunk,
                                                           int experts, int* __restrict__ counts) {
  extern __shared__ int lds[];
  for (int e = threadIdx.x; e < experts; e += 256) lds[e] = 0;
  __syncthreads();
  const long long first = blockIdx.x * chunk, last = first + chunk < pairs ? first + chunk : pairs;
  for (long long i = first + threadIdx.x; i < last; i += 256) {
    const int e = expert_at(expert, index64, i, experts);
    if (e >= 0) atomicAdd(&lds[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += 256) counts[(long long)blockIdx.x * experts + e] = lds[e];
}

// Each wave places a quarter of the block's pairs, 64 at a time: lanes of one expert find each other bit by bit, rank among themselves by
// lane and take the next places of the wave's counter for that expert.
__global__ __launch_bounds__(256) void expert_place_kernel(const void* __restrict__ expert, int index64, long long pairs, long long chunk,
                                                           int experts, int bits, const int* __restrict__ counts, int blocks,
                                                           int* __restrict__ position, int* __restrict__ source, int* __restrict__ offsets) {
  extern __shared__ int lds[];
  int* next = lds;                     // [4][experts]: counts, then the next place
  int* total = lds + 4 * experts;      // pairs of each expert, then its first place
  int* before = lds + 5 * experts;     // pairs of each expert in the blocks before this one
  __shared__ int all;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int e = threadIdx.x; e < 6 * experts; e += 256) lds[e] = 0;
  __syncthreads();
  const long long quarter = chunk / 4;
  long long first = blockIdx.x * chunk + wave * quarter, last = first + quarter;
  first = first < pairs ? first : pairs;
  last = last < pairs ? last : pairs;
  for (long long i = first + lane; i < last; i += 64) {
    const int e = expert_at(expert, index64, i, experts);
    if (e >= 0) atomicAdd(&next[wave * experts + e], 1);
  }
  if (blocks > 1) {                    // threads of one expert share the blocks
    const int shares = experts < 256 ? 256 / experts : 1;
    for (int u = threadIdx.x; u < experts * shares; u += 256) {
      const int e = u % experts;
      int sum = 0, left = 0;
#pragma unroll 8
      for (int b = u / experts; b < blocks; b += shares) {
        const int c = counts[(long long)b * experts + e];
        sum += c;
        left += b < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&total[e], sum);
      atomicAdd(&before[e], left);
    }
  }
  __syncthreads();
  if (blocks == 1) {
    for (int e = threadIdx.x; e < experts; e += 256)
      total[e] = next[e] + next[experts + e] + next[2 * experts + e] + next[3 * experts + e];
    __syncthreads();
  }
  if (wave == 0) {                     // exclusive sums over the experts
    int carry = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
      const int e = e0 + lane, c = e < experts ? total[e] : 0;
      int x = c;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off, 64);
        if (lane >= off) x += y;
      }
      if (e < experts) {
        total[e] = carry + x - c;
        if (blockIdx.x == 0) offsets[e] = carry + x - c;
      }
      carry += __shfl(x, 63, 64);
    }
    if (lane == 0) {
      all = carry;
      if (blockIdx.x == 0) offsets[experts] = carry;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += 256) {
    int at = total[e] + before[e];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int c = next[w * experts + e];
      next[w * experts + e] = at;
      at += c;
    }
  }
  __syncthreads();
  volatile int* mine = next + wave * experts;
  for (long long i0 = first; i0 < last; i0 += 64) {
    const long long i = i0 + lane;
    const int e = i < last ? expert_at(expert, index64, i, experts) : -1;
    unsigned long long same = __ballot(e >= 0);
    for (int b = 0; b < bits; ++b) {
      const unsigned long long set = __ballot((e >> b) & 1);
      same &= (e >> b) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    int at = -1;
    if (e >= 0) at = mine[e] + rank;
    __builtin_amdgcn_wave_barrier();   // every lane has read its counter
    if (e >= 0 && rank == 0) mine[e] = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (i < last) position[i] = at;
    if (e >= 0) source[at] = (int)i;
  }
  const long long end = (blockIdx.x + 1) * chunk < pairs ? (blockIdx.x + 1) * chunk : pairs;
  for (long long i = blockIdx.x * chunk + threadIdx.x; i < end; i += 256)
    if (i >= all) source[i] = -1;
}

// ---- rows ----
// A piece of a row in one thread: BYTES of bf16 or fp32 elements.
template <int BYTES>
struct RawOf;
template <> struct RawOf<16> { typedef u32x4 type; };
template <> struct RawOf<8> { typedef u32x2 type; };
template <> struct RawOf<4> { typedef unsigned type; };
template <> struct RawOf<2> { typedef u16 type; };

template <int BYTES, bool F32>
struct Piece {
  static constexpr int N = BYTES / (F32 ? 4 : 2);
  typedef typename RawOf<BYTES>::type Raw;
  static __device__ __forceinline__ void unpack(Raw raw, float (&v)[N]) {
    if constexpr (F32) {
      if constexpr (N == 1) v[0] = __uint_as_float(raw);
      else
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = __uint_as_float(raw[e]);
    } else if constexpr (N == 1) {
      v[0] = __uint_as_float((unsigned)raw << 16);
    } else {
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        unsigned w;
        if constexpr (N == 2) w = raw;
        else w = raw[e];
        v[2 * e] = __uint_as_float(w << 16);
        v[2 * e + 1] = __uint_as_float(w & 0xffff0000u);
      }
    }
  }
  static __device__ __forceinline__ Raw pack(const float (&v)[N]) {
    Raw raw;
    if constexpr (F32) {
      if constexpr (N == 1) raw = __float_as_uint(v[0]);
      else
#pragma unroll
        for (int e = 0; e < N; ++e) raw[e] = __float_as_uint(v[e]);
    } else if constexpr (N == 1) {
      const f32x2 two = {v[0], 0.f};
      raw = (u16)(__builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2)) & 0xffffu);
    } else {
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        const f32x2 two = {v[2 * e], v[2 * e + 1]};
        const unsigned w = __builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2));
        if constexpr (N == 2) raw = w;
        else raw[e] = w;
      }
    }
    return raw;
  }
};

// The row of pair i, or -1: what is no row of this call counts as dropped.
__device__ __forceinline__ long long row_of(const ExpertRows& r, long long i) {
  const int p = r.position[i];
  return p >= 0 && p < r.tokens * r.top ? p : -1;
}
// Rows behind the last pair's are zero.  Each token clears those with its own pairs' numbers.
template <typename Raw>
__device__ __forceinline__ void clear_tail(const ExpertRows& r, long long token, Raw* rows, long long pieces, int at, int lanes) {
  const long long count = *r.count;
  for (int j = 0; j < r.top; ++j) {
    const long long row = token * r.top + j;
    if (row < count) continue;
    for (long long c = at; c < pieces; c += lanes) rows[row * pieces + c] = Raw{};
  }
}

template <typename Raw>
__global__ __launch_bounds__(256) void expert_dispatch_kernel(ExpertRows r, const unsigned char* __restrict__ x, long long x_stride,
                                                              Raw* __restrict__ rows, long long pieces, int lanes) {
  const long long token = blockIdx.x * (256ll / lanes) + threadIdx.x / lanes;
  const int at = threadIdx.x % lanes;
  if (token >= r.tokens) return;
  const Raw* mine = reinterpret_cast<const Raw*>(x + token * x_stride);
  for (long long c = at; c < pieces; c += lanes) {
    const Raw v = mine[c];
    for (int j = 0; j < r.top; ++j) {
      const long long row = row_of(r, token * r.top + j);
      if (row >= 0) rows[row * pieces + c] = v;
    }
  }
  clear_tail(r, token, rows, pieces, at, lanes);
}

template <int BYTES, bool F32>
__global__ __launch_bounds__(256) void expert_combine_kernel(ExpertRows r, const void* __restrict__ rows_, const float* __restrict__ weights,
                                                             void* __restrict__ out_, long long pieces, int lanes) {
  constexpr int ROWS = 8;
  using P = Piece<BYTES, F32>;
  using Raw = typename P::Raw;
  const Raw* rows = static_cast<const Raw*>(rows_);
  Raw* out = static_cast<Raw*>(out_);
  const long long token = blockIdx.x * (256ll / lanes) + threadIdx.x / lanes;
  if (token >= r.tokens) return;
  for (long long c = threadIdx.x % lanes; c < pieces; c += lanes) {
    float sum[P::N];
#pragma unroll
    for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
    for (int j0 = 0; j0 < r.top; j0 += ROWS) {   // ROWS rows on their way at a time
      long long row[ROWS];
      float w[ROWS];
      Raw v[ROWS];
#pragma unroll
      for (int u = 0; u < ROWS; ++u) {
        const long long i = token * r.top + j0 + u;
        row[u] = j0 + u < r.top ? row_of(r, i) : -1;
        w[u] = row[u] < 0 ? 0.f : weights ? weights[i] : 1.f;
      }
#pragma unroll
      for (int u = 0; u < ROWS; ++u) v[u] = row[u] < 0 ? Raw{} : rows[row[u] * pieces + c];
#pragma unroll
      for (int u = 0; u < ROWS; ++u) {
        float f[P::N];
        P::unpack(v[u], f);
#pragma unroll
        for (int e = 0; e < P::N; ++e) sum[e] = fmaf(w[u], f[e], sum[e]);
      }
    }
    out[token * pieces + c] = P::pack(sum);
  }
}

template <int BYTES, bool F32>
__global__ __launch_bounds__(256) void expert_combine_backward_kernel(ExpertRows r, const unsigned char* __restrict__ d_out,
                                                                      long long d_out_stride, const void* __restrict__ rows_,
                                                                      const float* __restrict__ weights, void* __restrict__ d_rows_,
                                                                      float* __restrict__ d_weights, long long pieces, int lanes) {
  using P = Piece<BYTES, F32>;
  using Raw = typename P::Raw;
  __shared__ float dots[kMaxExpertTop][4];
  const Raw* rows = static_cast<const Raw*>(rows_);
  Raw* d_rows = static_cast<Raw*>(d_rows_);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at = threadIdx.x % lanes;
  const long long token = blockIdx.x * (256ll / lanes) + threadIdx.x / lanes;
  const bool there = token < r.tokens;           // (of a whole wave)
  if (there) {
    const Raw* mine = reinterpret_cast<const Raw*>(d_out + token * d_out_stride);
    for (int j = 0; j < r.top; ++j) {
      const long long i = token * r.top + j, row = row_of(r, i);
      float dot = 0.f;
      if (row >= 0) {
        const float w = weights[i];
        for (long long c = at; c < pieces; c += lanes) {
          float g[P::N], y[P::N];
          P::unpack(mine[c], g);
          P::unpack(rows[row * pieces + c], y);
#pragma unroll
          for (int e = 0; e < P::N; ++e) {
            dot = fmaf(g[e], y[e], dot);
            g[e] *= w;
          }
          d_rows[row * pieces + c] = P::pack(g);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) dot += __shfl_xor(dot, off, 64);
      }
      if (lane == 0) dots[j][wave] = dot;
    }
    clear_tail(r, token, d_rows, pieces, at, lanes);
  }
  __syncthreads();
  if (!there) return;
  const int waves = lanes / 64, first = threadIdx.x / lanes * waves;
  for (int j = at; j < r.top; j += lanes) {
    float sum = 0.f;
    for (int u = 0; u < waves; ++u) sum += dots[j][first + u];
    d_weights[token * r.top + j] = sum;
  }
}

// The widest piece that rows of that many bytes and these addresses come in.
int piece_bytes(long long row_bytes, long long stride_bytes, const void* a, const void* b, const void* c) {
  const unsigned long long all = (unsigned long long)row_bytes | (unsigned long long)stride_bytes | reinterpret_cast<uintptr_t>(a) |
                                 reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c);
  return all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : 2;
}
// Threads per token: whole waves, as many as have a piece of the row each.
int lanes_for(long long pieces) { return pieces <= 64 ? 64 : pieces <= 128 ? 128 : 256; }

}  // namespace

hipError_t launch_expert_sort(const void* expert, int index64, int64_t pairs, int experts, int* position, int* source, int* offsets,
                              int* counts, hipStream_t s) {
  const int blocks = sort_blocks(pairs);
  const long long chunk = sort_chunk(pairs);
  int bits = 0;
  while ((1 << bits) < experts) ++bits;
  if (blocks > 1) {
    expert_count_kernel<<<blocks, 256, experts * sizeof(int), s>>>(expert, index64, pairs, chunk, experts, counts);
    if (hipError_t e = hipGetLastError()) return e;
  }
  const size_t lds = 6ull * experts * sizeof(int);
  if (lds > 65536) {
    if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(expert_place_kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           6 * kMaxExperts * (int)sizeof(int)))
      return e;
  }
  expert_place_kernel<<<blocks, 256, lds, s>>>(expert, index64, pairs, chunk, experts, bits, counts, blocks, position, source, offsets);
  return hipGetLastError();
}

hipError_t launch_expert_dispatch(const ExpertRows& r, const void* x, long long x_stride, void* rows, hipStream_t s) {
  const int size = r.f32 ? 4 : 2, bytes = piece_bytes(r.width * size, x_stride * size, x, rows, nullptr);
  const long long pieces = r.width * size / bytes;
  const int lanes = lanes_for(pieces), per = 256 / lanes;
  const unsigned blocks = (unsigned)((r.tokens + per - 1) / per);
  auto go = [&](auto raw) {
    using Raw = decltype(raw);
    expert_dispatch_kernel<Raw><<<blocks, 256, 0, s>>>(r, static_cast<const unsigned char*>(x), x_stride * size, static_cast<Raw*>(rows),
                                                       pieces, lanes);
    return hipGetLastError();
  };
  switch (bytes) {
    case 16: return go(u32x4{});
    case 8: return go(u32x2{});
    case 4: return go(unsigned{});
    default: return go(u16{});
  }
}

hipError_t launch_expert_combine(const ExpertRows& r, const void* rows, const float* weights, void* out, hipStream_t s) {
  const int size = r.f32 ? 4 : 2, bytes = piece_bytes(r.width * size, 0, rows, out, nullptr);
  const long long pieces = r.width * size / bytes;
  const int lanes = lanes_for(pieces), per = 256 / lanes;
  const unsigned blocks = (unsigned)((r.tokens + per - 1) / per);
  auto go = [&](auto kernel) {
    kernel<<<blocks, 256, 0, s>>>(r, rows, weights, out, pieces, lanes);
    return hipGetLastError();
  };
  if (r.f32) return bytes == 16 ? go(expert_combine_kernel<16, true>) : bytes == 8 ? go(expert_combine_kernel<8, true>) : go(expert_combine_kernel<4, true>);
  switch (bytes) {
    case 16: return go(expert_combine_kernel<16, false>);
    case 8: return go(expert_combine_kernel<8, false>);
    case 4: return go(expert_combine_kernel<4, false>);
    default: return go(expert_combine_kernel<2, false>);
  }
}

hipError_t launch_expert_combine_backward(const ExpertRows& r, const void* d_out, long long d_out_stride, const void* rows,
                                          const float* weights, void* d_rows, float* d_weights, hipStream_t s) {
  const int size = r.f32 ? 4 : 2, bytes = piece_bytes(r.width * size, d_out_stride * size, d_out, rows, d_rows);
  const long long pieces = r.width * size / bytes;
  const int lanes = lanes_for(pieces), per = 256 / lanes;
  const unsigned blocks = (unsigned)((r.tokens + per - 1) / per);
  auto go = [&](auto kernel) {
    kernel<<<blocks, 256, 0, s>>>(r, static_cast<const unsigned char*>(d_out), d_out_stride * size, rows, weights, d_rows, d_weights, pieces,
                                  lanes);
    return hipGetLastError();
  };
  if (r.f32)
    return bytes == 16 ? go(expert_combine_backward_kernel<16, true>)
           : bytes == 8 ? go(expert_combine_backward_kernel<8, true>) : go(expert_combine_backward_kernel<4, true>);
  switch (bytes) {
    case 16: return go(expert_combine_backward_kernel<16, false>);
    case 8: return go(expert_combine_backward_kernel<8, false>);
    case 4: return go(expert_combine_backward_kernel<4, false>);
    default: return go(expert_combine_backward_kernel<2, false>);
  }
}

}  // namespace muon
