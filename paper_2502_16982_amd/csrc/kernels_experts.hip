// Tokens to their experts and back: a stable sort of the pairs (token, choice) by expert, the tokens' rows copied into that order, the
// experts' rows summed back with weights, and the gradients.
//
//   position[t, j] = rank of (t, j) in the stable sort by expert        rows[position[t, j]] = x[t]
//   out[t] = sum_j w[t, j] rows[position[t, j]]                         d_x[t] = sum_j d_rows[position[t, j]]   (w = 1)
//   d_rows[position[t, j]] = w[t, j] d_out[t]                           d_w[t, j] = <d_out[t], rows[position[t, j]]>
//
// All of it is bound by memory: 8192 tokens x 6 rows of 2048 in bf16, dispatch 36 to 40 us (5.9 to 6.5 TB/s), combine 46 (5.1),
// combine_backward 79 (5.5), the sort 10 (two launches).  Every kernel goes by token: a token's row is read once and kept in registers while its `top` rows are
// written or read, so that x, out and d_out cross once and not `top` times.  Nothing is atomic but the integer counts of the sort, whose
// order does not matter.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "experts_launch.h"

namespace muon {
namespace {

typedef unsigned short u16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
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
// A thread moves 16 bytes of a row at a time, whatever the rows' alignment (global memory takes that at any address of an element; rows of
// 1409 fp32: 34 us for combine and its gradients in pieces of 4 bytes, 23 in these); what a row has left behind its last whole piece goes
// by element.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <bool F32>
struct Piece {
  static constexpr int N = F32 ? 4 : 8;
  typedef std::conditional_t<F32, float, u16> Elem;
  static __device__ __forceinline__ u32x4 load(const Elem* p) { return *reinterpret_cast<const u32x4_any*>(p); }
  // ONCE: with the streaming hint
  template <bool ONCE>
  static __device__ __forceinline__ u32x4 load_row(const Elem* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
    else return load(p);
  }
  static __device__ __forceinline__ void store(Elem* p, u32x4 v) { *reinterpret_cast<u32x4_any*>(p) = v; }
  static __device__ __forceinline__ void unpack(u32x4 raw, float (&v)[N]) {
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = __uint_as_float(raw[e]);
    } else {
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        v[2 * e] = __uint_as_float(raw[e] << 16);
        v[2 * e + 1] = __uint_as_float(raw[e] & 0xffff0000u);
      }
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&v)[N]) {
    u32x4 raw;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (F32) {
        raw[e] = __float_as_uint(v[e]);
      } else {
        const f32x2 two = {v[2 * e], v[2 * e + 1]};
        raw[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2));
      }
    }
    return raw;
  }
  static __device__ __forceinline__ float value(Elem x) {
    if constexpr (F32) return x;
    else return __uint_as_float((unsigned)x << 16);
  }
  static __device__ __forceinline__ Elem elem(float x) {
    if constexpr (F32) {
      return x;
    } else {
      const f32x2 two = {x, 0.f};
      return (u16)(__builtin_bit_cast(unsigned, __builtin_convertvector(two, bf16x2)) & 0xffffu);
    }
  }
};

// A token's threads are `lanes` neighbours (whole waves); a block takes 256 / lanes tokens at a time, and the grid goes on until all are done
// (a launch has fewer than 2^32 threads).  f(token, the thread's place among the token's).
constexpr long long kMaxBlocks = 1ll << 22;
template <typename F>
__device__ __forceinline__ void each_token(const ExpertRows& r, int lanes, F&& f) {
  const int per = 256 / lanes;
  for (long long first = (long long)blockIdx.x * per; first < r.tokens; first += (long long)gridDim.x * per)
    f(first + threadIdx.x / lanes, (int)(threadIdx.x % lanes));
}

// The row of pair i, or -1: what is no row of this call counts as dropped.
__device__ __forceinline__ long long row_of(const ExpertRows& r, long long i) {
  const int p = r.position[i];
  return p >= 0 && p < r.tokens * r.top ? p : -1;
}
// Rows behind the last pair's are zero.  Each token clears those with its own pairs' numbers.
template <bool F32>
__device__ __forceinline__ void clear_tail(const ExpertRows& r, long long token, typename Piece<F32>::Elem* rows, int at, int lanes) {
  using P = Piece<F32>;
  const long long count = *r.count;
  for (int j = 0; j < r.top; ++j) {
    const long long row = token * r.top + j;
    if (row < count) continue;
    for (long long c = (long long)at * P::N; c < r.width; c += (long long)lanes * P::N) {
      if (c + P::N <= r.width) P::store(rows + row * r.width + c, u32x4{0u, 0u, 0u, 0u});
      else
        for (long long e = c; e < r.width; ++e) rows[row * r.width + e] = 0;
    }
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void expert_dispatch_kernel(ExpertRows r, const void* __restrict__ x, long long x_stride,
                                                              void* __restrict__ rows_, int lanes) {
  using P = Piece<F32>;
  using Elem = typename P::Elem;
  Elem* rows = static_cast<Elem*>(rows_);
  each_token(r, lanes, [&](long long token, int at) {
    if (token >= r.tokens) return;
    const Elem* mine = static_cast<const Elem*>(x) + token * x_stride;
    for (long long c = (long long)at * P::N; c < r.width; c += (long long)lanes * P::N) {
      if (c + P::N <= r.width) {
        const u32x4 v = P::load(mine + c);
        for (int j = 0; j < r.top; ++j) {
          const long long row = row_of(r, token * r.top + j);
          if (row >= 0) P::store(rows + row * r.width + c, v);
        }
      } else {
        for (int j = 0; j < r.top; ++j) {
          const long long row = row_of(r, token * r.top + j);
          if (row >= 0)
            for (long long e = c; e < r.width; ++e) rows[row * r.width + e] = mine[e];
        }
      }
    }
    clear_tail<F32>(r, token, rows, at, lanes);
  });
}

// ROWS rows of a token on their way at a time.
template <bool F32, int ROWS, bool ONCE>
__global__ __launch_bounds__(256) void expert_combine_kernel(ExpertRows r, const void* __restrict__ rows_, const float* __restrict__ weights,
                                                             void* __restrict__ out_, int lanes) {
  using P = Piece<F32>;
  using Elem = typename P::Elem;
  const Elem* rows = static_cast<const Elem*>(rows_);
  each_token(r, lanes, [&](long long token, int at) {
    if (token >= r.tokens) return;
    Elem* out = static_cast<Elem*>(out_) + token * r.width;
    for (long long c = (long long)at * P::N; c < r.width; c += (long long)lanes * P::N) {
      const bool whole = c + P::N <= r.width;
      float sum[P::N];
#pragma unroll
      for (int e = 0; e < P::N; ++e) sum[e] = 0.f;
      for (int j0 = 0; j0 < r.top; j0 += ROWS) {
        long long row[ROWS];
        float w[ROWS];
        u32x4 v[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
          const long long i = token * r.top + j0 + u;
          row[u] = j0 + u < r.top ? row_of(r, i) : -1;
          w[u] = row[u] < 0 ? 0.f : weights ? weights[i] : 1.f;
        }
        if (whole) {
#pragma unroll
          for (int u = 0; u < ROWS; ++u) v[u] = row[u] < 0 ? u32x4{0u, 0u, 0u, 0u} : P::template load_row<ONCE>(rows + row[u] * r.width + c);
#pragma unroll
          for (int u = 0; u < ROWS; ++u) {
            float f[P::N];
            P::unpack(v[u], f);
#pragma unroll
            for (int e = 0; e < P::N; ++e)
              if (row[u] >= 0) sum[e] = fmaf(w[u], f[e], sum[e]);
          }
        } else {
#pragma unroll
          for (int u = 0; u < ROWS; ++u)
#pragma unroll
            for (int e = 0; e < P::N; ++e)
              if (row[u] >= 0 && c + e < r.width) sum[e] = fmaf(w[u], P::value(rows[row[u] * r.width + c + e]), sum[e]);
        }
      }
      if (whole) {
        P::store(out + c, P::pack(sum));
      } else {
#pragma unroll
        for (int e = 0; e < P::N; ++e)
          if (c + e < r.width) out[c + e] = P::elem(sum[e]);
      }
    }
  });
}

template <bool F32, bool ONCE>
__global__ __launch_bounds__(256) void expert_combine_backward_kernel(ExpertRows r, const void* __restrict__ d_out, long long d_out_stride,
                                                                      const void* __restrict__ rows_, const float* __restrict__ weights,
                                                                      void* __restrict__ d_rows_, float* __restrict__ d_weights, int lanes) {
  using P = Piece<F32>;
  using Elem = typename P::Elem;
  __shared__ float dots[kMaxExpertTop][4];
  const Elem* rows = static_cast<const Elem*>(rows_);
  Elem* d_rows = static_cast<Elem*>(d_rows_);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  each_token(r, lanes, [&](long long token, int at) {
    const bool there = token < r.tokens;         // (of a whole wave)
    if (there) {
      const Elem* mine = static_cast<const Elem*>(d_out) + token * d_out_stride;
      for (int j = 0; j < r.top; ++j) {
        const long long i = token * r.top + j, row = row_of(r, i);
        float dot = 0.f;
        if (row >= 0) {
          const float w = weights[i];
          const Elem* y = rows + row * r.width;
          Elem* dy = d_rows + row * r.width;
          for (long long c = (long long)at * P::N; c < r.width; c += (long long)lanes * P::N) {
            if (c + P::N <= r.width) {
              float g[P::N], f[P::N];
              P::unpack(P::load(mine + c), g);
              P::unpack(P::template load_row<ONCE>(y + c), f);
#pragma unroll
              for (int e = 0; e < P::N; ++e) {
                dot = fmaf(g[e], f[e], dot);
                g[e] *= w;
              }
              P::store(dy + c, P::pack(g));
            } else {
              for (long long e = c; e < r.width; ++e) {
                const float g = P::value(mine[e]);
                dot = fmaf(g, P::value(y[e]), dot);
                dy[e] = P::elem(w * g);
              }
            }
          }
#pragma unroll
          for (int off = 32; off > 0; off >>= 1) dot += __shfl_xor(dot, off, 64);
        }
        if (lane == 0) dots[j][wave] = dot;
      }
      clear_tail<F32>(r, token, d_rows, at, lanes);
    }
    __syncthreads();
    if (there) {
      const int waves = lanes / 64, first = threadIdx.x / lanes * waves;
      for (int j = at; j < r.top; j += lanes) {
        float sum = 0.f;
        for (int u = 0; u < waves; ++u) sum += dots[j][first + u];
        d_weights[token * r.top + j] = sum;
      }
    }
    __syncthreads();                             // (the next token's dots go to the same place)
  });
}

// Rows from 128 MB on, which with what is written beside them fill the memory-side cache (256 MB), are read with the streaming hint.  Without -> with it, in us,
// rows of 2048 bf16: combine and its gradients on new rows each time, 64 MB 44 -> 49, 96 MB 71 -> 69, 128 MB 96 -> 86, 192 MB 140 -> 124, 256 MB
// 185 -> 182, 384 MB 271 -> 273; the gradients alone on rows read before, 96 MB 37 -> 44, 128 MB 59 -> 55, 192 MB 92 -> 78.  combine alone
// loses by it where its rows are in the cache (128 MB 28 -> 31, 192 MB 38 -> 48), is even where they are not (33 -> 31, 46 -> 47) and wins
// behind a dispatch of as many rows (201 MB: the two 116 -> 94).  fp32 rows of 1408 alike.
bool rows_once(const ExpertRows& r) { return r.tokens * r.top * r.width * (r.f32 ? 4 : 2) >= 128ll << 20; }
// Threads per token: whole waves, as many as have a piece of the row each.
int lanes_for(const ExpertRows& r) {
  const long long pieces = r.width * (r.f32 ? 4 : 2) / 16;
  return pieces <= 64 ? 64 : pieces <= 128 ? 128 : 256;
}
unsigned blocks_for(const ExpertRows& r, int lanes) {
  const long long blocks = (r.tokens + 256 / lanes - 1) / (256 / lanes);
  return (unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks);
}

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
  const int lanes = lanes_for(r);
  if (r.f32) expert_dispatch_kernel<true><<<blocks_for(r, lanes), 256, 0, s>>>(r, x, x_stride, rows, lanes);
  else expert_dispatch_kernel<false><<<blocks_for(r, lanes), 256, 0, s>>>(r, x, x_stride, rows, lanes);
  return hipGetLastError();
}

hipError_t launch_expert_combine(const ExpertRows& r, const void* rows, const float* weights, void* out, hipStream_t s) {
  const int lanes = lanes_for(r);
  auto go = [&](auto kernel) {
    kernel<<<blocks_for(r, lanes), 256, 0, s>>>(r, rows, weights, out, lanes);
    return hipGetLastError();
  };
#define MUON_COMBINE_CASE(F32, ROWS, ONCE) \
  if ((r.f32 != 0) == F32 && (r.top <= 2 ? 2 : 8) == ROWS && once == ONCE) return go(expert_combine_kernel<F32, ROWS, ONCE>)
  const bool once = rows_once(r);
  MUON_COMBINE_CASE(false, 2, false);
  MUON_COMBINE_CASE(false, 2, true);
  MUON_COMBINE_CASE(false, 8, false);
  MUON_COMBINE_CASE(false, 8, true);
  MUON_COMBINE_CASE(true, 2, false);
  MUON_COMBINE_CASE(true, 2, true);
  MUON_COMBINE_CASE(true, 8, false);
  MUON_COMBINE_CASE(true, 8, true);
#undef MUON_COMBINE_CASE
  return hipErrorInvalidValue;
}

hipError_t launch_expert_combine_backward(const ExpertRows& r, const void* d_out, long long d_out_stride, const void* rows,
                                          const float* weights, void* d_rows, float* d_weights, hipStream_t s) {
  const int lanes = lanes_for(r);
  auto go = [&](auto kernel) {
    kernel<<<blocks_for(r, lanes), 256, 0, s>>>(r, d_out, d_out_stride, rows, weights, d_rows, d_weights, lanes);
    return hipGetLastError();
  };
  if (rows_once(r)) return r.f32 ? go(expert_combine_backward_kernel<true, true>) : go(expert_combine_backward_kernel<false, true>);
  return r.f32 ? go(expert_combine_backward_kernel<true, false>) : go(expert_combine_backward_kernel<false, false>);
}

}  // namespace muon
