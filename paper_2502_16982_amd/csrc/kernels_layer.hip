// A mixture's layer on a few tokens: out_t = sum_j w_tj  h_tj Down_e,  h_tj = act(x_t Gate_e) * (x_t Up_e)  (no gate: act(x_t Up_e)),  e = expert of (t, j).
//
// Bound by memory: each chosen expert's matrices are read once, whatever the number of its tokens, and are all there is to read.  A wave
// multiplies 32 rows of a matrix at a time, straight from memory to registers: its lanes hold 8 (fp32: 4) neighbouring columns of 8 rows
// each, so that every load takes 256 bytes of a row, and the matrix instruction's own freedom does the rest: the order in which a sum over
// rows is taken and the columns that a tile of 16 is made of are free, so 8 x 8 blocks are transposed within a lane's registers (32 byte
// permutes for 64 elements), no LDS, no shuffles.  Tokens are the instruction's other 16 columns; an expert with more of them takes further tiles of 16.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "layer_launch.h"

namespace muon {
namespace {

typedef unsigned short u16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
// global memory takes 16 bytes at any address of an element
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

__device__ __forceinline__ unsigned pack_bf16(float x, float y) {
  const f32x2 v = {x, y};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

__device__ __forceinline__ int expert_of(const LayerPairs& p, int i) {
  const long long e = p.index64 ? static_cast<const long long*>(p.expert)[i] : (long long)static_cast<const int*>(p.expert)[i];
  return e >= 0 && e < p.experts ? (int)e : -1;
}

constexpr int kTile = 16;                        // pairs of a tile

// Pairs of expert e numbered [base, base + room) into list, in their order; the number of all its pairs is returned.  By the whole block of
// 256 threads; counts: 4 ints of LDS.
__device__ __forceinline__ int find_pairs(const LayerPairs& p, int e, int base, int room, int* list, int* counts) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int seen = 0;
  for (int at = 0; at < p.pairs; at += 256) {
    const int i = at + threadIdx.x;
    const bool mine = i < p.pairs && expert_of(p, i) == e;
    const unsigned long long ballot = __ballot(mine);
    __syncthreads();                             // (the counts of the round before are read)
    if (lane == 0) counts[wave] = __popcll(ballot);
    __syncthreads();
    int before = seen;
    for (int w = 0; w < wave; ++w) before += counts[w];
    const int rank = before + __popcll(ballot & ((1ull << lane) - 1)) - base;
    if (mine && rank >= 0 && rank < room) list[rank] = i;
    seen += counts[0] + counts[1] + counts[2] + counts[3];
  }
  __syncthreads();
  return seen;
}

__device__ __forceinline__ float activate(int act, float z) { return act == 0 ? z / (1.f + expf(-z)) : fmaxf(z, 0.f); }

template <bool F32>
struct Elem {
  using T = u16;
  static constexpr int COLS = 8, STEPS = 8;      // neighbouring columns of a lane; matrix instructions of 32 rows
};
template <>
struct Elem<true> {
  using T = float;
  static constexpr int COLS = 4, STEPS = 32;
};

// 32 rows of a matrix: 8 accesses of 16 bytes per lane.  Row of access j: bf16 8 g + j, fp32 16 (j / 4) + 4 g + j % 4, with g = lane / 16.
template <bool F32>
struct Slab {
  u32x4 v[8];
  static __device__ __forceinline__ int row(int j, int g) { return F32 ? 16 * (j / 4) + 4 * g + j % 4 : 8 * g + j; }
  __device__ __forceinline__ void load(const typename Elem<F32>::T* w, long long stride, int g) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const u32x4_any*>(w + row(j, g) * stride);
  }
  // rows [0, there) only; the others are zero
  __device__ __forceinline__ void load_some(const typename Elem<F32>::T* w, long long stride, int g, int there) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = u32x4{0u, 0u, 0u, 0u};
      if (row(j, g) < there) v[j] = *reinterpret_cast<const u32x4_any*>(w + row(j, g) * stride);
    }
  }
  // the same of `cols` columns
  __device__ __forceinline__ void load_few(const typename Elem<F32>::T* w, long long stride, int g, int there, int cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = u32x4{0u, 0u, 0u, 0u};
      if (row(j, g) >= there) continue;
#pragma unroll
      for (int c = 0; c < Elem<F32>::COLS; ++c) {
        if (c >= cols) continue;
        if constexpr (F32) v[j][c] = __float_as_uint(w[row(j, g) * stride + c]);
        else v[j][c / 2] |= (unsigned)w[row(j, g) * stride + c] << 16 * (c & 1);
      }
    }
  }
};

// 32 elements of a row of the pairs' operand, 8 per lane, as the slab's rows ask for them.
template <bool F32>
struct RowPart {
  u32x4 v[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const typename Elem<F32>::T* x, int g) {
    if constexpr (F32) {
#pragma unroll
      for (int u = 0; u < 2; ++u) v[u] = __builtin_bit_cast(u32x4, *reinterpret_cast<const f32x4_any*>(x + 16 * u + 4 * g));
    } else {
      v[0] = *reinterpret_cast<const u32x4_any*>(x + 8 * g);
    }
  }
  __device__ __forceinline__ void load_some(const typename Elem<F32>::T* x, int g, int there) {
    zero();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int k = F32 ? 16 * (e / 4) + 4 * g + e % 4 : 8 * g + e;
      if (k >= there) continue;
      if constexpr (F32) v[e / 4][e % 4] = __float_as_uint(x[k]);
      else v[0][e / 2] |= (unsigned)x[k] << 16 * (e & 1);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (auto& u : v) u = u32x4{0u, 0u, 0u, 0u};
  }
};

// acc[i]: tile of 16 columns (columns COLS a + i of the block, a = 0 .. 15) x 16 pairs.
template <bool F32>
struct Acc {
  f32x4 v[Elem<F32>::COLS];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (auto& u : v) u = f32x4{0.f, 0.f, 0.f, 0.f};
  }
};
template <bool F32, int NT>
__device__ __forceinline__ void multiply(const Slab<F32>& w, const RowPart<F32> (&x)[NT], Acc<F32> (&acc)[NT]) {
  if constexpr (F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const unsigned a = w.v[j][i], b = x[t].v[j / 4][j % 4];
          acc[t].v[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), acc[t].v[i], 0, 0, 0);
        }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u32x4 a;
#pragma unroll
      for (int q = 0; q < 4; ++q)                // column i of rows 2 q and 2 q + 1
        a[q] = __builtin_amdgcn_perm(w.v[2 * q + 1][i / 2], w.v[2 * q][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        acc[t].v[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, x[t].v[0]), acc[t].v[i], 0, 0, 0);
    }
  }
}

// Block: (run of the summed axis, tile of columns, slot).  NT tiles of pairs at a time.
template <bool F32, int MATS, int NT>
__device__ __forceinline__ void product_tiles(const LayerPairs& p, const LayerProduct& g, const LayerRows& rows, const typename Elem<F32>::T* const (&w)[MATS],
                                              const long long (&stride)[MATS], int run, long long col0, const int* list, int here, int act,
                                              void* out, float* lds) {
  using E = Elem<F32>;
  using T = typename E::T;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, a = lane & 15, q = lane >> 4;
  // a lane's columns end with the matrix at the latest: the last ones are then computed twice, alike
  long long col = col0 + E::COLS * a;
  const int cols = g.n < E::COLS ? (int)g.n : E::COLS;
  if (col > g.n - cols) col = g.n - cols;
  const long long k0 = (long long)run * g.run, k1 = k0 + g.run < g.k ? k0 + g.run : g.k;
  const T* x[NT];
  bool there[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    there[t] = t * kTile + a < here;
    x[t] = static_cast<const T*>(rows.x) + (long long)(list[there[t] ? t * kTile + a : 0] / rows.per) * rows.stride;
  }
  Acc<F32> acc[MATS][NT];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[m][t].zero();
  Slab<F32> s[MATS];
  RowPart<F32> r[NT];
  auto load = [&](long long k) {
#pragma unroll
    for (int m = 0; m < MATS; ++m) s[m].load(w[m] + k * stride[m] + col, stride[m], q);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      r[t].load(x[t] + k, q);
      if (!there[t]) r[t].zero();
    }
  };
  auto take = [&]() {
#pragma unroll
    for (int m = 0; m < MATS; ++m) multiply<F32, NT>(s[m], r, acc[m]);
  };
  constexpr int kStep = kLayerRows * kLayerWaves;
  long long k = k0 + wave * kLayerRows;
  if (cols == E::COLS)
    for (; k + kLayerRows <= k1; k += kStep) {
      load(k);
      take();
    }
  for (; k < k1; k += kStep) {                   // the last rows, or a matrix of a few columns
    const int left = k1 - k < kLayerRows ? (int)(k1 - k) : kLayerRows;
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      if (cols == E::COLS) s[m].load_some(w[m] + k * stride[m] + col, stride[m], q, left);
      else s[m].load_few(w[m] + k * stride[m] + col, stride[m], q, left, cols);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      r[t].zero();
      if (there[t]) r[t].load_some(x[t] + k, q, left);
    }
    take();
  }
  // the waves' sums through LDS, [wave][pair][column]; then a thread has a pair's COLS neighbouring columns
  constexpr int kColumns = 16 * E::COLS, kPitch = kColumns + 4;
  const int pair = threadIdx.x >> 4, chunk = threadIdx.x & 15;
  long long at = col0 + E::COLS * chunk;
  if (at > g.n - cols) at = g.n - cols;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float sum[MATS][E::COLS];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      __syncthreads();
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < E::COLS; ++i) lds[(wave * 16 + a) * kPitch + E::COLS * (4 * q + u) + i] = acc[m][t].v[i][u];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < E::COLS; ++i) {
        float x0 = lds[pair * kPitch + E::COLS * chunk + i];
#pragma unroll
        for (int v = 1; v < kLayerWaves; ++v) x0 += lds[(v * 16 + pair) * kPitch + E::COLS * chunk + i];
        sum[m][i] = x0;
      }
    }
    if (t * kTile + pair >= here) continue;
    const long long id = list[t * kTile + pair];
    if (act >= 0) {
      T* to = static_cast<T*>(out) + id * g.n + at;
#pragma unroll
      for (int i = 0; i < E::COLS; ++i) {
        if (i >= cols) continue;
        const float h = MATS == 2 ? activate(act, sum[MATS - 1][i]) * sum[0][i] : activate(act, sum[0][i]);
        if constexpr (F32) to[i] = h;
        else to[i] = (u16)(pack_bf16(h, 0.f) & 0xffffu);
      }
    } else {
#pragma unroll
      for (int m = 0; m < MATS; ++m) {
        float* to = static_cast<float*>(out) + (((long long)run * p.pairs + id) * MATS + m) * g.n + at;
#pragma unroll
        for (int i = 0; i < E::COLS; ++i)
          if (i < cols) to[i] = sum[m][i];
      }
    }
  }
}

template <bool F32, int MATS>
__global__ __launch_bounds__(256) void layer_product_kernel(LayerPairs p, LayerProduct g, LayerRows rows, LayerMatrix w, LayerMatrix gate, int act,
                                                            void* __restrict__ out) {
  using T = typename Elem<F32>::T;
  __shared__ float lds[kLayerWaves * 16 * (16 * Elem<F32>::COLS + 4)];
  __shared__ int list[2 * kTile];
  __shared__ int counts[4];
  int b = blockIdx.x;
  const int run = b % g.runs;
  b /= g.runs;
  const int tile = b % g.tiles, slot = b / g.tiles;
  const int e = p.slot_is_pair ? expert_of(p, slot) : slot;
  if (e < 0) return;
  const int all = find_pairs(p, e, 0, 2 * kTile, list, counts);
  if (all == 0 || (p.slot_is_pair && list[0] != slot)) return;       // nobody's, or another slot's
  const T* base[MATS];
  long long stride[MATS];
  base[0] = static_cast<const T*>(w.w) + e * w.expert_stride;
  stride[0] = w.row_stride;
  if constexpr (MATS == 2) {
    base[1] = static_cast<const T*>(gate.w) + e * gate.expert_stride;
    stride[1] = gate.row_stride;
  }
  const long long col0 = (long long)tile * (16 * Elem<F32>::COLS);
  for (int first = 0; first < all; first += 2 * kTile) {
    if (first) {
      __syncthreads();
      find_pairs(p, e, first, 2 * kTile, list, counts);
    }
    const int here = all - first < 2 * kTile ? all - first : 2 * kTile;
    if (here <= kTile) product_tiles<F32, MATS, 1>(p, g, rows, base, stride, run, col0, list, here, act, out, lds);
    else product_tiles<F32, MATS, 2>(p, g, rows, base, stride, run, col0, list, here, act, out, lds);
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void layer_act_kernel(LayerPairs p, int runs, long long n, int gated, int act, const float* __restrict__ part,
                                                        void* __restrict__ inner) {
  const long long spans = (n + 255) / 256, pair = blockIdx.x / spans, c = blockIdx.x % spans * 256 + threadIdx.x;
  if (c >= n || expert_of(p, (int)pair) < 0) return;
  const int mats = gated ? 2 : 1;
  float up = 0.f, lead = 0.f;
  for (int r = 0; r < runs; ++r) {
    const float* at = part + (((long long)r * p.pairs + pair) * mats) * n + c;
    up += at[0];
    if (gated) lead += at[n];
  }
  const float h = gated ? activate(act, lead) * up : activate(act, up);
  if constexpr (F32) static_cast<float*>(inner)[pair * n + c] = h;
  else static_cast<u16*>(inner)[pair * n + c] = (u16)(pack_bf16(h, 0.f) & 0xffffu);
}

template <bool F32>
__global__ __launch_bounds__(256) void layer_join_kernel(LayerPairs p, int runs, long long n, const float* __restrict__ rows, const float* __restrict__ weights,
                                                         void* __restrict__ out) {
  const long long spans = (n + 255) / 256, token = blockIdx.x / spans, c = blockIdx.x % spans * 256 + threadIdx.x;
  if (c >= n) return;
  float sum = 0.f;
  for (int j = 0; j < p.top; ++j) {
    const int pair = (int)token * p.top + j;
    if (expert_of(p, pair) < 0) continue;
    float y = 0.f;
    for (int r = 0; r < runs; ++r) y += rows[((long long)r * p.pairs + pair) * n + c];
    sum = fmaf(weights ? weights[pair] : 1.f, y, sum);
  }
  if constexpr (F32) static_cast<float*>(out)[token * n + c] = sum;
  else static_cast<u16*>(out)[token * n + c] = (u16)(pack_bf16(sum, 0.f) & 0xffffu);
}

}  // namespace

hipError_t launch_layer_product(const LayerPairs& p, const LayerProduct& g, const LayerRows& x, const LayerMatrix& w, const LayerMatrix* gate, bool f32,
                                int act, void* out, hipStream_t s) {
  const unsigned blocks = (unsigned)((long long)p.slots * g.tiles * g.runs);
  const LayerMatrix none{};
  auto go = [&](auto kernel) {
    kernel<<<blocks, 256, 0, s>>>(p, g, x, w, gate ? *gate : none, act, out);
    return hipGetLastError();
  };
  if (gate) return f32 ? go(layer_product_kernel<true, 2>) : go(layer_product_kernel<false, 2>);
  return f32 ? go(layer_product_kernel<true, 1>) : go(layer_product_kernel<false, 1>);
}

hipError_t launch_layer_act(const LayerPairs& p, int runs, long long n, bool gated, bool f32, int act, const float* part, void* inner, hipStream_t s) {
  const unsigned blocks = (unsigned)((n + 255) / 256 * p.pairs);
  if (f32) layer_act_kernel<true><<<blocks, 256, 0, s>>>(p, runs, n, gated, act, part, inner);
  else layer_act_kernel<false><<<blocks, 256, 0, s>>>(p, runs, n, gated, act, part, inner);
  return hipGetLastError();
}

hipError_t launch_layer_join(const LayerPairs& p, int runs, long long n, bool f32, const float* rows, const float* weights, void* out, hipStream_t s) {
  const unsigned blocks = (unsigned)((n + 255) / 256 * (p.pairs / p.top));
  if (f32) layer_join_kernel<true><<<blocks, 256, 0, s>>>(p, runs, n, rows, weights, out);
  else layer_join_kernel<false><<<blocks, 256, 0, s>>>(p, runs, n, rows, weights, out);
  return hipGetLastError();
}

}  // namespace muon
