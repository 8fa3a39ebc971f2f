// A mixture's layer on a few tokens: out_t = sum_j w_tj  h_tj Down_e,  h_tj = act(x_t Gate_e) * (x_t Up_e)  (no gate: act(x_t Up_e)),  e = expert of (t, j).
//
// Bound by memory: each chosen expert's matrices are read once for up to 32 of its pairs, again for each 32 more, and are all there is to read.  A wave
// multiplies 32 rows of a matrix at a time, straight from memory to registers: its lanes hold 8 (fp32: 4) neighbouring columns of 8 rows
// each, so that every load takes 256 bytes of a row, and the matrix instruction's own freedom does the rest: the order in which a sum over
// rows is taken and the columns that a tile of 16 is made of are free, so 8 x 8 blocks are transposed within a lane's registers (32 byte
// permutes for 64 elements), no LDS, no shuffles.  Tokens are the instruction's other 16 columns; an expert with more of them takes a second tile of 16.
//
// In bf16 h is rounded to bf16, as the operand of an instruction that takes nothing wider; outputs are off by 2.3e-3 of their norm, of which their own
// rounding is 1.7e-3.  Sums, their joins and the activation are fp32.
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

constexpr int kRoom = 2 * kTile;                 // pairs that a block takes at a time

// Pairs of expert e numbered [base, base + kRoom) into the wave's list, in their order; the number of all its pairs is returned.  By the whole
// block of THREADS threads; counts: an int of LDS per wave.
template <int THREADS>
__device__ __forceinline__ int find_pairs(const LayerPairs& p, int e, int base, int (*lists)[kRoom], int* counts) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (p.pairs <= 64) {                           // every wave for itself, without a barrier, which would wait for the loads on their way
    const unsigned long long ballot = __ballot(lane < p.pairs && expert_of(p, lane) == e);
    const int rank = __popcll(ballot & ((1ull << lane) - 1)) - base;
    if ((ballot >> lane & 1) && rank >= 0 && rank < kRoom) lists[wave][rank] = lane;
    return __popcll(ballot);
  }
  int seen = 0;
  for (int at = 0; at < p.pairs; at += THREADS) {
    const int i = at + threadIdx.x;
    const bool mine = i < p.pairs && expert_of(p, i) == e;
    const unsigned long long ballot = __ballot(mine);
    __syncthreads();                             // (the counts of the round before are read)
    if (lane == 0) counts[wave] = __popcll(ballot);
    __syncthreads();
    int before = seen;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) before += counts[w];
      seen += counts[w];
    }
    const int rank = before + __popcll(ballot & ((1ull << lane) - 1)) - base;
    if (mine && rank >= 0 && rank < kRoom)
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) lists[w][rank] = i;
  }
  __syncthreads();
  return seen;
}

// (a comparison, not the maximum instruction, which would make a NaN 0)
__device__ __forceinline__ float activate(int act, float z) { return act == 0 ? z / (1.f + expf(-z)) : z < 0.f ? 0.f : z; }

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

// 32 rows of a matrix: 8 accesses of 16 bytes per lane.  Row of access j: bf16 8 g + j, fp32 16 (j / 4) + 4 g + j % 4, with g = lane / 16.  `at` is the
// same for the whole wave, `lane` the lane's own offset in bytes (of its first row and column): scalar addresses, one register per lane.
template <bool F32>
struct Slab {
  u32x4 v[8];
  static constexpr int kOwn = F32 ? 4 : 8;       // rows from a group of lanes to the next
  static __device__ __forceinline__ constexpr int common(int j) { return F32 ? 16 * (j / 4) + j % 4 : j; }
  __device__ __forceinline__ void load(const char* at, long long stride, unsigned lane) {
    // (else the compiler adds the lane's offset to a base outside the loop, and every row has an address of two registers per lane)
    asm volatile("" : "+v"(lane));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const u32x4_any*>(at + common(j) * stride + lane);
  }
  // the same of `cols` columns and of rows [0, there) only; the others are zero
  __device__ __forceinline__ void load_some(const char* at, long long stride, unsigned lane, int g, int there, int cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = u32x4{0u, 0u, 0u, 0u};
      if (common(j) + kOwn * g >= there) continue;
      const char* p = at + common(j) * stride + lane;
      if (cols == Elem<F32>::COLS) {
        v[j] = *reinterpret_cast<const u32x4_any*>(p);
        continue;
      }
#pragma unroll
      for (int c = 0; c < Elem<F32>::COLS; ++c) {
        if (c >= cols) continue;
        if constexpr (F32) v[j][c] = reinterpret_cast<const unsigned*>(p)[c];
        else v[j][c / 2] |= (unsigned)reinterpret_cast<const u16*>(p)[c] << 16 * (c & 1);
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

// A wave's part of a product: columns [col0, ..) and rows [k0, k1) of one expert's matrix, 32 rows at a time, every fourth of them.
template <bool F32>
struct Part {
  static constexpr int COLS = Elem<F32>::COLS, kStep = kLayerRows * kLayerWaves;
  const char* w;                                 // row 0 of the expert's matrix
  long long stride;                              // bytes
  unsigned own;                                  // bytes from a row of the wave's to the lane's columns in its own first row
  long long k0, k1;
  int cols, wave, lane;                          // wave: of those that share the matrix

  __device__ __forceinline__ bool whole(long long k) const { return cols == COLS && k + kLayerRows <= k1; }
  __device__ __forceinline__ long long first_row() const { return k0 + wave * kLayerRows; }
  __device__ __forceinline__ void load(long long k, Slab<F32>& s) const { s.load(w + k * stride, stride, own); }
  __device__ __forceinline__ void load_rest(long long k, Slab<F32>& s) const {
    s.load_some(w + k * stride, stride, own, lane >> 4, k1 - k < kLayerRows ? (int)(k1 - k) : kLayerRows, cols);
  }
};

// The part for NT tiles of pairs.  STAGED: the pairs' operand lies in LDS, [pair][row - k0] at a pitch of `staged` elements, zeros behind k1.
// first: the wave's first rows, already loaded where `loaded`.
template <bool F32, int NT, bool STAGED>
__device__ __forceinline__ void multiply_part(const Part<F32>& part, const LayerRows& rows, const int* list, int here, const unsigned char* lds, int staged,
                                              Slab<F32>& first, bool loaded, Acc<F32> (&acc)[NT]) {
  using T = typename Elem<F32>::T;
  const int a = part.lane & 15, q = part.lane >> 4;
  const T* x[NT];
  bool there[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    there[t] = t * kTile + a < here;
    const int at = there[t] ? t * kTile + a : 0;
    if constexpr (STAGED) x[t] = reinterpret_cast<const T*>(lds) + at * staged - part.k0;
    else x[t] = static_cast<const T*>(rows.x) + (long long)(list[at] / rows.per) * rows.stride;
    acc[t].zero();
  }
  const auto load_rows = [&](long long k, RowPart<F32> (&r)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) r[t].load(x[t] + k, q);
  };
  const auto take = [&](const Slab<F32>& s, RowPart<F32> (&r)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (!there[t]) r[t].zero();
    multiply<F32, NT>(s, r, acc);
  };
  // 32 rows are multiplied while the next 32 are on their way
  long long k = part.first_row();
  RowPart<F32> r0[NT], r1[NT];
  if (part.whole(k)) {
    Slab<F32> second;
    if (!loaded) part.load(k, first);
    load_rows(k, r0);
    for (;;) {
      const long long next = k + part.kStep, after = next + part.kStep;
      const bool more = part.whole(next);
      if (more) {
        part.load(next, second);
        load_rows(next, r1);
      }
      take(first, r0);
      k = next;
      if (!more) break;
      const bool again = part.whole(after);
      if (again) {
        part.load(after, first);
        load_rows(after, r0);
      }
      take(second, r1);
      k = after;
      if (!again) break;
    }
  }
  for (; k < part.k1; k += part.kStep) {         // the last rows, or a matrix of a few columns
    part.load_rest(k, first);
    const int left = part.k1 - k < kLayerRows ? (int)(part.k1 - k) : kLayerRows;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if constexpr (STAGED) r0[t].load(x[t] + k, q);
      else r0[t].load_some(x[t] + k, q, left);
    }
    take(first, r0);
  }
}

// The waves' sums through LDS, [wave][pair][column]; then a thread of the first 256 has a pair's COLS neighbouring columns, of both matrices.
template <bool F32, int MATS, int NT>
__device__ __forceinline__ void store_tiles(const LayerPairs& p, const Part<F32>& part, const Acc<F32> (&acc)[NT], long long col0, long long n, int run,
                                            int apart, int matrix, const int* list, int here, int act, void* out, unsigned char* lds) {
  using T = typename Elem<F32>::T;
  constexpr int COLS = Elem<F32>::COLS, kPitch = 16 * COLS + 4, kWaves = kLayerWaves * MATS;
  float* sums = reinterpret_cast<float*>(lds);
  const int wave = threadIdx.x >> 6, a = part.lane & 15, q = part.lane >> 4, pair = threadIdx.x >> 4, chunk = threadIdx.x & 15;
  long long at = col0 + COLS * chunk;
  if (at > n - part.cols) at = n - part.cols;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < COLS; ++i) sums[(wave * 16 + a) * kPitch + COLS * (4 * q + u) + i] = acc[t].v[i][u];
    __syncthreads();
    if (kWaves > 4 && threadIdx.x >= 256) continue;
    if (t * kTile + pair >= here) continue;
    float sum[MATS][COLS];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        const float* of = sums + (m * kLayerWaves * 16 + pair) * kPitch + COLS * chunk + i;
        float x = of[0];
#pragma unroll
        for (int v = 1; v < kLayerWaves; ++v) x += of[v * 16 * kPitch];
        sum[m][i] = x;
      }
    const long long id = list[t * kTile + pair];
    if (act >= 0) {
      T* to = static_cast<T*>(out) + id * n + at;
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        if (i >= part.cols) continue;
        const float h = MATS == 2 ? activate(act, sum[MATS - 1][i]) * sum[0][i] : activate(act, sum[0][i]);
        if constexpr (F32) to[i] = h;
        else to[i] = (u16)(pack_bf16(h, 0.f) & 0xffffu);
      }
    } else {
#pragma unroll
      for (int m = 0; m < MATS; ++m) {
        float* to = static_cast<float*>(out) + (((long long)run * p.pairs + id) * (MATS * apart) + (MATS == 1 ? matrix : m)) * n + at;
#pragma unroll
        for (int i = 0; i < COLS; ++i)
          if (i < part.cols) to[i] = sum[m][i];
      }
    }
  }
}

// The operand of the second product from the sums of the first one's runs, activated, into LDS.
template <bool F32>
__device__ __forceinline__ void stage(const LayerPairs& p, const LayerSums& from, long long k0, long long k1, int staged, const int* list, int here,
                                      unsigned char* lds) {
  using T = typename Elem<F32>::T;
  for (int i = threadIdx.x; i < here * staged; i += 256) {
    const int pair = i / staged;
    const long long k = k0 + i % staged;
    float h = 0.f;
    if (k < k1) {
      const float* at = from.part + (long long)list[pair] * from.mats * from.n + k;
      const long long run = (long long)p.pairs * from.mats * from.n;
      float up = 0.f, lead = 0.f;
#pragma unroll 8
      for (int r = 0; r < from.runs; ++r) {
        up += at[r * run];
        if (from.mats == 2) lead += at[r * run + from.n];
      }
      h = from.mats == 2 ? activate(from.act, lead) * up : activate(from.act, up);
    }
    if constexpr (F32) reinterpret_cast<T*>(lds)[i] = h;
    else reinterpret_cast<T*>(lds)[i] = (u16)(pack_bf16(h, 0.f) & 0xffffu);
  }
  __syncthreads();
}

// Block: (matrix, run of the summed axis, tile of columns) and slot; four waves to a matrix, MATS matrices to a block.  NT: tiles of pairs that there may
// be at a time.
template <bool F32, int MATS, int NT, bool STAGED>
__global__ __launch_bounds__(256 * MATS, 2) void layer_product_kernel(LayerPairs p, LayerProduct g, LayerRows rows, LayerMatrix w, LayerMatrix gate, LayerSums from,
                                                                      int act, void* __restrict__ out) {
  using T = typename Elem<F32>::T;
  using E = Elem<F32>;
  constexpr int kThreads = 256 * MATS, kSums = kLayerWaves * MATS * 16 * (16 * E::COLS + 4) * 4;
  __shared__ __align__(16) unsigned char lds[STAGED && kLayerStage > kSums ? kLayerStage : kSums];
  __shared__ int lists[kThreads / 64][kRoom];
  __shared__ int counts[kThreads / 64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b = blockIdx.x;
  const int apart = MATS == 1 ? g.mats : 1, matrix = MATS == 1 ? b % apart : wave / kLayerWaves;
  b /= apart;
  const int run = b % g.runs, tile = b / g.runs, slot = blockIdx.y;
  const int e = __builtin_amdgcn_readfirstlane(p.slot_is_pair ? expert_of(p, slot) : slot);
  if (e < 0) return;
  const long long col0 = (long long)tile * (16 * E::COLS);
  Part<F32> part;
  part.wave = wave % kLayerWaves;
  part.lane = threadIdx.x & 63;
  part.k0 = (long long)run * g.run;
  part.k1 = part.k0 + g.run < g.k ? part.k0 + g.run : g.k;
  // a lane's columns end with the matrix at the latest: the last ones are then computed twice, alike
  part.cols = g.n < E::COLS ? (int)g.n : E::COLS;
  long long col = col0 + E::COLS * (part.lane & 15);
  if (col > g.n - part.cols) col = g.n - part.cols;
  const LayerMatrix& m = matrix ? gate : w;
  part.w = reinterpret_cast<const char*>(static_cast<const T*>(m.w) + e * m.expert_stride);
  part.stride = m.row_stride * (long long)sizeof(T);
  part.own = (unsigned)((Slab<F32>::kOwn * (part.lane >> 4) * m.row_stride + col) * (long long)sizeof(T));
  // where a slot stands for a pair it has tokens, so that the first rows can be on their way while they are looked up
  Slab<F32> first;
  const bool ahead = p.slot_is_pair && part.whole(part.first_row());
  if (ahead) part.load(part.first_row(), first);
  const int* list = lists[wave];
  const int all = find_pairs<kThreads>(p, e, 0, lists, counts);
  if (all == 0 || (p.slot_is_pair && list[0] != slot)) return;       // nobody's, or another slot's
  const int staged = (int)((part.k1 - part.k0 + kLayerRows - 1) / kLayerRows * kLayerRows);
  for (int at = 0; at < all; at += kRoom) {
    if (at) {
      __syncthreads();
      find_pairs<kThreads>(p, e, at, lists, counts);
    }
    const int here = all - at < kRoom ? all - at : kRoom;
    if constexpr (STAGED) stage<F32>(p, from, part.k0, part.k1, staged, list, here, lds);
    const auto tiles = [&](auto count) {
      constexpr int N = decltype(count)::value;
      Acc<F32> acc[N];
      multiply_part<F32, N, STAGED>(part, rows, list, here, lds, staged, first, ahead && at == 0, acc);
      store_tiles<F32, MATS, N>(p, part, acc, col0, g.n, run, apart, matrix, list, here, act, out, lds);
    };
    if (NT == 1 || here <= kTile) tiles(std::integral_constant<int, 1>{});
    else tiles(std::integral_constant<int, NT>{});
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void layer_act_kernel(LayerPairs p, int runs, long long n, int gated, int act, const float* __restrict__ part,
                                                        void* __restrict__ inner) {
  const long long pair = blockIdx.y, c = blockIdx.x * 256ll + threadIdx.x;
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

// kJoinColumns columns of a token per block: four neighbouring ones per thread, the token's terms over eight groups of threads, joined in LDS.
template <bool F32>
__global__ __launch_bounds__(256) void layer_join_kernel(LayerPairs p, int runs, long long n, const float* __restrict__ rows, const float* __restrict__ weights,
                                                         void* __restrict__ out) {
  __shared__ f32x4 parts[8][32];
  const long long token = blockIdx.y;
  const int quad = threadIdx.x & 31, group = threadIdx.x >> 5, terms = p.top * runs;
  const long long c = blockIdx.x * (long long)kJoinColumns + 4 * quad;
  const int count = c >= n ? 0 : n - c < 4 ? (int)(n - c) : 4;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = group; i < terms; i += 8) {
    const int j = i / runs, pair = (int)token * p.top + j;
    const bool there = expert_of(p, pair) >= 0;
    const float w = !there ? 0.f : weights ? weights[pair] : 1.f;
    const float* at = rows + ((long long)(i - j * runs) * p.pairs + pair) * n + c;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (there) {
      if (count == 4) {
        y = *reinterpret_cast<const f32x4_any*>(at);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < count) y[e] = at[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(w, y[e], sum[e]);
  }
  parts[group][quad] = sum;
  __syncthreads();
  if (threadIdx.x >= kJoinColumns) return;
  const long long at = blockIdx.x * (long long)kJoinColumns + threadIdx.x;
  if (at >= n) return;
  const float* of = reinterpret_cast<const float*>(parts) + threadIdx.x;
  float x = of[0];
#pragma unroll
  for (int g = 1; g < 8; ++g) x += of[g * kJoinColumns];
  if constexpr (F32) static_cast<float*>(out)[token * n + at] = x;
  else static_cast<u16*>(out)[token * n + at] = (u16)(pack_bf16(x, 0.f) & 0xffffu);
}

dim3 blocks_of(const LayerGrid& g) { return dim3((unsigned)g.x, (unsigned)g.y); }

}  // namespace

hipError_t launch_layer_product(const LayerPairs& p, const LayerProduct& g, const LayerRows& x, const LayerMatrix& w, const LayerMatrix* gate,
                                const LayerSums* from, bool f32, int act, void* out, hipStream_t s) {
  const bool together = gate && g.mats == 1;
  const LayerGrid grid = layer_product_grid(g, p.slots, together);
  const LayerMatrix none{};
  const LayerSums rows{};
  auto go = [&](auto kernel) {
    kernel<<<blocks_of(grid), grid.threads, 0, s>>>(p, g, x, w, gate ? *gate : none, from ? *from : rows, act, out);
    return hipGetLastError();
  };
#define MUON_LAYER_CASE(NT)                                                                                            \
  if (together) return f32 ? go(layer_product_kernel<true, 2, NT, false>) : go(layer_product_kernel<false, 2, NT, false>);     \
  if (from) return f32 ? go(layer_product_kernel<true, 1, NT, true>) : go(layer_product_kernel<false, 1, NT, true>);           \
  return f32 ? go(layer_product_kernel<true, 1, NT, false>) : go(layer_product_kernel<false, 1, NT, false>)
  if (p.pairs <= 16) {
    MUON_LAYER_CASE(1);
  }
  MUON_LAYER_CASE(2);
#undef MUON_LAYER_CASE
}

hipError_t launch_layer_act(const LayerPairs& p, int runs, long long n, bool gated, bool f32, int act, const float* part, void* inner, hipStream_t s) {
  const LayerGrid grid = layer_act_grid(n, p.pairs);
  if (f32) layer_act_kernel<true><<<blocks_of(grid), grid.threads, 0, s>>>(p, runs, n, gated, act, part, inner);
  else layer_act_kernel<false><<<blocks_of(grid), grid.threads, 0, s>>>(p, runs, n, gated, act, part, inner);
  return hipGetLastError();
}

hipError_t launch_layer_join(const LayerPairs& p, int runs, long long n, bool f32, const float* rows, const float* weights, void* out, hipStream_t s) {
  const LayerGrid grid = layer_join_grid(n, p.pairs / p.top);
  if (f32) layer_join_kernel<true><<<blocks_of(grid), grid.threads, 0, s>>>(p, runs, n, rows, weights, out);
  else layer_join_kernel<false><<<blocks_of(grid), grid.threads, 0, s>>>(p, runs, n, rows, weights, out);
  return hipGetLastError();
}

}  // namespace muon
