// Softmax losses of a language model's head from hidden states H [T, D] and the head's weight W [V, D], logits never kept whole.
//
//   z = H W^T / tau     lse_t = log sum_v exp z_tv     dz_tv = g_t tau (p_tv - q_tv),  p = exp(z - lse)     dH = dz W     dW = dz^T H
//
// q is the target: one entry of 1 (cross entropy) or the softmax of a teacher's few best logits.  The logits' product runs over tiles of
// vocabulary x tokens whose epilogue leaves, per block of the vocabulary and token, a bias and the sum of 2^(z log2(e) + bias), and, for the
// gradient, these powers in f16.  Joining the blocks gives lse and loss; one pass scales the powers to dz in bf16, in place, and writes
// the target's few entries from logits computed in fp32 (p - q there cancels); two more products give the gradients.
#include <hip/hip_runtime.h>

#include <atomic>

#include "head_gemm.h"

namespace muon {
namespace {

using namespace head;

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

template <bool F32>
__global__ __launch_bounds__(256) void head_pack_kernel(const void* __restrict__ src, long long stride, long long n, long long width,
                                                        u16* __restrict__ dst, long long ld, long long plane) {
  const long long chunks = ld / 8;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n * chunks; i += gridDim.x * 256ll) {
    const long long row = i / chunks, c = (i - row * chunks) * 8;
    store_planes8<F32>(load_row8<F32>(src, row * stride, c, width), dst + row * ld + c, plane);
  }
}

// ---- targets ----
__device__ __forceinline__ long long index_at(const HeadTarget& t, long long i) {
  return t.index64 ? static_cast<const long long*>(t.index)[i] : (long long)static_cast<const int*>(t.index)[i];
}
__device__ __forceinline__ float teacher_at(const HeadTarget& t, long long i) {
  return t.logits_bf16 ? bf16_value(static_cast<const u16*>(t.logits)[i]) : static_cast<const float*>(t.logits)[i];
}
// Entry i is one: an index of the vocabulary whose teacher's logit is not -inf.
__device__ __forceinline__ bool entry_there(const HeadTarget& t, long long i, long long vocab) {
  const long long v = index_at(t, i);
  return v >= 0 && v < vocab && !(t.logits && teacher_at(t, i) == -INFINITY);
}
struct TokenState {
  bool some, beyond;        // has entries; has an index beyond the vocabulary
};
// By a whole wave.
__device__ __forceinline__ TokenState token_state(const HeadTarget& t, long long token, long long vocab) {
  bool some = false, beyond = false;
  for (int j = threadIdx.x & 63; j < t.top; j += 64) {
    some |= entry_there(t, token * t.top + j, vocab);
    beyond |= index_at(t, token * t.top + j) >= vocab;
  }
  return {__any(some) != 0, __any(beyond) != 0};
}
__device__ __forceinline__ float token_scale(const HeadTarget& t, long long token, TokenState state) {
  const float g = t.token_scale ? t.token_scale[token] : 1.f;
  return state.some && !state.beyond ? g : 0.f;
}

// <a, b> over `width` elements by a whole wave, in fp32.
template <bool F32>
__device__ __forceinline__ float row_dot(const void* a, long long a_at, const void* b, long long b_at, long long width) {
  float sum = 0.f;
  for (long long c = (threadIdx.x & 63) * 8; c < width; c += 512) {
    const Row8 x = load_row8<F32>(a, a_at, c, width), y = load_row8<F32>(b, b_at, c, width);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(x.v[e], y.v[e], sum);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
  return sum;
}

// One block per token.  Each wave takes every fourth entry: a dot product of two rows in fp32.  Bound by W's rows, which come in no order:
// 4096 tokens x 64 entries of width 2048 in bf16, 1.07 GB, 212 us (5.1 TB/s); one entry of 8192 tokens of width 4096, with the copy, 47 us.
template <bool F32>
__global__ __launch_bounds__(256) void head_entries_kernel(HeadTarget t, const void* __restrict__ hidden, long long hidden_stride,
                                                           const void* __restrict__ weight, long long weight_stride, long long vocab,
                                                           long long width, float* __restrict__ entry, u16* __restrict__ masked, long long ld,
                                                           long long plane, float* __restrict__ kept_scale) {
  const long long token = blockIdx.x, at = token * hidden_stride;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int j = wave; j < t.top; j += 4) {
    const long long v = index_at(t, token * t.top + j);
    float sum = 0.f;
    if (v >= 0 && v < vocab) sum = row_dot<F32>(hidden, at, weight, v * weight_stride, width);
    if (lane == 0) entry[token * t.top + j] = t.inv_tau * sum;
  }
  if (!masked && !kept_scale) return;
  const float g = token_scale(t, token, token_state(t, token, vocab));
  if (kept_scale && threadIdx.x == 0) kept_scale[token] = g;
  if (masked) {
    for (long long c = threadIdx.x * 8; c < ld; c += 2048) {
      Row8 r{};
      if (g != 0.f) r = load_row8<F32>(hidden, at, c, width);
      store_planes8<F32>(r, masked + token * ld + c, plane);
    }
  }
}

// ---- logits ----
// A block of statistics is 128 vocabulary entries: the rows of one wave in a tile of 256, of two in a tile of 128, which compare notes in
// LDS (the two have one grain, so that a launch may mix them).  A lane holds half of a wave's rows for each of its tokens.  Powers of two throughout: 2^(unit z + bias) is one multiply-add and one
// exponential, and as every power of a block carries the very bias that is stored, rounding the bias costs nothing.
// Bound by the matrix cores under the power limit (8192 x 131072 x 4096 bf16: 7.2 ms, 1.22 PFLOP/s, cores busy 70 % at 1.66 GHz), for short K by
// the epilogue: 3 us of a tile, 13 with the powers stored by all compute units at once (2048 x 32768 x 1024: 170 us, K's share 105).
template <int B, int S, bool PROB, bool F32>
__device__ __forceinline__ void logits_tile(const HeadOperand& weight, const HeadOperand& hidden, const HeadTiles& g, float unit, float2* stats,
                                            long long stats_pitch, void* prob, long long prob_pitch, long long row0, long long col0,
                                            unsigned char* smem) {
  using T = Tile<B, B, false, false, S>;
  T tile;
  tile.run(weight, hidden, row0, col0, g.k, g.pairs, 0, g.slabs_per_split, smem);
  const int fr = tile.lane & 31, fh = tile.lane >> 5;
  const long long v0 = row0 + tile.wm * T::WM;
  // rows of the wave's that there are; MASKED: not all of them
  const int there = (int)(weight.rows - v0 < T::WM ? weight.rows - v0 : T::WM);
  auto row = [&](int i, int v) { return 32 * i + 8 * (v / 4) + 4 * fh + v % 4; };
  if constexpr (PROB && F32) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const long long token = col0 + tile.wn * T::WN + 32 * j + fr;
      float* z = static_cast<float*>(prob) + token * prob_pitch + v0 + 4 * fh;
      if (token >= hidden.rows) continue;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = tile.acc[i][j][4 * q + e];
          *reinterpret_cast<f32x4*>(z + 32 * i + 8 * q) = x;
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  }
  float top[T::FN];
  auto find_top = [&](auto masked) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      top[j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < T::FM; ++i) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!decltype(masked)::value || row(i, v) < there) top[j] = fmaxf(top[j], tile.acc[i][j][v]);
        __builtin_amdgcn_sched_barrier(0);
      }
      top[j] = fmaxf(top[j], __shfl_xor(top[j], 32, 64));
    }
  };
  if (there == T::WM) find_top(std::false_type{});
  else find_top(std::true_type{});
  float* notes = reinterpret_cast<float*>(smem + T::kStage);          // behind the image
  if constexpr (B == 128) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j) notes[tile.wm * 128 + tile.wn * 64 + 32 * j + fr] = top[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::FN; ++j) top[j] = fmaxf(top[j], notes[(tile.wm ^ 1) * 128 + tile.wn * 64 + 32 * j + fr]);
  }
  float sums[T::FN];
  auto take_powers = [&](auto masked) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const float bias = kProbTop - (top[j] == -INFINITY ? 0.f : unit * top[j]);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = __builtin_amdgcn_exp2f(fmaf(unit, tile.acc[i][j][4 * q + e], bias));
            if (decltype(masked)::value && row(i, 4 * q + e) >= there) x[e] = 0.f;
            sum += x[e];
          }
          if constexpr (PROB && !F32) {
            tile.put(smem, i, j, q, u32x2{pack_f16(x[0], x[1]), pack_f16(x[2], x[3])});
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      sums[j] = sum + __shfl_xor(sum, 32, 64);
      if constexpr (B == 128) notes[256 + tile.wm * 128 + tile.wn * 64 + 32 * j + fr] = sums[j];
      top[j] = bias;
    }
  };
  if (there == T::WM) take_powers(std::false_type{});
  else take_powers(std::true_type{});
  if constexpr (B == 128 || (PROB && !F32)) __syncthreads();
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const int c = tile.wn * T::WN + 32 * j + fr;
    if constexpr (B == 128) sums[j] += notes[256 + (tile.wm ^ 1) * 128 + c];
    if (fh == 0 && (B == 256 || tile.wm == 0) && v0 < weight.rows && col0 + c < hidden.rows)
      stats[v0 / kHeadGrain * stats_pitch + col0 + c] = make_float2(top[j], sums[j]);
  }
  if constexpr (PROB && !F32) {
    tile.image_out(smem, [&](int c, int r, u32x4 v) {
      if (col0 + c < hidden.rows) *reinterpret_cast<u32x4*>(static_cast<u16*>(prob) + (col0 + c) * prob_pitch + row0 + r) = v;
    });
  }
}

// B x B tiles on a ring of S stages: 256 on two (with quarters on four), 128 on two, two blocks to a compute unit, or 128 on four.
template <int B, int S, bool PROB, bool F32>
__global__ __launch_bounds__(256, B == 128 && S == 2 ? 2 : 1) void head_logits_kernel(HeadOperand weight, HeadOperand hidden, HeadTiles g, float unit,
                                                                            float2* __restrict__ stats, long long stats_pitch,
                                                                            void* __restrict__ prob, long long prob_pitch) {
#if defined(__HIP_DEVICE_COMPILE__)            // (the host's pass knows no buffer descriptors)
  extern __shared__ __align__(16) unsigned char smem[];
  const TileAt at = tile_at(g);
  long long row0 = (long long)at.m * B, col0 = (long long)at.n * B;
  if (B == 128 || at.quarter < 0) {
    logits_tile<B, S, PROB, F32>(weight, hidden, g, unit, stats, stats_pitch, prob, prob_pitch, row0, col0, smem);
  } else if constexpr (B == 256) {
    row0 += 128 * (at.quarter >> 1);
    col0 += 128 * (at.quarter & 1);
    if (row0 < weight.rows && col0 < hidden.rows)
      logits_tile<128, 4, PROB, F32>(weight, hidden, g, unit, stats, stats_pitch, prob, prob_pitch, row0, col0, smem);
  }
#endif
}

// ---- join ----
__global__ __launch_bounds__(1024) void head_peak_kernel(const float* __restrict__ kept, long long tokens, float* __restrict__ peak) {
  __shared__ float waves[16];
  float top = 0.f;
  for (long long i = threadIdx.x; i < tokens; i += 1024) {
    const float g = fabsf(kept[i]);
    if (g < INFINITY) top = fmaxf(top, g);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) top = fmaxf(top, waves[w]);
    *peak = top > 0.f ? top : 1.f;
  }
}

// Where a piece has no more tokens than this, every block of the join looks through all its scales itself: a launch less.
constexpr long long kPeakInJoin = 16384;

// Bound by the chain of its loads (6.5 us for 16 tokens of 256 blocks with their entries' logits, 36 for 8192 of 1024).
// Sixteen tokens per block (a line of statistics), their blocks of the vocabulary over 64 threads each, eight loads at a time; then a wave
// per token for its entries, of which the first 64 are loaded at the start.
__global__ __launch_bounds__(1024) void head_join_kernel(HeadTarget t, float unit, const float* __restrict__ kept, float* __restrict__ peak,
                                                         const float2* __restrict__ stats, long long stats_pitch, long long blocks,
                                                         const float* __restrict__ entry, HeadRows rows, long long tokens, long long vocab,
                                                         float* __restrict__ loss, float* __restrict__ lse, float* __restrict__ value,
                                                         float* __restrict__ scale, float2* __restrict__ log2sum) {
  __shared__ float tops[64][17];
  __shared__ float sums[64][17];
  __shared__ float peaks[16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long tk = blockIdx.x * 16ll + wave;
  // this wave's token: entry `lane` of its target
  struct Entry {
    int v;                                       // -1: none
    float s, z;
  };
  auto load_entry = [&](int j, bool* beyond) -> Entry {
    Entry e{-1, -INFINITY, 0.f};
    if (tk >= tokens || j >= t.top) return e;
    const long long i = tk * t.top + j, v = index_at(t, i);
    if (v >= vocab) *beyond = true;
    if (v < 0 || v >= vocab) return e;
    e.s = t.logits ? teacher_at(t, i) : 0.f;
    if (entry) e.z = entry[i];
    if (!(e.s == -INFINITY)) e.v = (int)v;
    return e;
  };
  bool beyond = false;
  Entry mine = load_entry(lane, &beyond);
  float g = tk < tokens && t.token_scale ? t.token_scale[tk] : 1.f;
  float most = 0.f;
  if (kept)
    for (long long i = threadIdx.x; i < tokens; i += 1024) {
      const float x = fabsf(kept[i]);
      if (x < INFINITY) most = fmaxf(most, x);
    }

  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
  const long long token = blockIdx.x * 16ll + x, read = token < tokens ? token : tokens - 1;
  float top = -INFINITY, sum = 0.f;              // the sum is sum * 2^top
  float2 v[8];
  auto load_stats = [&](long long b0) {
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = b0 + 64 * u < blocks ? stats[(b0 + 64 * u) * stats_pitch + read] : make_float2(0.f, 0.f);
  };
  load_stats(y);
  if (!entry && tk < tokens) {                   // one entry, and nobody has made its logit
    const long long v = index_at(t, tk);
    if (v >= 0 && v < vocab)
      mine.z = t.inv_tau * (rows.f32 ? row_dot<true>(rows.hidden, tk * rows.hidden_stride, rows.weight, v * rows.weight_stride, rows.width)
                                     : row_dot<false>(rows.hidden, tk * rows.hidden_stride, rows.weight, v * rows.weight_stride, rows.width));
  }
  for (long long b0 = y; b0 < blocks; b0 += 64 * 8) {
    if (b0 != y) load_stats(b0);
    float here = top;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (v[u].y != 0.f) here = fmaxf(here, -v[u].x);
    const float shift = here == -INFINITY ? 0.f : here;
    sum *= __builtin_amdgcn_exp2f(top - shift);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (v[u].y != 0.f) sum += v[u].y * __builtin_amdgcn_exp2f(-v[u].x - shift);
    top = here;
  }
  tops[y][x] = top;
  sums[y][x] = sum;
  if (kept) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
    if (lane == 0) peaks[wave] = most;
  }
  __syncthreads();
  float largest = 1.f;
  if (kept) {
    most = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) most = fmaxf(most, peaks[w]);
    largest = most > 0.f ? most : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0) *peak = largest;
  } else if (peak) {
    largest = *peak;
  }
  if (tk >= tokens) return;
  // wave w: token w, lane: its thread's share
  const float share = tops[lane][wave];
  float all = share;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) all = fmaxf(all, __shfl_xor(all, off, 64));
  const float shift = all == -INFINITY ? 0.f : all;
  double part = (double)(sums[lane][wave] * __builtin_amdgcn_exp2f(share - shift));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) part += __shfl_xor(part, off, 64);
  const double y2 = (double)shift + log2(part), l = y2 * ((double)t.inv_tau / (double)unit);       // log2 and natural log of the sum

  bool some = mine.v >= 0;
  for (int j = lane + 64; j < t.top; j += 64) some |= load_entry(j, &beyond).v >= 0;
  some = __any(some) != 0;
  beyond = __any(beyond) != 0;
  if (!some || beyond) g = 0.f;
  const float r = g == 0.f ? 0.f : g / largest;
  if (lane == 0) {
    if (lse) lse[tk] = (float)l;
    if (value) {
      scale[tk] = r;
      const float hi = (float)y2;
      log2sum[tk] = make_float2(hi, (float)(y2 - (double)hi));
    }
  }
  double sum_loss = 0.0;
  // log p of an entry.  Its logit was summed in another order than the ones in l: what rounding leaves above 0 is cut off (NaN stays)
  auto log_p = [&](const Entry& e) {
    const double d = (double)e.z - l;
    return d > 0.0 ? 0.0 : d;
  };
  if (!t.logits) {
    if (lane == 0) {
      sum_loss = some ? -log_p(mine) : 0.0;
      if (value) value[tk] = r == 0.f ? 0.f : (float)((double)r * expm1(log_p(mine)));
    }
  } else if (some) {
    bool ignored = false;
    float best = mine.v >= 0 ? mine.s : -INFINITY;
    for (int j = lane + 64; j < t.top; j += 64) {
      const Entry e = load_entry(j, &ignored);
      if (e.v >= 0) best = fmaxf(best, e.s);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) best = fmaxf(best, __shfl_xor(best, off, 64));
    // the teacher's logits over tau, from the best one down, in double: a lowest finite logit stays an entry whatever tau
    auto behind = [&](const Entry& e) { return ((double)e.s - (double)best) * (double)t.inv_tau; };
    double mass = mine.v >= 0 ? exp(behind(mine)) : 0.0;
    for (int j = lane + 64; j < t.top; j += 64) {
      const Entry e = load_entry(j, &ignored);
      if (e.v >= 0) mass += exp(behind(e));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) mass += __shfl_xor(mass, off, 64);
    const double log_mass = log(mass);
    for (int j0 = 0; j0 < t.top; j0 += 64) {
      const int j = j0 + lane;
      const Entry e = j0 == 0 ? mine : load_entry(j, &ignored);
      const bool there = e.v >= 0;
      const double logp = log_p(e), logq = there ? behind(e) - log_mass : 0.0, own = there ? exp(logq) : 0.0;
      if (there) sum_loss += own * (logq - logp);
      if (value) {
        double q = 0.0;                          // of every entry with this index
        for (int k0 = 0; k0 < t.top; k0 += 64) {
          int vk = e.v;
          double qk = own;
          if (k0 != j0) {
            const Entry o = k0 == 0 ? mine : load_entry(k0 + lane, &ignored);
            vk = o.v;
            qk = o.v >= 0 ? exp(behind(o) - log_mass) : 0.0;
          }
          const int n = t.top - k0 < 64 ? t.top - k0 : 64;
          for (int w = 0; w < n; ++w) {
            const int vw = __shfl(vk, w, 64);
            const double qw = __shfl(qk, w, 64);
            if (vw == e.v) q += qw;
          }
        }
        if (j < t.top) value[tk * t.top + j] = there && r != 0.f ? (float)((double)r * (exp(logp) - q)) : 0.f;
      }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum_loss += __shfl_xor(sum_loss, off, 64);
  } else if (value) {
    for (int j = lane; j < t.top; j += 64) value[tk * t.top + j] = 0.f;
  }
  if (lane == 0) loss[tk] = beyond ? __builtin_nanf("") : (float)((double)t.tau * (double)t.tau * sum_loss);
}

// ---- dz ----
// Bound by HBM: 8192 x 131072 in bf16, 2 bytes in and 2 out, 721 us (6.0 TB/s); fp32, 4 in and 6 out, 34 us for 1000 x 20011 (5.9).
constexpr int kGradSpan = 4096;                  // vocabulary entries per block
template <bool F32>
__global__ __launch_bounds__(256) void head_grad_kernel(HeadTarget t, float unit, const float2* __restrict__ stats, long long stats_pitch,
                                                        const float2* __restrict__ log2sum, const float* __restrict__ value,
                                                        const float* __restrict__ scale, long long vocab, int spans,
                                                        const void* prob, long long pitch, u16* grad, long long plane) {
  const long long token = blockIdx.x / spans, v0 = (long long)(blockIdx.x % spans) * kGradSpan;
  const float g = scale[token];
  const float2 l = log2sum[token];
  const long long row = token * pitch;
  for (long long v = v0 + threadIdx.x * 8; v < v0 + kGradSpan && v < pitch; v += 2048) {
    Row8 r{};
    if (g != 0.f && v < vocab) {
      if constexpr (F32) {
        const f32x4* z = reinterpret_cast<const f32x4*>(static_cast<const float*>(prob) + row + v);     // (rows end on whole tiles)
        const f32x4 two[2] = {z[0], z[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = two[e / 4][e % 4];
          r.v[e] = v + e < vocab ? g * __builtin_amdgcn_exp2f(fmaf(unit, x, -l.x) - l.y) : 0.f;
        }
      } else {
        const u32x4 p = *reinterpret_cast<const u32x4*>(static_cast<const u16*>(prob) + row + v);
        const float f = g * __builtin_amdgcn_exp2f(-stats[v / kHeadGrain * stats_pitch + token].x - l.x - l.y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned pair = p[e / 2];        // (a bit cast of the vector's element itself would take its first)
          const f16x2 two = __builtin_bit_cast(f16x2, pair);
          r.v[e] = v + e < vocab ? f * (float)two[e & 1] : 0.f;
        }
      }
    }
    store_planes8<F32>(r, grad + row + v, plane);
  }
  if (g == 0.f) return;
  __syncthreads();                               // the entries go over what this block wrote
  for (int j = threadIdx.x; j < t.top; j += 256) {
    const long long i = token * t.top + j;
    const long long v = index_at(t, i);
    if (v < v0 || v >= v0 + kGradSpan || !entry_there(t, i, vocab)) continue;
    float x = value[i];
#pragma unroll
    for (int q = 0; q < (F32 ? 3 : 1); ++q) {
      const u16 b = bf16_bits(x);
      grad[q * plane + row + v] = b;
      x -= bf16_value(b);
    }
  }
}

// ---- gradients ----
// L (hidden states or weight) is read K-major, so that a lane's four accumulator rows are four neighbours of the result's row; so is dz for
// the weight's gradient: nothing is transposed in memory.  Bound by the matrix cores under the power limit: 8192 x 131072 x 4096 bf16
// 6.5 ms (hidden, 1.35 PFLOP/s, cores busy 80 % at 1.61 GHz) and 6.7 (weight), the library's product 6.5 and 7.6.
// Four neighbours of the results, or as many of them as there are.
__device__ __forceinline__ void finish_out4(const HeadOut& o, long long at, f32x4 x, int count) {
  float* to = o.keep ? o.sum : o.f32 ? static_cast<float*>(o.out) : nullptr;
  if (count >= 4) {
    if (o.add) x += *reinterpret_cast<const f32x4_any*>(o.sum + at);
    if (to) *reinterpret_cast<f32x4_any*>(to + at) = x;
    else *reinterpret_cast<u32x2_any*>(static_cast<u16*>(o.out) + at) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e >= count) continue;
    const float y = o.add ? x[e] + o.sum[at + e] : x[e];
    if (to) to[at + e] = y;
    else static_cast<u16*>(o.out)[at + e] = bf16_bits(y);
  }
}

// fp32 results, parts of a sum, or both: four elements per lane and store.
template <typename T>
__device__ __forceinline__ void store_parts(const T& tile, const HeadOperand& l, const HeadOperand& r, const HeadTiles& g, const HeadOut& out, float scale,
                                            int split, long long row0, long long col0) {
  const int fr = tile.lane & 31, fh = tile.lane >> 5;
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const long long n = col0 + tile.wn * T::WN + 32 * j + fr;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const long long m = row0 + tile.wm * T::WM + 32 * i + 8 * q + 4 * fh, p = n * l.rows + m;
        if (n >= r.rows || m >= l.rows) continue;
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = scale * tile.acc[i][j][4 * q + e];
        const int count = (int)(l.rows - m < 4 ? l.rows - m : 4);
        if (g.splits == 1) {
          finish_out4(out, p, x, count);
        } else {
          float* part = out.partial + (long long)split * r.rows * l.rows + p;
          if (count == 4) *reinterpret_cast<f32x4_any*>(part) = x;
          else
            for (int e = 0; e < count; ++e) part[e] = x[e];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// bf16 results in whole, through the image in LDS.
template <typename T>
__device__ __forceinline__ void store_whole(const T& tile, const HeadOperand& l, const HeadOperand& r, const HeadOut& out, float scale,
                                            long long row0, long long col0, unsigned char* smem) {
#pragma unroll
  for (int j = 0; j < T::FN; ++j)
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = scale * tile.acc[i][j][4 * q + e];
        tile.put(smem, i, j, q, u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])});
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  __syncthreads();
  tile.image_out(smem, [&](int c, int m, u32x4 v) {
    const long long n = col0 + c;
    if (n >= r.rows || row0 + m >= l.rows) return;
    u16* to = static_cast<u16*>(out.out) + n * l.rows + row0 + m;
    if (row0 + m + 8 <= l.rows) {
      *reinterpret_cast<u32x4_any*>(to) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (row0 + m + e < l.rows) to[e] = (u16)(v[e / 2] >> (16 * (e & 1)));
    }
  });
}

template <int B, int S, bool RKM, bool IMAGE>
__device__ __forceinline__ void product_tile(const HeadOperand& l, const HeadOperand& r, const HeadTiles& g, const HeadOut& out, int split,
                                             long long row0, long long col0, unsigned char* smem) {
  using T = Tile<B, B, true, RKM, S>;
  const int slabs = (int)((g.k + kHeadSlab - 1) / kHeadSlab) * g.pairs;
  const int first = split * g.slabs_per_split, last = first + g.slabs_per_split < slabs ? first + g.slabs_per_split : slabs;
  T tile;
  tile.run(l, r, row0, col0, g.k, g.pairs, first, last, smem);
  const float scale = out.scale * (out.peak ? *out.peak : 1.f);
  if constexpr (IMAGE) store_whole(tile, l, r, out, scale, row0, col0, smem);
  else store_parts(tile, l, r, g, out, scale, split, row0, col0);
}

template <int B, int S, bool RKM, bool IMAGE>
__global__ __launch_bounds__(256, B == 128 && S == 2 ? 2 : 1) void head_product_kernel(HeadOperand l, HeadOperand r, HeadTiles g, HeadOut out) {
#if defined(__HIP_DEVICE_COMPILE__)            // (the host's pass knows no buffer descriptors)
  extern __shared__ __align__(16) unsigned char smem[];
  const TileAt at = tile_at(g);
  long long row0 = (long long)at.m * B, col0 = (long long)at.n * B;
  if (B == 128 || at.quarter < 0) {
    product_tile<B, S, RKM, IMAGE>(l, r, g, out, at.split, row0, col0, smem);
  } else if constexpr (B == 256) {
    row0 += 128 * (at.quarter >> 1);
    col0 += 128 * (at.quarter & 1);
    if (row0 < l.rows && col0 < r.rows) product_tile<128, 4, RKM, IMAGE>(l, r, g, out, at.split, row0, col0, smem);
  }
#endif
}

// 256 elements per block, four per thread; the splits over the block's waves, joined in LDS.
__global__ __launch_bounds__(256) void head_sum_splits_kernel(HeadOut out, int splits, long long count) {
  __shared__ f32x4 parts[3][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long at = blockIdx.x * 256ll + 4 * lane;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (at + 4 <= count) {
#pragma unroll 4
    for (int u = wave; u < splits; u += 4) x += *reinterpret_cast<const f32x4_any*>(out.partial + u * count + at);
  } else {
    for (int u = wave; u < splits; u += 4)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < count) x[e] += out.partial[u * count + at + e];
  }
  if (wave > 0) parts[wave - 1][lane] = x;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) x += parts[w][lane];
  if (at < count) finish_out4(out, at, x, (int)(count - at < 4 ? count - at : 4));
}

__global__ __launch_bounds__(256) void fill_zero_kernel(u16* p, size_t n) {
  for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += gridDim.x * 256ull) p[i] = 0;
}

HeadTiles tiles_of(const HeadProduct& g, int pairs) {
  return {g.k, pairs, g.tiles_m, g.tiles_n, g.whole, g.splits, g.slabs_per_split};
}
unsigned blocks_for(long long threads) {
  const long long b = (threads + 255) / 256;
  return (unsigned)(b < (1ll << 20) ? b : (1ll << 20));
}

}  // namespace

// More than 64 KB of LDS has to be asked for, once per kernel and device (two threads that get here together ask twice).
hipError_t allow_lds(std::atomic<uint64_t>& done, const void* kernel, int bytes) {
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
  if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes)) return e;
  done.fetch_or(bit, std::memory_order_release);
  return hipSuccess;
}

template <int B, int S, bool PROB, bool F32>
hipError_t logits_of(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, float2* stats,
                     long long stats_pitch, void* prob, long long prob_pitch, hipStream_t s) {
  constexpr int lds = Tile<B, B, false, false, S>::kLds;
  static std::atomic<uint64_t> done{0};
  if (hipError_t e = allow_lds(done, reinterpret_cast<const void*>(&head_logits_kernel<B, S, PROB, F32>), lds)) return e;
  head_logits_kernel<B, S, PROB, F32><<<(unsigned)g.blocks(), 256, lds, s>>>(weight, hidden, tiles_of(g, pairs), unit, stats, stats_pitch, prob,
                                                                     prob_pitch);
  return hipGetLastError();
}

hipError_t launch_head_logits(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit,
                              float2* stats, long long stats_pitch, void* prob, long long prob_pitch, int prob_f32, hipStream_t s) {
#define MUON_HEAD_CASE(B, S)                                                                                                              \
  if (g.tile == B && (g.alone ? 4 : 2) == S)                                                                                              \
    return !prob      ? logits_of<B, S, false, false>(weight, hidden, g, pairs, unit, stats, stats_pitch, prob, prob_pitch, s)            \
           : prob_f32 ? logits_of<B, S, true, true>(weight, hidden, g, pairs, unit, stats, stats_pitch, prob, prob_pitch, s)              \
                      : logits_of<B, S, true, false>(weight, hidden, g, pairs, unit, stats, stats_pitch, prob, prob_pitch, s)
  MUON_HEAD_CASE(256, 2);
  MUON_HEAD_CASE(128, 2);
  MUON_HEAD_CASE(128, 4);
#undef MUON_HEAD_CASE
  return hipErrorInvalidValue;
}

template <int B, int S, bool RKM, bool IMAGE>
hipError_t product_of(const HeadOperand& l, const HeadOperand& r, const HeadProduct& g, int pairs, const HeadOut& out, hipStream_t s) {
  constexpr int lds = Tile<B, B, true, RKM, S>::kLds;
  static std::atomic<uint64_t> done{0};
  if (hipError_t e = allow_lds(done, reinterpret_cast<const void*>(&head_product_kernel<B, S, RKM, IMAGE>), lds)) return e;
  head_product_kernel<B, S, RKM, IMAGE><<<(unsigned)g.blocks(), 256, lds, s>>>(l, r, tiles_of(g, pairs), out);
  return hipGetLastError();
}

hipError_t launch_head_product(const HeadOperand& l, const HeadOperand& r, int r_kmajor, const HeadProduct& g, int pairs,
                               const HeadOut& out, hipStream_t s) {
  const bool image = g.splits == 1 && !out.f32 && !out.add && !out.keep;
#define MUON_HEAD_CASE(B, S, KM)                                                                     \
  if (g.tile == B && (g.alone ? 4 : 2) == S && (r_kmajor != 0) == KM)                                \
    return image ? product_of<B, S, KM, true>(l, r, g, pairs, out, s) : product_of<B, S, KM, false>(l, r, g, pairs, out, s)
  MUON_HEAD_CASE(256, 2, false);
  MUON_HEAD_CASE(256, 2, true);
  MUON_HEAD_CASE(128, 2, false);
  MUON_HEAD_CASE(128, 2, true);
  MUON_HEAD_CASE(128, 4, false);
  MUON_HEAD_CASE(128, 4, true);
#undef MUON_HEAD_CASE
  return hipErrorInvalidValue;
}

hipError_t launch_head_pack(const void* src, long long stride, int f32, long long n, long long width, u16* dst, long long ld,
                            long long plane, hipStream_t s) {
  const unsigned blocks = blocks_for(n * (ld / 8));
  if (f32) head_pack_kernel<true><<<blocks, 256, 0, s>>>(src, stride, n, width, dst, ld, plane);
  else head_pack_kernel<false><<<blocks, 256, 0, s>>>(src, stride, n, width, dst, ld, plane);
  return hipGetLastError();
}

hipError_t launch_head_entries(const HeadTarget& t, const void* hidden, long long hidden_stride, const void* weight,
                               long long weight_stride, int f32, long long tokens, long long vocab, long long width, float* entry,
                               u16* masked, long long ld, long long plane, float* kept, hipStream_t s) {
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)tokens, 256, 0, s>>>(t, hidden, hidden_stride, weight, weight_stride, vocab, width, entry, masked, ld, plane, kept);
    return hipGetLastError();
  };
  return f32 ? go(head_entries_kernel<true>) : go(head_entries_kernel<false>);
}

hipError_t launch_head_peak(const float* kept, long long tokens, float* peak, hipStream_t s) {
  if (tokens <= kPeakInJoin) return hipSuccess;  // launch_head_join finds it
  head_peak_kernel<<<1, 1024, 0, s>>>(kept, tokens, peak);
  return hipGetLastError();
}

hipError_t launch_head_join(const HeadTarget& t, float unit, const float* kept, float* peak, const float2* stats,
                            long long stats_pitch, long long blocks, const float* entry, const HeadRows& rows, long long tokens, long long vocab,
                            float* loss, float* lse, float* value, float* scale, float2* log2sum, hipStream_t s) {
  head_join_kernel<<<(unsigned)((tokens + 15) / 16), 1024, 0, s>>>(t, unit, peak && tokens <= kPeakInJoin ? kept : nullptr, peak,
                                                                  stats, stats_pitch, blocks, entry, rows, tokens, vocab, loss, lse, value, scale,
                                                                  log2sum);
  return hipGetLastError();
}

hipError_t launch_head_grad(const HeadTarget& t, float unit, const float2* stats, long long stats_pitch, const float2* log2sum,
                            const float* value, const float* scale, long long tokens, long long vocab, const void* prob, long long pitch,
                            int f32, u16* grad, long long plane, hipStream_t s) {
  const int spans = (int)((pitch + kGradSpan - 1) / kGradSpan);
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)(tokens * spans), 256, 0, s>>>(t, unit, stats, stats_pitch, log2sum, value, scale, vocab, spans, prob, pitch, grad, plane);
    return hipGetLastError();
  };
  return f32 ? go(head_grad_kernel<true>) : go(head_grad_kernel<false>);
}

hipError_t launch_head_sum_splits(const HeadOut& out, int splits, long long count, hipStream_t s) {
  head_sum_splits_kernel<<<(unsigned)((count + 255) / 256), 256, 0, s>>>(out, splits, count);
  return hipGetLastError();
}

hipError_t launch_fill_zero(void* p, size_t bytes, hipStream_t s) {
  fill_zero_kernel<<<blocks_for((long long)(bytes / 2)), 256, 0, s>>>(static_cast<u16*>(p), bytes / 2);
  return hipGetLastError();
}

}  // namespace muon
