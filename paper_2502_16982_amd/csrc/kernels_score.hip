// Log probabilities of given tokens with the entropy of the whole distribution and its top alternatives, and their gradients, from hidden states
// H [T, D] and the head's weight W [V, D], logits never kept whole.
//
//   z = H W^T / tau    lse = log sum_v exp z_v    log p_v = z_v - lse    entropy = -sum_v p_v log p_v
//   d log p_y / d z_v = [v = y] - p_v             d entropy / d z_v = -p_v (log p_v + entropy)
//
// Forward: the logits' product with an epilogue that leaves, per 128 vocabulary entries and token, the largest logit, the sum of powers of two
// and the sum of powers times exponents (from which lse and entropy follow), and, where alternatives are asked for, the largest logit of
// each group of 32 with a bound on its second: the k largest logits lie in the k groups with the largest maxima, and only a group whose
// second may be among them is looked at again, so an eighth of the logits' own size is written and read.  One block per token then joins
// all of it.  Which alternatives come first is decided by logits that are summed in double, as the given token's is: in fp32 sums the order of two
// that are nearly alike would depend on the tiles.
// Backward: with lse known the product is done again and its epilogue writes the logits' gradient itself; the other two products are the losses'.
#include <hip/hip_runtime.h>

#include <atomic>

#include "head_gemm.h"
#include "head_rows.h"
#include "score_launch.h"
#include "score_plan.h"

namespace muon {

hipError_t allow_lds(std::atomic<uint64_t>& done, const void* kernel, int bytes);

namespace {

using namespace head;

__device__ __forceinline__ long long target_at(const ScoreTarget& t, long long i) {
  return t.index64 ? static_cast<const long long*>(t.index)[i] : (long long)static_cast<const int*>(t.index)[i];
}

// <a, b> over `width` elements by a whole wave, in double.
template <bool F32>
__device__ __forceinline__ double row_dot64(const void* a, long long a_at, const void* b, long long b_at, long long width) {
  double sum = 0.0;
  for (long long c = (threadIdx.x & 63) * 8; c < width; c += 512) {
    const Row8 x = load_row8<F32>(a, a_at, c, width), y = load_row8<F32>(b, b_at, c, width);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)x.v[e], (double)y.v[e], sum);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
  return sum;
}

// ---- forward: the product's epilogue ----
constexpr float kFarBelow = -1e4f;               // 2^this is 0: an infinite exponent times its power of 0 has to be 0

// Groups of a token in order of (64 vocabulary entries, half): a lane's 32 accumulators of a column, in two MFMA tiles.
__device__ __forceinline__ int place_row(int place, int half) { return 32 * (place >> 4) + 8 * ((place >> 2) & 3) + 4 * half + (place & 3); }

template <int B, int S, bool BEST>
__device__ __forceinline__ void score_tile(const HeadOperand& weight, const HeadOperand& hidden, const HeadTiles& g, float unit, ScoreStats* stats,
                                           long long stats_pitch, ScoreBest* best, long long best_pitch, long long row0, long long col0,
                                           unsigned char* smem) {
  using T = Tile<B, B, false, false, S>;
  T tile;
  tile.run(weight, hidden, row0, col0, g.k, g.pairs, 0, g.slabs_per_split, smem);
  const int fr = tile.lane & 31, fh = tile.lane >> 5;
  const long long v0 = row0 + tile.wm * T::WM;
  const int there = (int)(weight.rows - v0 < T::WM ? weight.rows - v0 : T::WM);      // rows of the wave's that there are
  auto work = [&](auto masked) {
    auto z = [&](int i, int j, int v) {
      const float x = tile.acc[i][j][v];
      return decltype(masked)::value && 32 * i + 8 * (v / 4) + 4 * fh + v % 4 >= there ? -INFINITY : x;
    };
    float top[T::FN];
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      top[j] = -INFINITY;
#pragma unroll
      for (int s = 0; s < T::FM / 2; ++s) {
        float first = -INFINITY, second = -INFINITY;
        int place = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float x = z(2 * s + u, j, v);
            if constexpr (BEST) {
              second = __builtin_amdgcn_fmed3f(first, second, x);
              place = x > first ? 16 * u + v : place;
            }
            first = fmaxf(first, x);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        top[j] = fmaxf(top[j], first);
        if constexpr (BEST) {
          const long long token = col0 + tile.wn * T::WN + 32 * j + fr, group = (v0 / 64 + s) * 2 + fh;
          if (token < hidden.rows && 64 * s < there)
            best[token * best_pitch + group] = ScoreBest{first, (__float_as_uint(second) & ~31u) | (unsigned)place};
        }
      }
      top[j] = fmaxf(top[j], __shfl_xor(top[j], 32, 64));
    }
    float* notes = reinterpret_cast<float*>(smem);
    if constexpr (B == 128) {                    // two waves share a block of statistics
#pragma unroll
      for (int j = 0; j < T::FN; ++j) notes[tile.wm * 128 + tile.wn * 64 + 32 * j + fr] = top[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < T::FN; ++j) top[j] = fmaxf(top[j], notes[(tile.wm ^ 1) * 128 + tile.wn * 64 + 32 * j + fr]);
    }
    float sums[T::FN], slopes[T::FN];
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      top[j] = top[j] == -INFINITY ? 0.f : unit * top[j];
      float sum = 0.f, slope = 0.f;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = fmaf(unit, z(i, j, 4 * q + e), -top[j]), x = __builtin_amdgcn_exp2f(y);
            sum += x;
            slope = fmaf(x, fmaxf(y, kFarBelow), slope);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      sums[j] = sum + __shfl_xor(sum, 32, 64);
      slopes[j] = slope + __shfl_xor(slope, 32, 64);
      if constexpr (B == 128) {
        if (tile.wm == 1) {
          notes[256 + tile.wn * 64 + 32 * j + fr] = sums[j];
          notes[384 + tile.wn * 64 + 32 * j + fr] = slopes[j];
        }
      }
    }
    if constexpr (B == 128) __syncthreads();
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const int c = tile.wn * T::WN + 32 * j + fr;
      if constexpr (B == 128) {
        sums[j] += notes[256 + c];
        slopes[j] += notes[384 + c];
      }
      if (fh == 0 && (B == 256 || tile.wm == 0) && v0 < weight.rows && col0 + c < hidden.rows)
        stats[v0 / kHeadGrain * stats_pitch + col0 + c] = ScoreStats{top[j], sums[j], slopes[j], 0.f};
    }
  };
  if (weight.rows - row0 >= B) work(std::false_type{});              // (by tile, not by wave: both sides hold barriers)
  else work(std::true_type{});
}

template <int B, int S, bool BEST>
__global__ __launch_bounds__(256, B == 128 && S == 2 ? 2 : 1) void score_logits_kernel(HeadOperand weight, HeadOperand hidden, HeadTiles g, float unit,
                                                                             ScoreStats* __restrict__ stats, long long stats_pitch,
                                                                             ScoreBest* __restrict__ best, long long best_pitch) {
#if defined(__HIP_DEVICE_COMPILE__)            // (the host's pass knows no buffer descriptors)
  extern __shared__ __align__(16) unsigned char smem[];
  const TileAt at = tile_at(g);
  long long row0 = (long long)at.m * B, col0 = (long long)at.n * B;
  if (B == 128 || at.quarter < 0) {
    score_tile<B, S, BEST>(weight, hidden, g, unit, stats, stats_pitch, best, best_pitch, row0, col0, smem);
  } else if constexpr (B == 256) {
    row0 += 128 * (at.quarter >> 1);
    col0 += 128 * (at.quarter & 1);
    if (row0 < weight.rows && col0 < hidden.rows)
      score_tile<128, 4, BEST>(weight, hidden, g, unit, stats, stats_pitch, best, best_pitch, row0, col0, smem);
  }
#endif
}

// ---- forward: one block per token joins the blocks and picks the alternatives ----
typedef unsigned long long u64;

// Larger keys are larger values, then lower rows; 0 is none.
__device__ __forceinline__ unsigned rising(unsigned bits) { return bits ^ ((unsigned)((int)bits >> 31) | 0x80000000u); }
__device__ __forceinline__ u64 key_of(float z, unsigned row) { return (u64)rising(__float_as_uint(z)) << 32 | (0xffffffffu - row); }
__device__ __forceinline__ unsigned key_row(u64 key) { return 0xffffffffu - (unsigned)key; }
__device__ __forceinline__ float second_bound(unsigned w) { return __uint_as_float((int)w < 0 ? w & ~31u : w | 31u); }

template <typename T, typename F>
__device__ __forceinline__ T wave_all(T x, F&& f) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = f(x, __shfl_xor(x, off, 64));
  return x;
}

template <bool F32>
__global__ __launch_bounds__(256) void score_finish_kernel(ScoreTarget t, float inv_tau, float unit, const ScoreStats* __restrict__ stats, long long stats_pitch,
                                                           long long blocks, const ScoreBest* __restrict__ best, long long groups, int top, HeadRows rows,
                                                           long long vocab, ScoreOut out) {
  constexpr int kPick = kScoreMaxTop + kScoreMargin, kList = 1024, kRows = kPick * 32;
  __shared__ float tops[4];
  __shared__ double sums[8];
  __shared__ u64 list[kList], picked[kPick];
  __shared__ double value[kRows];
  __shared__ int row_of[kRows];
  __shared__ int counts[3];
  __shared__ u64 bound;
  const long long token = blockIdx.x;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const auto larger = [](auto x, auto y) { return x > y ? x : y; };
  const auto add = [](auto x, auto y) { return x + y; };

  // lse and entropy: sums relative to the largest block's top, joined in double
  float m = -INFINITY, sum = 0.f, slope = 0.f;
  for (long long b = tid; b < blocks; b += 256) {
    const ScoreStats v = stats[b * stats_pitch + token];
    if (v.sum == 0.f) continue;
    const float now = fmaxf(m, v.top), down = m == -INFINITY ? 0.f : m - now, here = v.top - now, f = __builtin_amdgcn_exp2f(down), h = __builtin_amdgcn_exp2f(here);
    slope = f * fmaf(sum, down, slope) + h * fmaf(v.sum, here, v.slope);
    sum = f * sum + h * v.sum;
    m = now;
  }
  const float wave_top = wave_all(m, larger);
  if (lane == 0) tops[wave] = wave_top;
  if (tid < 3) counts[tid] = 0;
  if (tid == 0) bound = 0;
  __syncthreads();
  float all = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  if (all == -INFINITY) all = 0.f;
  const double down = m == -INFINITY ? 0.0 : (double)m - (double)all, f = m == -INFINITY ? 0.0 : exp2(down);
  const double s0 = wave_all(f * sum, add), e0 = wave_all(f * (slope + sum * down), add);
  if (lane == 0) sums[wave] = s0, sums[4 + wave] = e0;
  __syncthreads();
  const double mass = (sums[0] + sums[1]) + (sums[2] + sums[3]), tilt = (sums[4] + sums[5]) + (sums[6] + sums[7]);
  const double per = (double)inv_tau / (double)unit, l2 = log2(mass), lse = per * ((double)all + l2);
  if (tid == 0) {
    const double h = per * (l2 - tilt / mass);
    out.entropy[token] = h < 0.0 ? 0.f : (float)h;       // (what rounding leaves below 0; NaN stays)
    const float hi = (float)lse;
    out.lse[token] = hi;
    out.lse_rest[token] = (float)(lse - (double)hi);
  }
  const auto log_prob = [&](double z) {                  // cut off at 0: the logits in lse were summed in another order (NaN stays)
    const double d = (double)inv_tau * z - lse;
    return d > 0.0 ? 0.f : (float)d;
  };
  const auto logit = [&](long long v) {
    return row_dot64<F32>(rows.hidden, token * rows.hidden_stride, rows.weight, v * rows.weight_stride, rows.width);
  };
  if (out.log_prob && wave == 3) {
    const long long y = target_at(t, token);
    const float lp = y < 0 ? 0.f : y >= vocab ? __builtin_nanf("") : log_prob(logit(y));
    if (lane == 0) out.log_prob[token] = lp;
  }
  if (!top) return;

  // the largest maxima: those of a thread's groups that reach what the threads' own largest ones bound from below
  const ScoreBest* mine = best + token * groups;
  const long long all_groups = groups;
  const auto group_key = [&](long long g) -> u64 {
    const ScoreBest b = mine[g];
    const long long row = 64 * (g >> 1) + place_row((int)(b.second & 31u), (int)(g & 1));
    return row < vocab ? key_of(b.z, (unsigned)row) : 0;
  };
  const auto there = [&](long long g) { return 64 * (g >> 1) + 4 * (g & 1) < vocab; };
  u64 own = 0;
  for (long long g = tid; g < all_groups; g += 256)
    if (there(g)) own = larger(own, group_key(g));
  list[tid] = own;
  __syncthreads();
  const int pick = top + kScoreMargin;
  {
    int rank = 0;
    for (int i = 0; i < 256; ++i) rank += list[i] > own;
    if (own && rank == pick - 1) bound = own;
  }
  __syncthreads();
  const auto collect = [&](u64 from) {
    for (long long g = tid; g < all_groups; g += 256) {
      if (!there(g)) continue;
      const u64 key = group_key(g);
      if (key >= from && key) {
        const int at = atomicAdd(&counts[0], 1);
        if (at < kList) list[at] = key;
      }
    }
  };
  collect(bound);
  __syncthreads();
  if (counts[0] > kList) {                               // a few threads hold most of the largest: the bound bit by bit instead
    u64 from = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const u64 tried = from | 1ull << bit;
      __syncthreads();
      if (tid == 0) counts[0] = 0;
      __syncthreads();
      int n = 0;
      for (long long g = tid; g < all_groups; g += 256) n += there(g) && group_key(g) >= tried;
      n = wave_all(n, add);
      if (lane == 0) atomicAdd(&counts[0], n);
      __syncthreads();
      if (counts[0] >= pick) from = tried;
    }
    __syncthreads();
    if (tid == 0) counts[0] = 0;
    __syncthreads();
    collect(from);
    __syncthreads();
  }
  const int n = counts[0];
  for (int i = tid; i < n; i += 256) {
    const u64 key = list[i];
    int rank = 0;
    for (int k = 0; k < n; ++k) rank += list[k] > key;
    if (rank < pick) picked[rank] = key;
  }
  __syncthreads();
  // their rows, and all rows of a group whose second may be among the largest as well
  const int have = n < pick ? n : pick;
  const u64 last = n >= pick ? picked[pick - 1] : 0;
  if (tid < have) {
    const unsigned row = key_row(picked[tid]);
    const long long slab = row / 64, half = (row >> 2) & 1, g = 2 * slab + half;
    row_of[tid] = (int)row;
    if (((u64)rising(__float_as_uint(second_bound(mine[g].second))) << 32 | 0xffffffffu) >= last) {
      const int at = have + 31 * atomicAdd(&counts[1], 1);
      int k = 0;
      for (int place = 0; place < 32; ++place) {
        const long long other = 64 * slab + place_row(place, (int)half);
        if (other != row) row_of[at + k++] = other < vocab ? (int)other : -1;
      }
    }
  }
  __syncthreads();
  const int c = have + 31 * counts[1];
  for (int i = wave; i < c; i += 4) {
    const int row = row_of[i];
    const double z = row < 0 ? 0.0 : logit(row);
    if (lane == 0) value[i] = z;
  }
  __syncthreads();
  const auto order = [&](int i) -> u64 {                 // NaN below everything
    const u64 bits = __double_as_longlong(value[i]);
    return value[i] != value[i] ? 0 : bits ^ ((u64)((long long)bits >> 63) | 0x8000000000000000ull);
  };
  for (int i = tid; i < c; i += 256) {
    if (row_of[i] < 0) continue;
    const u64 own_order = order(i);
    int rank = 0;
    for (int k = 0; k < c; ++k) {
      if (row_of[k] < 0) continue;
      const u64 o = order(k);
      rank += o > own_order || (o == own_order && row_of[k] < row_of[i]);
    }
    if (rank < top) {
      out.top_index[token * top + rank] = row_of[i];
      out.top_log_prob[token * top + rank] = log_prob(value[i]);
    }
  }
}

// ---- backward ----
// Gradients of a token's log probability and entropy; both 0 where it has none.
struct Given {
  float g, h;
};
__device__ __forceinline__ Given given(const ScoreTarget& t, const ScoreGrads& d, long long token, long long vocab) {
  Given x{0.f, d.d_entropy ? d.d_entropy[token] : 0.f};
  if (t.index && d.d_log_prob) {
    const long long y = target_at(t, token);
    if (y >= 0 && y < vocab) x.g = d.d_log_prob[token];
  }
  return x;
}

__global__ __launch_bounds__(1024) void score_peak_kernel(ScoreTarget t, ScoreGrads d, long long tokens, long long vocab, float* __restrict__ peak) {
  __shared__ float waves[16];
  float top = 0.f;
  for (long long i = threadIdx.x; i < tokens; i += 1024) {
    const Given x = given(t, d, i, vocab);
    if (fabsf(x.g) < INFINITY) top = fmaxf(top, fabsf(x.g));
    if (fabsf(x.h) < INFINITY) top = fmaxf(top, fabsf(x.h));
  }
  top = wave_all(top, [](float x, float y) { return fmaxf(x, y); });
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) top = fmaxf(top, waves[w]);
    *peak = top > 0.f ? top : 1.f;
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void score_prepare_kernel(ScoreTarget t, float inv_tau, float unit, ScoreGrads d, const float* __restrict__ peak, HeadRows rows,
                                                            long long vocab, ScoreCoef c, u16* __restrict__ masked, long long ld, long long plane) {
  const long long token = blockIdx.x, at = token * rows.hidden_stride;
  Given x = given(t, d, token, vocab);
  const bool some = x.g != 0.f || x.h != 0.f;            // (NaN counts)
  if (threadIdx.x < 64) {
    float a = 0.f, b = 0.f, value = 0.f;
    float2 l2 = make_float2(INFINITY, 0.f);
    if (some) {
      const double per = 1.0 / (double)*peak, g = per * x.g, h = per * x.h, lse = (double)d.lse[token] + (double)d.lse_rest[token],
                   entropy = x.h != 0.f ? (double)d.entropy[token] : 0.0;
      const double sum2 = lse * ((double)unit / (double)inv_tau);
      a = (float)(g + h * entropy);
      b = (float)(h * 0.69314718055994530942);
      l2.x = (float)sum2;
      l2.y = (float)(sum2 - (double)l2.x);
      const long long y = t.index ? target_at(t, token) : -1;
      if (y >= 0 && y < vocab) {
        const double z = row_dot64<F32>(rows.hidden, at, rows.weight, y * rows.weight_stride, rows.width);
        const double d0 = (double)inv_tau * z - lse, lp = d0 > 0.0 ? 0.0 : d0, p = exp(lp);
        value = (float)(-g * expm1(lp) - (x.h != 0.f && p > 0.0 ? h * p * (lp + entropy) : 0.0));
      }
    }
    if (threadIdx.x == 0) {
      c.a[token] = a;
      c.b[token] = b;
      c.value[token] = value;
      c.log2sum[token] = l2;
    }
  }
  if (masked) {
    for (long long k = threadIdx.x * 8; k < ld; k += 2048) {
      Row8 r{};
      if (some) r = load_row8<F32>(rows.hidden, at, k, rows.width);
      store_planes8<F32>(r, masked + token * ld + k, plane);
    }
  }
}

template <int B, int S, bool F32>
__device__ __forceinline__ void score_grad_tile(const HeadOperand& weight, const HeadOperand& hidden, const HeadTiles& g, float unit, const ScoreTarget& t,
                                                const ScoreCoef& c, u16* grad, long long pitch, long long plane, long long row0, long long col0,
                                                unsigned char* smem) {
  using T = Tile<B, B, false, false, S>;
  T tile;
  tile.run(weight, hidden, row0, col0, g.k, g.pairs, 0, g.slabs_per_split, smem);
  const int fr = tile.lane & 31, fh = tile.lane >> 5;
  const long long v0 = row0 + tile.wm * T::WM;
  const int there = (int)(weight.rows - v0 < T::WM ? weight.rows - v0 : T::WM);
  // the target's entry of this thread's column, which goes over what its wave wrote
  const int column = threadIdx.x;
  long long patch_row = -1;
  float patch = 0.f;
  if (column < B && col0 + column < hidden.rows && t.index) {
    patch_row = target_at(t, col0 + column) - row0;
    patch = c.value[col0 + column];
  }
  constexpr int kPlanes = F32 ? 3 : 1;
#pragma unroll
  for (int p = 0; p < kPlanes; ++p) {
    if (p) __syncthreads();                              // the image has left
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const long long token = col0 + tile.wn * T::WN + 32 * j + fr;
      float a = 0.f, b = 0.f;
      float2 l2 = make_float2(INFINITY, 0.f);
      if (p == 0 && token < hidden.rows) {
        a = c.a[token];
        b = c.b[token];
        l2 = c.log2sum[token];
      }
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (p == 0) {
              const float y = fmaxf(fmaf(unit, tile.acc[i][j][4 * q + e], -l2.x) - l2.y, kFarBelow);
              x[e] = -__builtin_amdgcn_exp2f(y) * fmaf(b, y, a);
              if (32 * i + 8 * q + 4 * fh + e >= there) x[e] = 0.f;
            } else {
              x[e] = tile.acc[i][j][4 * q + e];
            }
          }
          const u32x2 w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
          tile.put(smem, i, j, q, w);
          if constexpr (F32) {                           // what the plane leaves
            tile.acc[i][j][4 * q] = x[0] - bf16_lo(w.x);
            tile.acc[i][j][4 * q + 1] = x[1] - bf16_hi(w.x);
            tile.acc[i][j][4 * q + 2] = x[2] - bf16_lo(w.y);
            tile.acc[i][j][4 * q + 3] = x[3] - bf16_hi(w.y);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();
    if (patch_row >= 0 && patch_row < B && row0 + patch_row < weight.rows) {
      const int r = (int)patch_row;
      const u16 bits = bf16_bits(patch);
      *reinterpret_cast<u16*>(smem + column * (B * 2) + (((r / 8) ^ (column & T::KEY)) * 16) + (r % 8) * 2) = bits;
      patch -= bf16_value(bits);
    }
    __syncthreads();
    tile.image_out(smem, [&](int k, int r, u32x4 v) {
      if (col0 + k < hidden.rows) *reinterpret_cast<u32x4*>(grad + p * plane + (col0 + k) * pitch + row0 + r) = v;
    });
  }
}

template <int B, int S, bool F32>
__global__ __launch_bounds__(256, B == 128 && S == 2 ? 2 : 1) void score_grad_kernel(HeadOperand weight, HeadOperand hidden, HeadTiles g, float unit, ScoreTarget t,
                                                                           ScoreCoef c, u16* __restrict__ grad, long long pitch, long long plane) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __align__(16) unsigned char smem[];
  const TileAt at = tile_at(g);
  long long row0 = (long long)at.m * B, col0 = (long long)at.n * B;
  if (B == 128 || at.quarter < 0) {
    score_grad_tile<B, S, F32>(weight, hidden, g, unit, t, c, grad, pitch, plane, row0, col0, smem);
  } else if constexpr (B == 256) {
    row0 += 128 * (at.quarter >> 1);
    col0 += 128 * (at.quarter & 1);
    if (row0 < weight.rows && col0 < hidden.rows) score_grad_tile<128, 4, F32>(weight, hidden, g, unit, t, c, grad, pitch, plane, row0, col0, smem);
  }
#endif
}

}  // namespace

template <int B, int S, bool BEST>
hipError_t score_logits_of(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, ScoreStats* stats,
                           long long stats_pitch, ScoreBest* best, long long best_pitch, hipStream_t s) {
  constexpr int lds = Tile<B, B, false, false, S>::kLds;
  static std::atomic<uint64_t> done{0};
  if (hipError_t e = allow_lds(done, reinterpret_cast<const void*>(&score_logits_kernel<B, S, BEST>), lds)) return e;
  score_logits_kernel<B, S, BEST><<<(unsigned)g.blocks(), 256, lds, s>>>(weight, hidden, tiles_of(g, pairs), unit, stats, stats_pitch, best, best_pitch);
  return hipGetLastError();
}

hipError_t launch_score_logits(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, ScoreStats* stats,
                               long long stats_pitch, ScoreBest* best, long long best_pitch, hipStream_t s) {
#define MUON_SCORE_CASE(B, S)                                                                                             \
  if (g.tile == B && (g.alone ? 4 : 2) == S)                                                                              \
    return best ? score_logits_of<B, S, true>(weight, hidden, g, pairs, unit, stats, stats_pitch, best, best_pitch, s)   \
                : score_logits_of<B, S, false>(weight, hidden, g, pairs, unit, stats, stats_pitch, best, best_pitch, s)
  MUON_SCORE_CASE(256, 2);
  MUON_SCORE_CASE(128, 2);
  MUON_SCORE_CASE(128, 4);
#undef MUON_SCORE_CASE
  return hipErrorInvalidValue;
}

hipError_t launch_score_finish(const ScoreTarget& t, float inv_tau, float unit, const ScoreStats* stats, long long stats_pitch, long long blocks,
                               const ScoreBest* best, long long groups, int top, const HeadRows& rows, long long tokens, long long vocab, const ScoreOut& out,
                               hipStream_t s) {
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)tokens, 256, 0, s>>>(t, inv_tau, unit, stats, stats_pitch, blocks, best, groups, top, rows, vocab, out);
    return hipGetLastError();
  };
  return rows.f32 ? go(score_finish_kernel<true>) : go(score_finish_kernel<false>);
}

hipError_t launch_score_peak(const ScoreTarget& t, const ScoreGrads& d, long long tokens, long long vocab, float* peak, hipStream_t s) {
  score_peak_kernel<<<1, 1024, 0, s>>>(t, d, tokens, vocab, peak);
  return hipGetLastError();
}

hipError_t launch_score_prepare(const ScoreTarget& t, float inv_tau, float unit, const ScoreGrads& d, const float* peak, const HeadRows& rows,
                                long long tokens, long long vocab, const ScoreCoef& c, uint16_t* masked, long long ld, long long plane, hipStream_t s) {
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)tokens, 256, 0, s>>>(t, inv_tau, unit, d, peak, rows, vocab, c, masked, ld, plane);
    return hipGetLastError();
  };
  return rows.f32 ? go(score_prepare_kernel<true>) : go(score_prepare_kernel<false>);
}

template <int B, int S, bool F32>
hipError_t score_grad_of(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, const ScoreTarget& t,
                         const ScoreCoef& c, uint16_t* grad, long long pitch, long long plane, hipStream_t s) {
  constexpr int lds = Tile<B, B, false, false, S>::kLds;
  static std::atomic<uint64_t> done{0};
  if (hipError_t e = allow_lds(done, reinterpret_cast<const void*>(&score_grad_kernel<B, S, F32>), lds)) return e;
  score_grad_kernel<B, S, F32><<<(unsigned)g.blocks(), 256, lds, s>>>(weight, hidden, tiles_of(g, pairs), unit, t, c, grad, pitch, plane);
  return hipGetLastError();
}

hipError_t launch_score_grad(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, const ScoreTarget& t,
                             const ScoreCoef& c, bool f32, uint16_t* grad, long long pitch, long long plane, hipStream_t s) {
#define MUON_SCORE_CASE(B, S)                                                                                 \
  if (g.tile == B && (g.alone ? 4 : 2) == S)                                                                  \
    return f32 ? score_grad_of<B, S, true>(weight, hidden, g, pairs, unit, t, c, grad, pitch, plane, s)      \
               : score_grad_of<B, S, false>(weight, hidden, g, pairs, unit, t, c, grad, pitch, plane, s)
  MUON_SCORE_CASE(256, 2);
  MUON_SCORE_CASE(128, 2);
  MUON_SCORE_CASE(128, 4);
#undef MUON_SCORE_CASE
  return hipErrorInvalidValue;
}

}  // namespace muon
