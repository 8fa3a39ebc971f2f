// Log probabilities of given tokens with the entropy of the whole distribution and its top alternatives, and their gradients, from hidden states
// H [T, D] and the head's weight W [V, D].  Logits are not kept, but where the caller gives memory for their powers (fp32: for themselves).
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
// Backward: where the forward call kept its powers (f16 under each block's own top; fp32: the logits), one pass makes the logits' gradient of them;
// else, with lse known, the product is done again and its epilogue writes the gradient itself.  The other two products are the losses'.
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

// f over a wave's lanes, in all of them, with moves between registers only: rotations within 16 lanes, then exchanges of rows of 16 and 32.
template <typename T>
struct Words {
  unsigned w[sizeof(T) / 4];
};
template <int CTRL, typename T>
__device__ __forceinline__ T rotated(T x) {
  Words<T> v = __builtin_bit_cast(Words<T>, x);
#pragma unroll
  for (auto& w : v.w) w = __builtin_amdgcn_update_dpp(0u, w, CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(T, v);
}
template <bool BY32, typename T, typename F>
__device__ __forceinline__ T across(T x, F&& f) {
  const Words<T> v = __builtin_bit_cast(Words<T>, x);
  Words<T> a, b;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 4; ++i) {
    const auto both = BY32 ? __builtin_amdgcn_permlane32_swap(v.w[i], v.w[i], false, false) : __builtin_amdgcn_permlane16_swap(v.w[i], v.w[i], false, false);
    a.w[i] = both[0];
    b.w[i] = both[1];
  }
  return f(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
}
template <typename T, typename F>
__device__ __forceinline__ T wave_all(T x, F&& f) {
  x = f(x, rotated<0x128>(x));
  x = f(x, rotated<0x124>(x));
  x = f(x, rotated<0x122>(x));
  x = f(x, rotated<0x121>(x));
  return across<true>(across<false>(x, f), f);
}
struct Add {
  template <typename T>
  __device__ __forceinline__ T operator()(T x, T y) const {
    return x + y;
  }
};

// Elements [c, c + 8) of a row that has them, as they lie there.  (load_row8 decides for each row anew and waits for it there: the finish of
// 300 x 8191 x 512 fp32, top 20, 35 us so, 22 with these.)
template <bool F32>
struct Raw8 {
  u32x4 w[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ Raw8<F32> load_raw8(const void* base, long long row_at, long long c) {
  const char* p = static_cast<const char*>(base) + (row_at + c) * (F32 ? 4 : 2);
  Raw8<F32> r;
#pragma unroll
  for (int q = 0; q < (F32 ? 2 : 1); ++q) {
    if constexpr (F32) r.w[q] = __builtin_bit_cast(u32x4, (f32x4)*reinterpret_cast<const f32x4_any*>(p + 16 * q));
    else r.w[q] = *reinterpret_cast<const u32x4_any*>(p);
  }
  return r;
}
template <bool F32>
__device__ __forceinline__ double raw_value(const Raw8<F32>& r, int e) {
  if constexpr (F32) return (double)__uint_as_float(r.w[e / 4][e % 4]);
  else return (double)(e % 2 ? bf16_hi(r.w[0][e / 2]) : bf16_lo(r.w[0][e / 2]));
}
template <bool F32>
__device__ __forceinline__ float load_one(const void* base, long long at) {
  if constexpr (F32) return static_cast<const float*>(base)[at];
  else return bf16_value(static_cast<const u16*>(base)[at]);
}

// <a, b> over `width` elements by a whole wave, in double.
template <bool F32>
__device__ __forceinline__ double row_dot64(const void* a, long long a_at, const void* b, long long b_at, long long width) {
  double sum = 0.0;
  const int lane = threadIdx.x & 63;
  for (long long c = lane * 8; c + 8 <= width; c += 512) {
    const Raw8<F32> x = load_raw8<F32>(a, a_at, c), y = load_raw8<F32>(b, b_at, c);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma(raw_value(x, e), raw_value(y, e), sum);
  }
  const long long c = width / 8 * 8 + lane;              // the last elements, one per lane
  if (c < width) sum = fma((double)load_one<F32>(a, a_at + c), (double)load_one<F32>(b, b_at + c), sum);
  return wave_all(sum, Add{});
}

// ---- forward: the product's epilogue ----
constexpr float kProbScale = (float)(1 << (int)kProbTop);
constexpr float kFarBelow = -1e4f;               // 2^this is 0: an infinite exponent times its power of 0 has to be 0

// Groups of a token in order of (64 vocabulary entries, half): a lane's 32 accumulators of a column, in two MFMA tiles.
__device__ __forceinline__ int place_row(int place, int half) { return 32 * (place >> 4) + 8 * ((place >> 2) & 3) + 4 * half + (place & 3); }

// KEEP: 1 the powers in f16, up to 2^15 in a block, 2 the logits in fp32, 0 neither.
template <int B, int S, bool BEST, int KEEP>
__device__ __forceinline__ void score_tile(const HeadOperand& weight, const HeadOperand& hidden, const HeadTiles& g, float unit, ScoreStats* stats,
                                           ScoreBest* best, const ScoreKept& kept, long long row0, long long col0, unsigned char* smem) {
  using T = Tile<B, B, false, false, S>;
  T tile;
  tile.run(weight, hidden, row0, col0, g.k, g.pairs, 0, g.slabs_per_split, smem);
  const int fr = tile.lane & 31, fh = tile.lane >> 5;
  const long long v0 = row0 + tile.wm * T::WM;
  const int there = (int)(weight.rows - v0 < T::WM ? weight.rows - v0 : T::WM);      // rows of the wave's that there are
  auto row = [&](int i, int v) { return 32 * i + 8 * (v / 4) + 4 * fh + v % 4; };
  // in LDS: what two waves tell each other, then what leaves, a token's neighbouring entries in whole lines
  // (in tiles of 128 behind the powers' image, in tiles of 256 after it)
  constexpr int kGroups = B / kScoreGroup, kBlocks = B / kHeadGrain;
  static_assert(KEEP == 0 || !BEST, "one of both");
  unsigned char* room = smem + (B == 128 ? T::kStage : 0);
  float* notes = reinterpret_cast<float*>(room);
  ScoreStats* sheet = reinterpret_cast<ScoreStats*>(room + 2048);                    // [column][block]
  ScoreBest* image = reinterpret_cast<ScoreBest*>(room + 2048 + B * kBlocks * 16);   // [column][group]
  if constexpr (KEEP == 2) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const long long token = col0 + tile.wn * T::WN + 32 * j + fr;
      if (token >= hidden.rows) continue;
      float* z = static_cast<float*>(kept.values) + token * kept.pitch + v0 + 4 * fh;
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
  auto find_top = [&](auto masked) {             // MASKED: not all rows of the wave's are there
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
            float x = tile.acc[2 * s + u][j][v];
            if (decltype(masked)::value && row(2 * s + u, v) >= there) x = -INFINITY;
            if constexpr (BEST) {
              second = __builtin_amdgcn_fmed3f(first, second, x);
              place = x > first ? 16 * u + v : place;
            }
            first = fmaxf(first, x);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        top[j] = fmaxf(top[j], first);
        if constexpr (BEST)
          image[(tile.wn * T::WN + 32 * j + fr) * kGroups + (tile.wm * T::WM / 64 + s) * 2 + fh] =
              ScoreBest{first, (__float_as_uint(second) & ~31u) | (unsigned)place};
      }
      top[j] = fmaxf(top[j], __shfl_xor(top[j], 32, 64));
    }
  };
  if (there >= T::WM) find_top(std::false_type{});
  else find_top(std::true_type{});
  if constexpr (B == 128) {                      // two waves share a block of statistics
#pragma unroll
    for (int j = 0; j < T::FN; ++j) notes[tile.wm * 128 + tile.wn * 64 + 32 * j + fr] = top[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T::FN; ++j) top[j] = fmaxf(top[j], notes[(tile.wm ^ 1) * 128 + tile.wn * 64 + 32 * j + fr]);
  }
  float sums[T::FN], slopes[T::FN];
  auto take_powers = [&](auto masked) {
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      top[j] = top[j] == -INFINITY ? 0.f : unit * top[j];
      float sum = 0.f, slope = 0.f;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = fmaf(unit, tile.acc[i][j][4 * q + e], -top[j]);
            x[e] = __builtin_amdgcn_exp2f(y);
            if (decltype(masked)::value && row(i, 4 * q + e) >= there) x[e] = 0.f;
            sum += x[e];
            slope = fmaf(x[e], fmaxf(y, kFarBelow), slope);
          }
          // (only what is kept is times 2^kProbTop: in the sums, exponents 15 from 0 would carry the rounding steps of 15, and the entropy is their difference)
          if constexpr (KEEP == 1)
            tile.put(smem, i, j, q, u32x2{pack_f16(kProbScale * x[0], kProbScale * x[1]), pack_f16(kProbScale * x[2], kProbScale * x[3])});
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
  };
  if (there >= T::WM) take_powers(std::false_type{});
  else take_powers(std::true_type{});
  if constexpr (KEEP == 1) {
    __syncthreads();
    tile.image_out(smem, [&](int c, int r, u32x4 v) {
      if (col0 + c < hidden.rows) *reinterpret_cast<u32x4*>(static_cast<u16*>(kept.values) + (col0 + c) * kept.pitch + row0 + r) = v;
    });
    if constexpr (B == 256) __syncthreads();
  }
  if constexpr (B == 128) __syncthreads();
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const int c = tile.wn * T::WN + 32 * j + fr;
    if constexpr (B == 128) {
      sums[j] += notes[256 + c];
      slopes[j] += notes[384 + c];
    }
    if (fh == 0 && (B == 256 || tile.wm == 0)) sheet[c * kBlocks + (B == 256 ? tile.wm : 0)] = ScoreStats{top[j], sums[j], slopes[j], 0.f};
  }
  __syncthreads();
  // 16 bytes per thread: a block's statistics, two groups
  const long long blocks = (weight.rows + kHeadGrain - 1) / kHeadGrain;
  for (int i = threadIdx.x; i < B * kBlocks; i += 256) {
    const long long token = col0 + i / kBlocks, block = row0 / kHeadGrain + i % kBlocks;
    if (token < hidden.rows && block < blocks) {
      stats[token * blocks + block] = sheet[i];
      if constexpr (KEEP == 1) kept.tops[token * blocks + block] = sheet[i].top;
    }
  }
  if constexpr (BEST) {
#pragma unroll
    for (int i0 = 0; i0 < B * kGroups / 2; i0 += 256) {
      const int i = i0 + threadIdx.x, pair = i % (kGroups / 2);
      const long long token = col0 + i / (kGroups / 2), group = row0 / kScoreGroup + 2 * pair, groups = blocks * (kHeadGrain / kScoreGroup);
      if (token < hidden.rows && group < groups)
        *reinterpret_cast<u32x4*>(best + token * groups + group) = *reinterpret_cast<const u32x4*>(image + 2 * i);
    }
  }
}

template <int B, int S, bool BEST, int KEEP>
__global__ __launch_bounds__(256, B == 128 && S == 2 ? 2 : 1) void score_logits_kernel(HeadOperand weight, HeadOperand hidden, HeadTiles g, float unit,
                                                                             ScoreStats* __restrict__ stats, ScoreBest* __restrict__ best, ScoreKept kept) {
#if defined(__HIP_DEVICE_COMPILE__)            // (the host's pass knows no buffer descriptors)
  extern __shared__ __align__(16) unsigned char smem[];
  const TileAt at = tile_at(g);
  long long row0 = (long long)at.m * B, col0 = (long long)at.n * B;
  if (B == 128 || at.quarter < 0) {
    score_tile<B, S, BEST, KEEP>(weight, hidden, g, unit, stats, best, kept, row0, col0, smem);
  } else if constexpr (B == 256) {
    row0 += 128 * (at.quarter >> 1);
    col0 += 128 * (at.quarter & 1);
    if (row0 < weight.rows && col0 < hidden.rows)
      score_tile<128, 4, BEST, KEEP>(weight, hidden, g, unit, stats, best, kept, row0, col0, smem);
  }
#endif
}

// ---- forward, few tokens: the same statistics straight from the rows ----
// 16 rows of W or H and 64 (fp32 32) columns, as the matrix instruction of 16 x 16 takes them: lane l holds row l % 16 and, of its group l / 16, 32
// neighbouring bytes, so that four lanes take whole lines; which columns a step is made of is free as long as both operands agree.
template <bool F32>
struct FewPart {
  static constexpr int COLS = F32 ? 32 : 64, OWN = COLS / 4, SIZE = F32 ? 4 : 2;
  u32x4 v[2];
  __device__ __forceinline__ void load(const unsigned char* p) {
    v[0] = *reinterpret_cast<const u32x4_any*>(p);
    v[1] = *reinterpret_cast<const u32x4_any*>(p + 16);
  }
  // its first `count` elements, zeros behind them
  __device__ __forceinline__ void load_some(const unsigned char* p, int count) {
    v[0] = v[1] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < OWN; ++e) {
      if (e >= count) continue;
      if constexpr (F32) v[e / 4][e % 4] = reinterpret_cast<const unsigned*>(p)[e];
      else v[e / 8][e / 2 % 4] |= (unsigned)reinterpret_cast<const u16*>(p)[e] << 16 * (e & 1);
    }
  }
};
typedef float few_acc __attribute__((ext_vector_type(4)));
template <bool F32>
__device__ __forceinline__ few_acc few_multiply(const FewPart<F32>& w, const FewPart<F32>& h, few_acc acc) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned a = w.v[u][e], b = h.v[u][e];
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), acc, 0, 0, 0);
      }
    } else {
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.v[u]), __builtin_bit_cast(bf16x8, h.v[u]), acc, 0, 0, 0);
    }
  }
  return acc;
}

// Block: 128 vocabulary entries x up to 16 NT tokens, 32 entries per wave.  fp32 rows as they are, on the fp32 matrix instructions.  Bound by W's
// rows: fp32 100003 x 2048, 819 MB, with one token 200 us with the finish (4.1 TB/s), with 64 by the matrix instructions, 481.
template <bool F32, int NT, bool BEST>
__global__ __launch_bounds__(256) void score_few_kernel(HeadRows rows, long long tokens, long long vocab, float unit, ScoreStats* __restrict__ stats,
                                                        ScoreBest* __restrict__ best) {
  using P = FewPart<F32>;
  constexpr int kAhead = NT == 1 ? 4 : NT == 2 ? 2 : 1, kPitch = kHeadGrain + 4;
  __shared__ float zs[16 * kPitch];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const long long block = blockIdx.x, v0 = block * kHeadGrain;
  const unsigned char *w[2], *h[NT];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const long long row = v0 + 32 * wave + 16 * u + r;
    w[u] = static_cast<const unsigned char*>(rows.weight) + ((row < vocab ? row : vocab - 1) * rows.weight_stride + P::OWN * g) * P::SIZE;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const long long token = 16 * t + r;
    h[t] = static_cast<const unsigned char*>(rows.hidden) + ((token < tokens ? token : tokens - 1) * rows.hidden_stride + P::OWN * g) * P::SIZE;
  }
  few_acc acc[2][NT];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[u][t] = few_acc{0.f, 0.f, 0.f, 0.f};
  struct Batch {
    P w[kAhead][2], h[kAhead][NT];
  };
  const long long batch = (long long)kAhead * P::COLS, whole = rows.width / batch * batch;
  const auto load = [&](long long k, Batch& b) {
#pragma unroll
    for (int c = 0; c < kAhead; ++c) {
#pragma unroll
      for (int u = 0; u < 2; ++u) b.w[c][u].load(w[u] + (k + c * P::COLS) * P::SIZE);
#pragma unroll
      for (int t = 0; t < NT; ++t) b.h[c][t].load(h[t] + (k + c * P::COLS) * P::SIZE);
    }
  };
  const auto take = [&](const Batch& b) {
#pragma unroll
    for (int c = 0; c < kAhead; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[u][t] = few_multiply<F32>(b.w[c][u], b.h[c][t], acc[u][t]);
  };
  // a batch is multiplied while the next one is on its way
  if (whole) {
    Batch b0, b1;
    load(0, b0);
    for (long long k = 0;;) {
      k += batch;
      const bool more = k < whole;
      if (more) load(k, b1);
      take(b0);
      if (!more) break;
      k += batch;
      const bool again = k < whole;
      if (again) load(k, b0);
      take(b1);
      if (!again) break;
    }
  }
  for (long long k = whole; k < rows.width; k += P::COLS) {           // the rest of the rows
    const long long left = rows.width - k - P::OWN * g;
    const int count = left < 0 ? 0 : left < P::OWN ? (int)left : P::OWN;
    P a[2], b[NT];
#pragma unroll
    for (int u = 0; u < 2; ++u) a[u].load_some(w[u] + k * P::SIZE, count);
#pragma unroll
    for (int t = 0; t < NT; ++t) b[t].load_some(h[t] + k * P::SIZE, count);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[u][t] = few_multiply<F32>(a[u], b[t], acc[u][t]);
  }
  // 16 tokens at a time through LDS; then 16 threads to a token, four to a group, eight entries each
  const int mine = threadIdx.x >> 4, c = threadIdx.x & 15, group = c >> 2, half = group & 1;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t) __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 32 * wave + 16 * u + 4 * g + e;
        zs[r * kPitch + row] = v0 + row < vocab ? acc[u][t][e] : -INFINITY;
      }
    __syncthreads();
    float z[8], first = -INFINITY, second = -INFINITY;
    int place = 8 * (c & 3);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = 8 * (c & 3) + e;
      z[e] = zs[mine * kPitch + 64 * (group >> 1) + place_row(at, half)];
      second = __builtin_amdgcn_fmed3f(first, second, z[e]);
      place = z[e] > first ? at : place;
      first = fmaxf(first, z[e]);
    }
#pragma unroll
    for (int off = 1; off < 4; off *= 2) {
      const float f = __shfl_xor(first, off, 64), s = __shfl_xor(second, off, 64);
      const int p = __shfl_xor(place, off, 64);
      second = fmaxf(fmaxf(second, s), fminf(first, f));
      place = f > first || (f == first && p < place) ? p : place;
      first = fmaxf(first, f);
    }
    float top = fmaxf(first, __shfl_xor(first, 4, 64));
    top = fmaxf(top, __shfl_xor(top, 8, 64));
    top = top == -INFINITY ? 0.f : unit * top;
    float sum = 0.f, slope = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = fmaf(unit, z[e], -top), x = __builtin_amdgcn_exp2f(y);
      sum += x;
      slope = fmaf(x, fmaxf(y, kFarBelow), slope);
    }
#pragma unroll
    for (int off = 1; off < 16; off *= 2) {
      sum += __shfl_xor(sum, off, 64);
      slope += __shfl_xor(slope, off, 64);
    }
    const long long token = 16 * t + mine, blocks = (vocab + kHeadGrain - 1) / kHeadGrain;
    if (token >= tokens) continue;
    if (BEST && (c & 3) == 0)
      best[(token * blocks + block) * (kHeadGrain / kScoreGroup) + group] = ScoreBest{first, (__float_as_uint(second) & ~31u) | (unsigned)place};
    if (c == 0) stats[token * blocks + block] = ScoreStats{top, sum, slope, 0.f};
  }
}

// ---- forward: one block per token joins the blocks and picks the alternatives ----
typedef unsigned long long u64;

// A value that a wave's lanes agree on, in scalar registers.
template <typename X>
__device__ __forceinline__ X same_in_all(X x) {
  static_assert(sizeof(X) == 8, "two words");
  u32x2 w = __builtin_bit_cast(u32x2, x);
  w.x = __builtin_amdgcn_readfirstlane(w.x);
  w.y = __builtin_amdgcn_readfirstlane(w.y);
  return __builtin_bit_cast(X, w);
}

// Threads, neighbours, that share one of n items: as many as there are, a power of two.
template <int NT>
__device__ __forceinline__ int sharers(int n) {
  int s = 1;
  while (s < 64 && 2 * s * n <= NT) s *= 2;
  return s;
}
// Sum over the `s` neighbours.
__device__ __forceinline__ int shared_sum(int x, int s) {
  for (int d = 1; d < s; d *= 2) x += __shfl_xor(x, d, 64);
  return x;
}

// Larger keys are larger values, then lower rows; 0 is none.
__device__ __forceinline__ unsigned rising(unsigned bits) { return bits ^ ((unsigned)((int)bits >> 31) | 0x80000000u); }
__device__ __forceinline__ u64 key_of(float z, unsigned row) { return (u64)rising(__float_as_uint(z)) << 32 | (0xffffffffu - row); }
__device__ __forceinline__ unsigned key_row(u64 key) { return 0xffffffffu - (unsigned)key; }
__device__ __forceinline__ float second_bound(unsigned w) { return __uint_as_float((int)w < 0 ? w & ~31u : w | 31u); }

constexpr int kPickGroups = 4096;                // groups whose keys stay in registers: all, up to 131072 vocabulary entries
constexpr int kPickList = 256;

// Bound by the chain of its memory accesses for a few tokens (8 x 32768 x 1024, top 5: 10 us), by the rows whose logits are summed again and the
// operations of the choice for many: 4096 x 100003 x 2048, top 8, 94 us, of which the statistics 16, the choice 36; 2048 x 32768 x 1024, top 64, 184.
// Blocks of 256 threads are held to registers for five waves: with four 138 and 249, with six, which spill, 169 and 284 us.
template <bool F32, bool PICK, int NT>
__global__ __launch_bounds__(NT, NT == 256 ? 5 : 1) void score_finish_kernel(ScoreTarget t, float inv_tau, float unit,
                                                                                const ScoreStats* __restrict__ stats, long long blocks,
                                                                                const ScoreBest* __restrict__ best, long long groups, int top, HeadRows rows,
                                                                                long long vocab, ScoreOut out) {
  constexpr int NW = NT / 64, kPickKeys = kPickGroups / NT;
  __shared__ float tops[NW];
  __shared__ double sums[2 * NW];
  __shared__ u64 bins[256], bound;               // PICK
  __shared__ int counts[2];
  extern __shared__ u64 dynamic[];               // PICK: a list of keys; logits and rows of the picks; the keys' seconds
  const long long token = blockIdx.x;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const auto larger = [](auto x, auto y) { return x > y ? x : y; };

  if constexpr (PICK) {
    if (tid < 256) bins[tid] = 0;
    if (tid < 2) counts[tid] = 0;
    if (tid == 0) bound = 0;
  }
  // the groups' largest, on their way while the sums are joined
  const ScoreBest* mine = best + token * groups;
  ScoreBest held[kPickKeys];
  if constexpr (PICK) {
    static_for<0, kPickKeys>([&](auto n) {
      constexpr int u = decltype(n)::value;
      const long long g = tid + NT * u;
      held[u] = g < groups ? mine[g] : ScoreBest{0.f, 0u};
    });
  }

  // lse and entropy: sums relative to the largest block's top, joined in double
  float m = -INFINITY, sum = 0.f, slope = 0.f;
  for (long long b0 = tid; b0 < blocks; b0 += 4 * NT) {
    ScoreStats v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = b0 + NT * u < blocks ? stats[token * blocks + b0 + NT * u] : ScoreStats{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (v[u].sum == 0.f) continue;
      const float now = fmaxf(m, v[u].top), down = m == -INFINITY ? 0.f : m - now, here = v[u].top - now, f = __builtin_amdgcn_exp2f(down),
                  h = __builtin_amdgcn_exp2f(here);
      slope = f * fmaf(sum, down, slope) + h * fmaf(v[u].sum, here, v[u].slope);
      sum = f * sum + h * v[u].sum;
      m = now;
    }
  }
  // the given token's logit: here, or, with picks, beside theirs
  const long long y = same_in_all(out.log_prob ? target_at(t, token) : -1);
  const bool there = y >= 0 && y < vocab;
  double given = 0.0;
  if (!PICK && there && wave == NW - 1)
    given = row_dot64<F32>(rows.hidden, token * rows.hidden_stride, rows.weight, y * rows.weight_stride, rows.width);
  const float wave_top = wave_all(m, larger);
  if (lane == 0) tops[wave] = wave_top;
  __syncthreads();
  float all = tops[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) all = fmaxf(all, tops[w]);
  if (all == -INFINITY) all = 0.f;
  const double down = m == -INFINITY ? 0.0 : (double)m - (double)all, f = m == -INFINITY ? 0.0 : (double)__builtin_amdgcn_exp2f((float)down);
  const double s0 = wave_all(f * sum, Add{}), e0 = wave_all(f * (slope + sum * down), Add{});
  if (lane == 0) sums[wave] = s0, sums[NW + wave] = e0;
  __syncthreads();
  double mass = 0.0, tilt = 0.0;
#pragma unroll
  for (int w = 0; w < NW; ++w) mass += sums[w], tilt += sums[NW + w];
  const double per = (double)inv_tau / (double)unit, l2 = log2(mass), lse = same_in_all(per * ((double)all + l2));
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
  if (out.log_prob && tid == NT - 64 && !(PICK && there)) out.log_prob[token] = y < 0 ? 0.f : y >= vocab ? __builtin_nanf("") : log_prob(given);

  if constexpr (PICK) {
    const int pick = top + kScoreMargin;
    u64* list = dynamic;                                 // [kPickList]
    u64* rank_of = list + kPickList;                     // [33 pick]
    double* value = reinterpret_cast<double*>(rank_of + 33 * pick);    // [33 pick]
    int* row_of = reinterpret_cast<int*>(value + 33 * pick);           // [33 pick]
    int* open = row_of + 33 * pick;                      // [pick], rows whose groups are looked through
    unsigned* seconds = reinterpret_cast<unsigned*>(open + pick);      // [kPickList], of the list
    const auto key_at = [&](long long g, ScoreBest b) -> u64 {
      const long long row = 64 * (g >> 1) + place_row((int)(b.second & 31u), (int)(g & 1));
      return row < vocab && g < groups && 64 * (g >> 1) + 4 * (g & 1) < vocab ? key_of(b.z, (unsigned)row) : 0;
    };
    u64 keys[kPickKeys];
    static_for<0, kPickKeys>([&](auto n) {
      constexpr int u = decltype(n)::value;
      keys[u] = key_at(tid + NT * u, held[u]);
    });
    // f(key, second) of each of the thread's groups
    const auto each = [&](auto&& f) {
      static_for<0, kPickKeys>([&](auto n) { f(keys[decltype(n)::value], held[decltype(n)::value].second); });
      for (long long g = tid + NT * kPickKeys; g < groups; g += NT) {
        const ScoreBest b = mine[g];
        f(key_at(g, b), b.second);
      }
    };
    // A bound that at least `pick` keys reach: of the largest keys of 64 (for many picks 256) shares of the groups the pick-th largest.
    u64 own = 0;
    each([&](u64 key, unsigned) { own = larger(own, key); });
    const bool coarse = pick <= 32;
    const int shares = coarse ? 64 : 256;
    if (own) atomicMax(&bins[tid % shares], own);
    __syncthreads();
    {
      const int s = NT / shares, i = tid / s;
      const u64 share = bins[i];
      int rank = 0;
#pragma unroll 8
      for (int k = tid % s; k < shares; k += s) rank += bins[k] > share;
      rank = shared_sum(rank, s);
      if (share && rank == pick - 1) bound = share;
    }
    __syncthreads();
    const auto collect = [&](u64 from) {
      each([&](u64 key, unsigned second) {
        if (key && key >= from) {
          const int at = atomicAdd(&counts[0], 1);
          if (at < kPickList) list[at] = key, seconds[at] = second;
        }
      });
    };
    collect(bound);
    __syncthreads();
    if (counts[0] > kPickList) {                         // a few shares hold most of the largest: the bound bit by bit instead
      u64 from = 0;
      for (int bit = 63; bit >= 0; --bit) {
        const u64 tried = from | 1ull << bit;
        __syncthreads();
        if (tid == 0) counts[0] = 0;
        __syncthreads();
        int n = 0;
        each([&](u64 key, unsigned) { n += key >= tried; });
        n = wave_all(n, Add{});
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
    // the picks, by the threads that hold them: their rows, and all rows of a group whose second may be among the largest as well
    u64 key = 0;
    int rank = 0;
    const int s = sharers<NT>(n), item = tid / s;
    const bool holds = item < n && tid % s == 0;
    if (item < n) {
      key = list[item];
#pragma unroll 8
      for (int k = tid % s; k < n; k += s) rank += list[k] > key;
      rank = shared_sum(rank, s);
      if (rank == pick - 1) bound = key;
    }
    if (tid == 0 && n < pick) bound = 0;
    const int have = n < pick ? n : pick;
    __syncthreads();
    if (holds && rank < pick) {
      const unsigned row = key_row(key);
      row_of[rank] = (int)row;
      if (((u64)rising(__float_as_uint(second_bound(seconds[item]))) << 32 | 0xffffffffu) >= bound) open[atomicAdd(&counts[1], 1)] = (int)row;
    }
    __syncthreads();
    const int c = have + 32 * counts[1];
    for (int i = have + tid; i < c; i += NT) {
      const int row = open[(i - have) / 32], other = row / 64 * 64 + place_row((i - have) % 32, (row >> 2) & 1);
      row_of[i] = other != row && other < vocab ? other : -1;
    }
    __syncthreads();
    // the picks' logits and, behind them, the given token's; several rows of a wave at a time where there are more than waves
    const int all_rows = c + there;
    const auto sum_rows = [&](auto many) {
      constexpr int U = decltype(many)::value;
      for (int i0 = U * wave; i0 < all_rows; i0 += U * NW) {
        double z[U];
        long long at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u, row = i < c ? row_of[i] : i == c && there ? (int)y : -1;
          z[u] = 0.0;
          at[u] = (row < 0 ? 0 : row) * rows.weight_stride;
        }
        for (long long k = lane * 8; k + 8 <= rows.width; k += 512) {
          const Raw8<F32> x = load_raw8<F32>(rows.hidden, token * rows.hidden_stride, k);
          Raw8<F32> w[U];
#pragma unroll
          for (int u = 0; u < U; ++u) w[u] = load_raw8<F32>(rows.weight, at[u], k);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            __builtin_amdgcn_sched_barrier(0);           // a row after the other: doubles of all would not fit the registers
#pragma unroll
            for (int e = 0; e < 8; ++e) z[u] = fma(raw_value(x, e), raw_value(w[u], e), z[u]);
          }
        }
        if (lane < (int)(rows.width & 7)) {              // the last elements, one per lane
          const long long k = rows.width / 8 * 8 + lane;
          const double x = load_one<F32>(rows.hidden, token * rows.hidden_stride + k);
#pragma unroll
          for (int u = 0; u < U; ++u) z[u] = fma(x, (double)load_one<F32>(rows.weight, at[u] + k), z[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          z[u] = wave_all(z[u], Add{});
          const int i = i0 + u;
          if (lane != 0 || i > c) continue;
          if (i < c) {
            value[i] = z[u];
            const u64 bits = __double_as_longlong(z[u]);   // larger for larger logits, 0 for NaN and where there is no row
            rank_of[i] = row_of[i] < 0 || z[u] != z[u] ? 0 : bits ^ ((u64)((long long)bits >> 63) | 0x8000000000000000ull);
          } else if (there) {
            out.log_prob[token] = log_prob(z[u]);
          }
        }
      }
    };
    if (all_rows <= NW) sum_rows(std::integral_constant<int, 1>{});
    else sum_rows(std::integral_constant<int, 4>{});
    __syncthreads();
    const int s2 = sharers<NT>(c);
    for (int i = tid / s2; i < c; i += NT / s2) {
      const int row = row_of[i];
      const u64 mine_is = rank_of[i];
      int ahead = 0;
#pragma unroll 8
      for (int k = tid % s2; k < c; k += s2) {             // (no row, -1, is the largest)
        const unsigned other = row_of[k];
        const u64 is = rank_of[k];
        ahead += (int)(is > mine_is) | ((int)(is == mine_is) & (int)(other < (unsigned)row));
      }
      ahead = shared_sum(ahead, s2);
      if (row >= 0 && ahead < top && tid % s2 == 0) {
        out.top_index[token * top + ahead] = row;
        out.top_log_prob[token * top + ahead] = log_prob(value[i]);
      }
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

// The largest finite |gradient| of so many tokens, or 1, in every thread of the block.
template <int THREADS>
__device__ __forceinline__ float peak_of(const ScoreTarget& t, const ScoreGrads& d, long long tokens, long long vocab) {
  __shared__ float waves[THREADS / 64];
  float top = 0.f;
  for (long long i = threadIdx.x; i < tokens; i += THREADS) {
    const Given x = given(t, d, i, vocab);
    if (fabsf(x.g) < INFINITY) top = fmaxf(top, fabsf(x.g));
    if (fabsf(x.h) < INFINITY) top = fmaxf(top, fabsf(x.h));
  }
  top = wave_all(top, [](float x, float y) { return fmaxf(x, y); });
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) top = fmaxf(top, waves[w]);
  return top > 0.f ? top : 1.f;
}

__global__ __launch_bounds__(1024) void score_peak_kernel(ScoreTarget t, ScoreGrads d, long long tokens, long long vocab, float* __restrict__ peak) {
  const float top = peak_of<1024>(t, d, tokens, vocab);
  if (threadIdx.x == 0) *peak = top;
}

// Up to so many tokens every block of the preparation looks through all of them itself, a launch less (2048 tokens: 17.6 us in one, 8.2 + 5.2 in two).
constexpr long long kPeakInPrepare = 512;

template <bool F32>
__global__ __launch_bounds__(256) void score_prepare_kernel(ScoreTarget t, float inv_tau, float unit, ScoreGrads d, float* __restrict__ peak, HeadRows rows,
                                                            long long tokens, long long vocab, ScoreCoef c, u16* __restrict__ masked, long long ld, long long plane) {
  const long long token = blockIdx.x, at = token * rows.hidden_stride;
  const bool own = tokens <= kPeakInPrepare;
  const float largest = own ? peak_of<256>(t, d, tokens, vocab) : *peak;
  if (own && token == 0 && threadIdx.x == 0) *peak = largest;
  const Given x = given(t, d, token, vocab);
  const bool some = x.g != 0.f || x.h != 0.f;            // (NaN counts)
  if (threadIdx.x < 64) {
    float a = 0.f, b = 0.f, value = 0.f;
    float2 l2 = make_float2(INFINITY, 0.f);
    if (some) {
      const double per = 1.0 / (double)largest, g = per * x.g, h = per * x.h, lse = (double)d.lse[token] + (double)d.lse_rest[token],
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
      // logits that are NaN or infinite: no gradient of the token is a number.  (The powers alone would not say so: a NaN exponent is cut off at
      // kFarBelow; and an infinite sum stands for a token without gradients.)
      if (!(fabsf(l2.x) < INFINITY)) a = value = l2.x = __builtin_nanf("");
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

// dz is rounded to bf16 (fp32: to three planes of it) as the operand of two products on the matrix cores.  That and their own rounding, 1.7e-3 of the norm
// each, are what bf16 gradients are off by, 2.4e-3.
//
// The logits' gradient from what the forward call kept, by spans of a token's row.  Bound by memory: 2 bytes in and 2 out, fp32 4 and 6.
// What is kept is read with the streaming hint, which leaves the memory-side cache to the gradient that two products read next (scores and gradients of
// 2048 x 32768 x 1024: 507 us without, 477 with; of 8192 x 100003 x 2048 the same).  6.2 TB/s at the latter.
constexpr int kDzSpan = 4096;
template <bool F32>
__global__ __launch_bounds__(256) void score_dz_kernel(ScoreTarget t, float unit, ScoreKept kept, long long blocks, ScoreCoef c, long long vocab, int spans,
                                                       u16* __restrict__ grad, long long pitch, long long plane) {
  const long long token = blockIdx.x / spans, v0 = (long long)(blockIdx.x % spans) * kDzSpan, row = token * pitch;
  const float a = c.a[token], b = c.b[token];
  const float2 l2 = c.log2sum[token];
  const bool some = l2.x < INFINITY || l2.x != l2.x;     // (infinite: no gradient)
  for (long long v = v0 + threadIdx.x * 8; v < v0 + kDzSpan && v < pitch; v += 2048) {
    Row8 r{};
    if (some && v < vocab) {
      float y[8], p[8];
      if constexpr (F32) {
        const f32x4* z = reinterpret_cast<const f32x4*>(static_cast<const float*>(kept.values) + row + v);
        const f32x4 two[2] = {__builtin_nontemporal_load(z), __builtin_nontemporal_load(z + 1)};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] = fmaxf(fmaf(unit, two[e / 4][e % 4], -l2.x) - l2.y, kFarBelow);
          p[e] = __builtin_amdgcn_exp2f(y[e]);
        }
      } else {
        const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const u16*>(kept.values) + row + v));
        const float shift = ((kept.tops[token * blocks + v / kHeadGrain] - l2.x) - l2.y) - kProbTop, f = __builtin_amdgcn_exp2f(shift);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const unsigned pair = w[e / 2];                // (a bit cast of the vector's element itself would take its first)
          const f16x2 both = __builtin_bit_cast(f16x2, pair);
          const float x = (float)both[e & 1];
          p[e] = f * x;
          y[e] = b == 0.f ? 0.f : fmaxf(__builtin_amdgcn_logf(x) + shift, kFarBelow);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) r.v[e] = v + e < vocab ? -p[e] * fmaf(b, y[e], a) : 0.f;
    }
    store_planes8<F32>(r, grad + row + v, plane);
  }
  if (!some || !t.index) return;
  __syncthreads();                                       // the target's entry goes over what this block wrote
  const long long y = target_at(t, token);
  if (threadIdx.x == 0 && y >= v0 && y < v0 + kDzSpan && y < vocab) {
    float x = c.value[token];
#pragma unroll
    for (int q = 0; q < (F32 ? 3 : 1); ++q) {
      const u16 bits = bf16_bits(x);
      grad[q * plane + row + y] = bits;
      x -= bf16_value(bits);
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
  // fp32: a plane after the other, each from the accumulators themselves; kept remainders would not fit the registers
#pragma unroll 1
  for (int p = 0; p < (F32 ? 3 : 1); ++p) {
    if (F32 && p) __syncthreads();                       // the image has left
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const long long token = col0 + tile.wn * T::WN + 32 * j + fr;
      float a = 0.f, b = 0.f;
      float2 l2 = make_float2(INFINITY, 0.f);
      if (token < hidden.rows) {
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
            const float y = fmaxf(fmaf(unit, tile.acc[i][j][4 * q + e], -l2.x) - l2.y, kFarBelow);
            x[e] = -__builtin_amdgcn_exp2f(y) * fmaf(b, y, a);
          }
          if (there < T::WM) {                           // what ends the logits' rows is zero
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (32 * i + 8 * q + 4 * fh + e >= there) x[e] = 0.f;
          }
          u32x2 w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
          if constexpr (F32) {
            for (int k = 0; k < p; ++k) {                // what the planes before leave
              x[0] -= bf16_lo(w.x), x[1] -= bf16_hi(w.x), x[2] -= bf16_lo(w.y), x[3] -= bf16_hi(w.y);
              w = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
            }
          }
          tile.put(smem, i, j, q, w);
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

template <int B, int S, bool BEST, int KEEP>
hipError_t score_logits_of(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, ScoreStats* stats,
                           ScoreBest* best, const ScoreKept& kept, hipStream_t s) {
  constexpr int lds = Tile<B, B, false, false, S>::kLds;
  static std::atomic<uint64_t> done{0};
  if (hipError_t e = allow_lds(done, reinterpret_cast<const void*>(&score_logits_kernel<B, S, BEST, KEEP>), lds)) return e;
  score_logits_kernel<B, S, BEST, KEEP><<<(unsigned)g.blocks(), 256, lds, s>>>(weight, hidden, tiles_of(g, pairs), unit, stats, best, kept);
  return hipGetLastError();
}

hipError_t launch_score_logits(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, ScoreStats* stats,
                               ScoreBest* best, const ScoreKept& kept, hipStream_t s) {
#define MUON_SCORE_CASE(B, S)                                                                                                       \
  if (g.tile == B && (g.alone ? 4 : 2) == S)                                                                                        \
    return best          ? score_logits_of<B, S, true, 0>(weight, hidden, g, pairs, unit, stats, best, kept, s)                     \
           : !kept.values ? score_logits_of<B, S, false, 0>(weight, hidden, g, pairs, unit, stats, best, kept, s)                   \
           : kept.tops    ? score_logits_of<B, S, false, 1>(weight, hidden, g, pairs, unit, stats, best, kept, s)                   \
                          : score_logits_of<B, S, false, 2>(weight, hidden, g, pairs, unit, stats, best, kept, s)
  MUON_SCORE_CASE(256, 2);
  MUON_SCORE_CASE(128, 2);
  MUON_SCORE_CASE(128, 4);
#undef MUON_SCORE_CASE
  return hipErrorInvalidValue;
}

hipError_t launch_score_few(const HeadRows& rows, long long tokens, long long vocab, float unit, ScoreStats* stats, ScoreBest* best, hipStream_t s) {
  const long long blocks = (vocab + kHeadGrain - 1) / kHeadGrain;
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)blocks, 256, 0, s>>>(rows, tokens, vocab, unit, stats, best);
    return hipGetLastError();
  };
  if (!rows.f32) return best ? go(score_few_kernel<false, 1, true>) : go(score_few_kernel<false, 1, false>);
  if (tokens <= 16) return best ? go(score_few_kernel<true, 1, true>) : go(score_few_kernel<true, 1, false>);
  if (tokens <= 32) return best ? go(score_few_kernel<true, 2, true>) : go(score_few_kernel<true, 2, false>);
  return best ? go(score_few_kernel<true, 4, true>) : go(score_few_kernel<true, 4, false>);
}

hipError_t launch_score_finish(const ScoreTarget& t, float inv_tau, float unit, const ScoreStats* stats, long long blocks,
                               const ScoreBest* best, long long groups, int top, const HeadRows& rows, long long tokens, long long vocab, const ScoreOut& out,
                               hipStream_t s) {
  const unsigned lds = top ? (top + kScoreMargin) * (33 * 20 + 4) + kPickList * 12 : 0;
  auto go = [&](auto kernel, int threads) {
    kernel<<<(unsigned)tokens, threads, lds, s>>>(t, inv_tau, unit, stats, blocks, best, groups, top, rows, vocab, out);
    return hipGetLastError();
  };
  if (!top) return rows.f32 ? go(score_finish_kernel<true, false, 256>, 256) : go(score_finish_kernel<false, false, 256>, 256);
  // Few tokens: threads enough to fill the chip with one block or two per compute unit.  Calls with 8 alternatives in graphs, us, with 256, 512 and 1024
  // threads: 32768 x 1024 with 8 tokens 28.2, 25.4, 25.7, 192 38.7, 33.0, 31.9, 256 35.2, 32.5, 32.6, 320 46.7, 45.2, 50.9, 512 54.6, 50.3, 57.2, 1024 94.4,
  // 94.6, 110.4; 100003 x 2048 with 64 123.2, 119.0, 118.2, 256 167.1, 160.8, 161.3, 512 226.2, 225.0, 229.5, 1024 409.5, 408.3, 419.7.
  if (tokens <= 256) return rows.f32 ? go(score_finish_kernel<true, true, 1024>, 1024) : go(score_finish_kernel<false, true, 1024>, 1024);
  if (tokens <= 512) return rows.f32 ? go(score_finish_kernel<true, true, 512>, 512) : go(score_finish_kernel<false, true, 512>, 512);
  return rows.f32 ? go(score_finish_kernel<true, true, 256>, 256) : go(score_finish_kernel<false, true, 256>, 256);
}

hipError_t launch_score_peak(const ScoreTarget& t, const ScoreGrads& d, long long tokens, long long vocab, float* peak, hipStream_t s) {
  if (tokens <= kPeakInPrepare) return hipSuccess;         // launch_score_prepare finds it
  score_peak_kernel<<<1, 1024, 0, s>>>(t, d, tokens, vocab, peak);
  return hipGetLastError();
}

hipError_t launch_score_prepare(const ScoreTarget& t, float inv_tau, float unit, const ScoreGrads& d, float* peak, const HeadRows& rows,
                                long long tokens, long long vocab, const ScoreCoef& c, uint16_t* masked, long long ld, long long plane, hipStream_t s) {
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)tokens, 256, 0, s>>>(t, inv_tau, unit, d, peak, rows, tokens, vocab, c, masked, ld, plane);
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

hipError_t launch_score_dz(const ScoreTarget& t, float unit, const ScoreKept& kept, long long blocks, const ScoreCoef& c, long long tokens, long long vocab, bool f32,
                           uint16_t* grad, long long pitch, long long plane, hipStream_t s) {
  const int spans = (int)((pitch + kDzSpan - 1) / kDzSpan);
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)(tokens * spans), 256, 0, s>>>(t, unit, kept, blocks, c, vocab, spans, grad, pitch, plane);
    return hipGetLastError();
  };
  return f32 ? go(score_dz_kernel<true>) : go(score_dz_kernel<false>);
}

}  // namespace muon
