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

// The largest power of a block is 2^15, high in f16's range: 2^-11 of relative precision holds down to 2^-29 of it.
constexpr float kProbTop = 15.f;

// The planes of the pair with that number: (0,0) alone, or (0,2) (2,0) (1,1) (0,1) (1,0) (0,0), the smallest first, so that they do not
// add their roundings to the large sum; what is left out is below 2^-24.
__device__ __forceinline__ int pair_left(int pairs, int pair) { return pairs == 1 ? 0 : (0x021010 >> 4 * (5 - pair)) & 15; }
__device__ __forceinline__ int pair_right(int pairs, int pair) { return pairs == 1 ? 0 : (0x201100 >> 4 * (5 - pair)) & 15; }

typedef __attribute__((address_space(3))) void* lptr;

// f(integral_constant<int, I>) for I = FIRST .. LAST-1, unrolled at compile time
template <int FIRST, int LAST, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (FIRST < LAST) {
    f(std::integral_constant<int, FIRST>{});
    static_for<FIRST + 1, LAST>(f);
  }
}

// The tile of block b of n: blocks go to the eight dies in turn, so each die is given a run of tiles, and a run goes through bands of
// eight columns row by row: the 32 tiles that run together on a die share four panels of L and eight of R in its L2.
struct TileAt {
  int m, n, split;
  int quarter;              // -1: the whole tile
};
__device__ __forceinline__ TileAt tile_at(const HeadTiles& g) {
  const int all = g.whole * g.splits, b = blockIdx.x;
  int t, split = 0, quarter = -1;
  if (b < all) {
    const int die = b & 7, per = all >> 3, rest = all & 7;
    t = die * per + (die < rest ? die : rest) + (b >> 3);
    split = t / g.whole;
    t -= split * g.whole;
  } else {                  // (splits = 1)
    t = g.whole + (b - all) / 4;
    quarter = (b - all) % 4;
  }
  constexpr int kBand = 8;
  const int band = t / (kBand * g.tiles_m), wide = g.tiles_n - band * kBand < kBand ? g.tiles_n - band * kBand : kBand;
  t -= band * kBand * g.tiles_m;
  return {t / wide, band * kBand + t % wide, split, quarter};
}

// Fragments of F rows of 32 for one k-step of 16, as LDS reads deliver them.
template <bool KM, int F>
struct Frag;
template <int F>
struct Frag<false, F> {
  u32x4 v[F];
  __device__ __forceinline__ bf16x8 at(int i) const { return __builtin_bit_cast(bf16x8, v[i]); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < F; ++i) v[i] = u32x4{0u, 0u, 0u, 0u};
  }
  // "these registers hold what the reads before the last wait have brought": what multiplies them cannot be moved ahead of it
  __device__ __forceinline__ void tie() {
    if constexpr (F == 4) asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]) : : "memory");
    else asm volatile("" : "+v"(v[0]), "+v"(v[1]) : : "memory");
  }
};
template <int F>
struct Frag<true, F> {
  u32x2 v[F][2];
  __device__ __forceinline__ bf16x8 at(int i) const {
    const u32x4 both = {v[i][0].x, v[i][0].y, v[i][1].x, v[i][1].y};
    return __builtin_bit_cast(bf16x8, both);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < F; ++i) v[i][0] = v[i][1] = u32x2{0u, 0u};
  }
  __device__ __forceinline__ void tie() {
    if constexpr (F == 4)
      asm volatile(""
                   : "+v"(v[0][0]), "+v"(v[0][1]), "+v"(v[1][0]), "+v"(v[1][1]), "+v"(v[2][0]), "+v"(v[2][1]), "+v"(v[3][0]), "+v"(v[3][1])
                   :
                   : "memory");
    else asm volatile("" : "+v"(v[0][0]), "+v"(v[0][1]), "+v"(v[1][0]), "+v"(v[1][1]) : : "memory");
  }
};

// One operand's share of a tile of B of its rows: where its slabs come from, how they lie in LDS, how fragments are read.  A wave
// instruction moves 1 KB from memory to LDS: 8 rows of 128 bytes, 16-byte chunks at position chunk ^ (row / 2) % 8, or, K-major, whole
// k-rows of 2 B bytes, chunks at position chunk ^ 4 (k-row % 4); so that the reads of a k-step meet every bank alike.  Loads go through
// a buffer descriptor that ends where the operand does: rows and k-rows behind its end arrive as zeros.
template <int B, int W, int F, bool KM>      // rows; rows of a wave = 32 F at W * (wave's place)
struct Side {
  static constexpr int NW = 4, LOADS = B / 8 / NW, READS = KM ? 2 * F : F;
  static constexpr int CHUNKS = B / 8, KROWS = 64 / CHUNKS;        // K-major: chunks of a k-row, k-rows per wave instruction
  const u16* base;        // element (row0, 0) or, K-major, (0, row0)
  long long slab;         // elements from one slab to the next
  long long plane;
  unsigned step;          // bytes from one load of a wave to its next
  unsigned offset;        // of the lane's chunk in a slab
  unsigned rows_bytes;    // descriptor's size at k = 0 for the rows there are (plain)
  long long ld;
  unsigned tail;          // K-major: bytes of the last k-row from row0 on
  int chunk;              // plain: the lane's chunk, 8 elements of K
  unsigned read[KM ? F : 4];

  __device__ __forceinline__ void init(const HeadOperand& o, long long row0, long long k, int wave, int lane, int place, unsigned lds) {
    const int fr = lane & 31, fh = lane >> 5;
    ld = o.ld;
    plane = o.plane;
    if constexpr (KM) {
      base = o.p + row0;
      const int row = wave * KROWS + lane / CHUNKS;
      offset = (unsigned)((row * o.ld + ((lane % CHUNKS) ^ (4 * (row & 3))) * 8) * 2);
      step = (unsigned)(NW * KROWS * o.ld * 2);
      slab = kHeadSlab * o.ld;
      const long long left = (o.rows + 7) / 8 * 8 - row0;
      tail = (unsigned)(2 * (left < 0 ? 0 : left));
      // the 16 lanes of a group each address 8 bytes of a 4 (k) x 16 block and receive one column's 4 consecutive k
      const int l16 = lane & 15, g = lane >> 4, r4 = l16 >> 2;
#pragma unroll
      for (int i = 0; i < F; ++i)
        read[i] = lds + (8 * (g >> 1) + r4) * (B * 2) + ((((place * (W / 8) + 4 * i) ^ (4 * r4)) + 2 * (g & 1) + ((l16 & 3) >> 1)) * 16) + (l16 & 1) * 8;
    } else {
      base = o.p + row0 * o.ld;
      const int row = wave * 8 + (lane >> 3);
      chunk = (lane & 7) ^ ((row >> 1) & 7);
      offset = (unsigned)((row * o.ld + chunk * 8) * 2);
      step = (unsigned)(8 * NW * o.ld * 2);
      slab = kHeadSlab;
      const long long left = o.rows - row0, rows = left < B ? left : B;
      rows_bytes = rows <= 0 ? 0u : (unsigned)(((rows - 1) * o.ld + (k + 7) / 8 * 8) * 2);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) read[kk] = lds + (place * W + fr) * 128 + (((2 * kk + fh) ^ ((fr >> 1) & 7)) * 16);
    }
  }
  // The slab that is loaded next: its descriptor's base and size, the lane's offset in it.
  const u16* at;
  int bytes;
  unsigned here;
  __device__ __forceinline__ void clip(int left) {                    // left: elements of K from this slab on, fewer than a slab
    if constexpr (KM) bytes = (int)((unsigned)(left - 1) * (unsigned)(ld * 2) + tail);
    else here = chunk * 8 >= left ? 0x80000000u : offset;             // behind K: out of the descriptor's range
  }
  __device__ __forceinline__ void start(int p, int kt, long long k) {
    at = base + p * plane + kt * slab;
    here = offset;
    if constexpr (KM) bytes = (int)((unsigned)(kHeadSlab - 1) * (unsigned)(ld * 2) + tail);
    else bytes = (int)(rows_bytes - (unsigned)kt * (kHeadSlab * 2));
    if (k - (long long)kt * kHeadSlab < kHeadSlab) clip((int)(k - (long long)kt * kHeadSlab));
  }
  __device__ __forceinline__ void advance(int left) {
    at += slab;
    if constexpr (!KM) bytes -= kHeadSlab * 2;
    if (left < kHeadSlab) clip(left);
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t source() const { return __builtin_amdgcn_make_buffer_rsrc(const_cast<u16*>(at), 0, bytes, 0x00020000); }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, int n, unsigned char* lds, int wave) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lptr)(lds + wave * 1024 + n * NW * 1024), 16, here + n * step, 0, 0, 0);
  }
  // Read number n of k-step KK from the stage that lies `stage` bytes behind the first.
  template <int KK, int N>
  __device__ __forceinline__ void fetch(Frag<KM, F>& f, unsigned stage) const {
    if constexpr (KM) {
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(f.v[N / 2][N % 2]) : "v"(read[N / 2] + stage), "n"((16 * KK + 4 * (N % 2)) * (B * 2)) : "memory");
    } else {
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f.v[N]) : "v"(read[KK] + stage), "n"(N * 32 * 128) : "memory");
    }
  }
};

template <int N>
__device__ __forceinline__ void wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(%0)" : : "n"(N) : "memory");
}

// At most N loads of this wave on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// A BM x BN tile of T = L R^T by four waves in 2 x 2: acc[i][j] of a wave holds, in lane (r, h), column 32 j + r and rows
// 32 i + 8 q + 4 h + e.  A ring of S stages of LDS, 64 of K each.  Two stages (what fills the chip): the loop is skewed by one k-step of 16 so that no product waits for LDS: in
// iteration kt (slab kt in stage `cur`, its first fragments in registers)
//   A  products of k-step 3 of slab kt - 1 | reads of k-step 1
//   B  products of k-step 0                | reads of k-steps 2, 3; then: my reads of `cur` and my loads of slab kt + 1 are done; barrier
//   C  products of k-steps 1, 2            | loads of slab kt + 2 into `cur`, reads of k-step 0 of slab kt + 1
// Four stages (a tile of 128 that has a compute unit to itself, whose phases would be too short to hide LDS and whose slabs would be waited
// for): all fragments of slab kt + 1 are read behind the first half of the products of slab kt, with two to three slabs on their way.
// One instruction of each kind between two products, never in bursts; the order is held by scheduling fences.  LDS reads are written in
// assembly (the compiler puts a wait for all loads in front of its own transposing read) and waited for by hand.
template <int BM_, int BN_, bool LKM, bool RKM, int S = 2>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = BM / 2, WN = BN / 2, FM = WM / 32, FN = WN / 32;
  static constexpr int kStage = (BM + BN) * 128, kLds = S * kStage;
  using L = Side<BM, WM, FM, LKM>;
  using R = Side<BN, WN, FN, RKM>;
  f32x16 acc[FM][FN];
  int lane, wave, wm, wn;

  __device__ __forceinline__ void run(const HeadOperand& lo, const HeadOperand& ro, long long row0, long long col0, long long k, int pairs, int first,
                                      int last, unsigned char* smem) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave >> 1;
    wn = wave & 1;
    const unsigned lds0 = (unsigned)(size_t)(lptr)smem;
    L l;
    R r;
    l.init(lo, row0, k, wave, lane, wm, lds0);
    r.init(ro, col0, k, wave, lane, wn, lds0 + BM * 128);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // A slab after the other; the descriptors move along with the loop, what K's end and the next pair of planes take is done where it occurs.
    const int per_pair = (int)((k + kHeadSlab - 1) / kHeadSlab);
    int pair = first / per_pair, ahead = (int)(k - (long long)(first - pair * per_pair) * kHeadSlab);       // of K from the next slab on
    l.start(pair_left(pairs, pair), first - pair * per_pair, k);
    r.start(pair_right(pairs, pair), first - pair * per_pair, k);
    auto take_next = [&]() {
      ahead -= kHeadSlab;
      if (ahead > 0) {
        l.advance(ahead);
        r.advance(ahead);
      } else {
        ++pair;
        ahead = (int)k;
        l.start(pair_left(pairs, pair), 0, k);
        r.start(pair_right(pairs, pair), 0, k);
      }
    };
    constexpr int LOADS = L::LOADS + R::LOADS;
    auto load_one = [&](int stage, int n) {
      if (n < L::LOADS) l.load(l.source(), n, smem + stage * kStage, wave);
      else r.load(r.source(), n - L::LOADS, smem + stage * kStage + BM * 128, wave);
    };
    const int count = last - first;
    static_for<0, S>([&](auto n_tag) {
      constexpr int n = decltype(n_tag)::value;
      if (n < count) {
        if constexpr (n > 0) take_next();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) load_one(n, u);
      }
    });
    if (count >= S) wait_loads<(S - 1) * LOADS>();                    // slab 0 has landed
    else wait_loads<0>();
    __syncthreads();

    constexpr int READS = L::READS + R::READS, MT = FM * FN;
    using std::integral_constant;
    if constexpr (S == 2) {
      Frag<LKM, FM> a[4];
      Frag<RKM, FN> b[4];
      auto read = [&](int stage, auto kk, auto n) {
        constexpr int KK = decltype(kk)::value, N = decltype(n)::value;
        if constexpr (N < L::READS) l.template fetch<KK, N>(a[KK], stage * kStage);
        else r.template fetch<KK, N - L::READS>(b[KK], stage * kStage);
      };
      auto multiply = [&](int kk, int t) {
        acc[t / FN][t % FN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[kk].at(t / FN), b[kk].at(t % FN), acc[t / FN][t % FN], 0, 0, 0);
      };
      a[3].zero();                                                      // the first pass of phase A multiplies zeros
      b[3].zero();
      static_for<0, READS>([&](auto n) { read(0, integral_constant<int, 0>{}, n); });

      int cur = 0;
      auto iteration = [&](auto refill_tag, auto sync_tag) {
        constexpr bool REFILL = decltype(refill_tag)::value, SYNC = decltype(sync_tag)::value;
        static_for<0, MT>([&](auto t_tag) {                             // A
          constexpr int t = decltype(t_tag)::value;
          multiply(3, t);
          static_for<t * READS / MT, (t + 1) * READS / MT>([&](auto n) { read(cur, integral_constant<int, 1>{}, n); });
          __builtin_amdgcn_sched_barrier(0);
        });
        wait_lds<(READS < 15 ? READS : 15)>();  // B: k-step 0 is in, k-step 1 may be on its way
        a[0].tie();
        b[0].tie();
        __builtin_amdgcn_sched_barrier(0);
        constexpr int LEAD = MT >= 8 ? 2 : 0, GROUPS = MT >= 8 ? 8 : 4;
        static_for<0, MT>([&](auto t_tag) {
          constexpr int t = decltype(t_tag)::value;
          constexpr int g = t - LEAD;
          if constexpr (g >= 0 && g < GROUPS) {
            static_for<g * 2 * READS / GROUPS, (g + 1) * 2 * READS / GROUPS>([&](auto n) {
              constexpr int N = decltype(n)::value;
              read(cur, integral_constant<int, 2 + N / READS>{}, integral_constant<int, N % READS>{});
            });
          }
          multiply(0, t);
          __builtin_amdgcn_sched_barrier(0);
        });
        wait_lds<0>();
#pragma unroll
        for (int kk = 1; kk < 4; ++kk) {
          a[kk].tie();
          b[kk].tie();
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (SYNC) {
          wait_loads<0>();                                              // my loads of slab kt + 1 have landed
          __builtin_amdgcn_s_barrier();                                 // everybody's; and nobody reads stage `cur` any more
        }
        constexpr int NC = 2 * MT;
        static_for<0, NC>([&](auto t_tag) {                             // C
          constexpr int t = decltype(t_tag)::value;
          multiply(1 + t / MT, t % MT);
          if constexpr (REFILL && t == 0) take_next();                // (in the shadow of a product)
          if constexpr (REFILL) {
#pragma unroll
            for (int n = t * LOADS / NC; n < (t + 1) * LOADS / NC; ++n) load_one(cur, n);
          }
          if constexpr (SYNC)
            static_for<t * READS / NC, (t + 1) * READS / NC>([&](auto n) { read(cur ^ 1, integral_constant<int, 0>{}, n); });
          __builtin_amdgcn_sched_barrier(0);
        });
        cur ^= 1;
      };
      int left = count;
      while (left > 2) {
        iteration(std::true_type{}, std::true_type{});
        --left;
      }
      if (left > 1) iteration(std::false_type{}, std::true_type{});
      iteration(std::false_type{}, std::false_type{});
#pragma unroll
      for (int t = 0; t < MT; ++t) multiply(3, t);
    } else {
      static_assert(S == 2 || (S == 4 && FM == 2 && FN == 2), "rings");
      Frag<LKM, FM> a[2][4];                                            // of two slabs: one multiplied, one read
      Frag<RKM, FN> b[2][4];
      constexpr int NR = 4 * READS, NM = 4 * MT;
      auto read = [&](int stage, auto set, auto n) {
        constexpr int SET = decltype(set)::value, KK = decltype(n)::value / READS, N = decltype(n)::value % READS;
        if constexpr (N < L::READS) l.template fetch<KK, N>(a[SET][KK], stage * kStage);
        else r.template fetch<KK, N - L::READS>(b[SET][KK], stage * kStage);
      };
      // BEHIND: slabs after the next one that are on their way; < 0: there is no next one
      int cur = 0;
      auto slab = [&](auto set_tag, auto refill_tag, auto behind_tag) {
        constexpr int SET = decltype(set_tag)::value, BEHIND = decltype(behind_tag)::value;
        constexpr bool REFILL = decltype(refill_tag)::value, MORE = BEHIND >= 0;
        wait_lds<0>();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          a[SET][kk].tie();
          b[SET][kk].tie();
        }
        __builtin_amdgcn_sched_barrier(0);
        const int next = (cur + 1) & 3;
        if constexpr (MORE) {
          wait_loads<BEHIND * LOADS>();                                 // my loads of the next slab have landed
          __builtin_amdgcn_s_barrier();                                 // everybody's; and everybody has read this one
        }
          static_for<0, NM>([&](auto t_tag) {
          constexpr int t = decltype(t_tag)::value, kk = t / MT, i = t % MT / FN, j = t % FN;
          if constexpr (MORE && t < NM / 2)
            static_for<t * NR / (NM / 2), (t + 1) * NR / (NM / 2)>([&](auto n) { read(next, integral_constant<int, SET ^ 1>{}, n); });
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[SET][kk].at(i), b[SET][kk].at(j), acc[i][j], 0, 0, 0);
          if constexpr (REFILL && t == 0) take_next();
          if constexpr (REFILL) {
#pragma unroll
            for (int n = t * LOADS / NM; n < (t + 1) * LOADS / NM; ++n) load_one(cur, n);
          }
          __builtin_amdgcn_sched_barrier(0);
        });
        cur = next;
      };
      using I0 = integral_constant<int, 0>;
      using I1 = integral_constant<int, 1>;
      using I2 = integral_constant<int, 2>;
      int left = count;                                                 // the slab that is next to be multiplied sits in set (left - 1) % 2
      if (left > 4 || (left & 1)) {
        if (left & 1) {
          static_for<0, NR>([&](auto n) { read(0, I0{}, n); });
        } else {
          static_for<0, NR>([&](auto n) { read(0, I1{}, n); });
          slab(I1{}, std::true_type{}, I2{});
          --left;
        }
        while (left > 5) {
          slab(I0{}, std::true_type{}, I2{});
          slab(I1{}, std::true_type{}, I2{});
          left -= 2;
        }
        if (left == 5) {
          slab(I0{}, std::true_type{}, I2{});
          --left;
        }
      } else {
        static_for<0, NR>([&](auto n) { read(0, I1{}, n); });
      }
      if (left >= 4) slab(I1{}, std::false_type{}, I2{});
      if (left >= 3) slab(I0{}, std::false_type{}, I1{});
      if (left >= 2) slab(I1{}, std::false_type{}, I0{});
      slab(I0{}, std::false_type{}, integral_constant<int, -1>{});
    }
    __syncthreads();                                                  // LDS is the epilogue's
  }

  // The tile as 16-bit values leaves through an image in LDS, [BN columns][BM], 16-byte chunks of column c at position chunk ^ c % 32 (or
  // % 16): each lane puts its 8 bytes of rows 8 q + 4 h .. + 3 of MFMA tile (i, j) there, and whole rows of the image go out.
  static constexpr int CHUNKS = BM / 8, KEY = (CHUNKS < 32 ? CHUNKS : 32) - 1;
  __device__ __forceinline__ void put(unsigned char* smem, int i, int j, int q, u32x2 v) const {
    const int c = wn * WN + 32 * j + (lane & 31), chunk = (wm * WM + 32 * i) / 8 + q;
    *reinterpret_cast<u32x2*>(smem + c * (BM * 2) + ((chunk ^ (c & KEY)) * 16) + (lane >> 5) * 8) = v;
  }
  // f(column, first row, 8 values)
  template <typename F>
  __device__ __forceinline__ void image_out(const unsigned char* smem, F&& f) const {
    constexpr int ROWS = 64 / CHUNKS, STEPS = BN / ROWS / 4, BATCH = STEPS < 8 ? STEPS : 8;
    for (int s0 = 0; s0 < STEPS; s0 += BATCH) {
      u32x4 v[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) v[u] = *reinterpret_cast<const u32x4*>(smem + ((s0 + u) * 4 + wave) * 1024 + lane * 16);
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int c = ((s0 + u) * 4 + wave) * ROWS + lane / CHUNKS;
        f(c, ((lane % CHUNKS) ^ (c & KEY)) * 8, v[u]);
      }
    }
  }
};

}  // namespace head
}  // namespace muon
