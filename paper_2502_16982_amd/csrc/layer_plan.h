// How a mixture's layer for few tokens is cut up: runs of the summed axis, the workspace's sections (plain C++, no HIP include).
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace muon {

constexpr int64_t kLayerMaxPairs = 1 << 14, kLayerMaxWidth = 1 << 17;
// Rows further apart than this would leave the 32 bits of a lane's offset.
constexpr int64_t kLayerMaxStride = 1 << 24;
constexpr int kLayerMaxTop = 64, kLayerMaxExperts = 4096;
constexpr int kLayerRows = 32;                   // rows of the summed axis that a wave takes at a time
constexpr int kLayerWaves = 4;                   // of a block, which share its run of the summed axis
constexpr int kLayerStage = 32768;               // bytes of LDS for the second product's operand, where it is made from sums of runs

struct LayerShape {
  int64_t tokens, width, inner;
  int top, experts;
  bool gated, f32;
};

// A product of the rows of the experts' pairs with their matrices: blocks of `columns` columns of one expert, the summed axis in `runs`.
struct LayerProduct {
  int64_t k, n;
  int tiles;                                     // of columns
  int runs;
  int64_t run;                                   // rows of the summed axis in a run, a multiple of kLayerRows
  int mats;                                      // matrices with blocks of their own: 2 where gate and up are summed in runs
};

struct LayerPlan {
  int slots;                                     // experts that may have pairs: one per pair, or all of them
  bool slot_is_pair;
  LayerProduct up, down;
  bool staged;                                   // the second product makes its operand itself
  // byte offsets of the workspace's sections: sums of the first product in runs, the inner rows, sums of the second product
  size_t part, inner, rows;
  size_t total;
};

LayerPlan layer_plan(const LayerShape& s);

inline int layer_columns(bool f32) { return f32 ? 64 : 128; }

// Blocks that the chip holds at a time.
constexpr int64_t kLayerBlocks = 512;
constexpr int64_t kLayerMostRuns = 16;

// One run where its blocks fill the chip; otherwise as many as it holds at a time, so that all of a product's loads are on their way at once, but none
// below what its waves take at once.  Experts' layers in graphs, us, aimed at 256, 512 and 1024 blocks: 1 x 6 of 64, 2048 x 1408 bf16 39.8, 30.3, 36.4;
// 1 x 2 of 16, 4096 x 1408 25.6, 24.5, 26.2; 5 x 2 of 16, 777 x 333 fp32 20.9, 19.2, 21.6; 1 x 8 of 8, 1024 x 4096 39.4, 39.8, 45.2; from 4 x 6 on alike.  Runs of at
// least 64, 128 and 256 rows: 30.2, 30.3, 30.1; 24.5, 24.5, 28.4; 18.3, 19.2, 21.7.  At most 4, 8, 16 or 32 runs: alike within 2 % at all of these; 16 bound
// what the sums take.
inline LayerProduct layer_product(int64_t k, int64_t n, int columns, int64_t slots, int mats) {
  LayerProduct p{};
  p.k = k;
  p.n = n;
  p.tiles = (int)((n + columns - 1) / columns);
  const int64_t blocks = std::max<int64_t>(1, slots * p.tiles * mats), least = kLayerRows * kLayerWaves;
  const int64_t runs = std::min<int64_t>({std::max<int64_t>(1, kLayerBlocks / blocks), std::max<int64_t>(1, k / least), kLayerMostRuns});
  p.run = ((k + runs - 1) / runs + kLayerRows - 1) / kLayerRows * kLayerRows;
  p.runs = (int)((k + p.run - 1) / p.run);
  p.mats = p.runs > 1 ? mats : 1;
  return p;
}

inline LayerPlan layer_plan(const LayerShape& s) {
  LayerPlan p{};
  const int64_t pairs = s.tokens * s.top;
  p.slot_is_pair = pairs <= s.experts;
  p.slots = (int)(p.slot_is_pair ? pairs : s.experts);
  p.up = layer_product(s.width, s.inner, layer_columns(s.f32), p.slots, s.gated ? 2 : 1);
  p.down = layer_product(s.inner, s.width, layer_columns(s.f32), p.slots, 1);
  p.staged = p.up.runs > 1 && p.down.run * 32 * (s.f32 ? 4 : 2) <= kLayerStage;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)((bytes + 255) / 256 * 256);
    return here;
  };
  p.part = take(p.up.runs > 1 ? (int64_t)p.up.runs * pairs * (s.gated ? 2 : 1) * s.inner * 4 : 0);
  p.inner = take(p.staged ? 0 : pairs * s.inner * (s.f32 ? 4 : 2));
  p.rows = take((int64_t)p.down.runs * pairs * s.width * 4);
  p.total = std::max<size_t>(at, 256);
  return p;
}

// A launch: blocks along two axes, the first one fastest, and threads per block.  An axis holds less than 2^32 threads, the second one 2^16 blocks; the largest
// calls have 2^32 in all, so that slots, tokens and pairs have an axis of their own.
struct LayerGrid {
  int64_t x, y;
  int threads;
};

constexpr int kJoinColumns = 128;                // of a block of the join

// together: gate and up by one block.
inline LayerGrid layer_product_grid(const LayerProduct& p, int slots, bool together) {
  return {(int64_t)p.tiles * p.runs * p.mats, slots, 64 * kLayerWaves * (together ? 2 : 1)};
}
inline LayerGrid layer_act_grid(int64_t n, int64_t pairs) { return {(n + 255) / 256, pairs, 256}; }
inline LayerGrid layer_join_grid(int64_t n, int64_t tokens) { return {(n + kJoinColumns - 1) / kJoinColumns, tokens, 256}; }

}  // namespace muon
