// How a mixture's layer for few tokens is cut up: runs of the summed axis, the workspace's sections (plain C++, no HIP include).
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace muon {

constexpr int64_t kLayerMaxPairs = 1 << 14, kLayerMaxWidth = 1 << 17;
constexpr int kLayerMaxTop = 64, kLayerMaxExperts = 4096;
constexpr int kLayerRows = 32;                   // rows of the summed axis that a wave takes at a time
constexpr int kLayerWaves = 4;                   // of a block, which share its run of the summed axis

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
};

struct LayerPlan {
  int slots;                                     // experts that may have pairs: one per pair, or all of them
  bool slot_is_pair;
  LayerProduct up, down;
  // byte offsets of the workspace's sections: sums of the first product in runs, the inner rows, sums of the second product
  size_t part, inner, rows;
  size_t total;
};

LayerPlan layer_plan(const LayerShape& s);

inline int layer_columns(bool f32) { return f32 ? 64 : 128; }

inline LayerProduct layer_product(int64_t k, int64_t n, int columns, int64_t slots) {
  LayerProduct p{};
  p.k = k;
  p.n = n;
  p.tiles = (int)((n + columns - 1) / columns);
  // blocks enough to fill 256 compute units twice, but no run below what its waves take at once
  const int64_t blocks = std::max<int64_t>(1, slots * p.tiles), want = std::max<int64_t>(1, (512 + blocks - 1) / blocks);
  const int64_t least = kLayerRows * kLayerWaves, most = std::max<int64_t>(1, k / least), runs = std::min<int64_t>({want, most, 16});
  p.run = ((k + runs - 1) / runs + kLayerRows - 1) / kLayerRows * kLayerRows;
  p.runs = (int)((k + p.run - 1) / p.run);
  return p;
}

inline LayerPlan layer_plan(const LayerShape& s) {
  LayerPlan p{};
  const int64_t pairs = s.tokens * s.top;
  p.slot_is_pair = pairs <= s.experts;
  p.slots = (int)(p.slot_is_pair ? pairs : s.experts);
  p.up = layer_product(s.width, s.inner, layer_columns(s.f32), p.slots);
  p.down = layer_product(s.inner, s.width, layer_columns(s.f32), p.slots);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)((bytes + 255) / 256 * 256);
    return here;
  };
  p.part = take(p.up.runs > 1 ? (int64_t)p.up.runs * pairs * (s.gated ? 2 : 1) * s.inner * 4 : 0);
  p.inner = take(pairs * s.inner * (s.f32 ? 4 : 2));
  p.rows = take((int64_t)p.down.runs * pairs * s.width * 4);
  p.total = std::max<size_t>(at, 256);
  return p;
}

}  // namespace muon
