// Walks the plans of a mixture's layer for few tokens over its range of sizes.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../paper_2502_16982_amd/csrc/layer_plan.h"

using namespace muon;

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      std::printf("line %d: %s\n", __LINE__, #x);             \
      std::exit(1);                                           \
    }                                                         \
  } while (0)

static void product(const LayerProduct& g, int64_t k, int64_t n, bool f32, int slots) {
  CHECK(g.k == k && g.n == n && g.runs >= 1 && g.run % kLayerRows == 0);
  CHECK((g.runs - 1) * g.run < k && g.runs * g.run >= k);          // no run is empty
  CHECK((int64_t)g.tiles * layer_columns(f32) >= n && (int64_t)(g.tiles - 1) * layer_columns(f32) < n);
  CHECK((int64_t)slots * g.tiles * g.runs * g.mats < (int64_t{1} << 24));
  CHECK(g.mats == 1 || (g.mats == 2 && g.runs > 1));
  CHECK(g.runs == 1 || (int64_t)slots * g.tiles * g.runs * g.mats <= kLayerBlocks);
}

static void walk(const LayerShape& s) {
  const LayerPlan p = layer_plan(s);
  const int64_t pairs = s.tokens * s.top;
  CHECK(p.slots <= pairs && p.slots <= s.experts && (p.slot_is_pair ? p.slots == pairs : p.slots == s.experts));
  product(p.up, s.width, s.inner, s.f32, p.slots);
  product(p.down, s.inner, s.width, s.f32, p.slots);
  const size_t part = p.up.runs > 1 ? (size_t)p.up.runs * pairs * (s.gated ? 2 : 1) * s.inner * 4 : 0;
  CHECK(p.part == 0 && p.inner >= part && p.rows >= p.inner + (p.staged ? 0 : (size_t)pairs * s.inner * (s.f32 ? 4 : 2)));
  CHECK(!p.staged || (p.up.runs > 1 && p.down.run * 32 * (s.f32 ? 4 : 2) <= kLayerStage));
  CHECK(p.total >= p.rows + (size_t)p.down.runs * pairs * s.width * 4 && p.total < (size_t{1} << 42));
  CHECK(p.inner % 256 == 0 && p.rows % 256 == 0);
  for (const int64_t n : {s.inner, s.width}) CHECK((n + 255) / 256 * pairs < (int64_t{1} << 24));
}

int main() {
  std::mt19937_64 rng(1);
  auto between = [&](double low, double high) { return (int64_t)std::llround(std::exp(std::uniform_real_distribution<>(std::log(low), std::log(high))(rng))); };
  for (int64_t tokens : {0, 1, 2, 5, 64})
    for (int64_t width : {1, 3, 31, 32, 33, 127, 128, 129, 2048, 131072})
      for (int64_t inner : {1, 7, 8, 9, 333, 1408, 131072})
        for (int top : {1, 6, 64})
          for (int n : {1, 64, 4096}) walk({tokens, width, inner, top, n, (width & 1) != 0, (inner & 1) != 0});
  for (int i = 0; i < 100000; ++i) {
    const int top = (int)between(1, 64);
    walk({between(1, (double)(kLayerMaxPairs / top)), between(1, (double)kLayerMaxWidth), between(1, (double)kLayerMaxWidth), top, (int)between(1, kLayerMaxExperts),
          rng() % 2 == 0, rng() % 2 == 0});
  }
  std::printf("ok\n");
}
