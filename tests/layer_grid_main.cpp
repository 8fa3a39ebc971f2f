// The launches of a mixture's layer for few tokens: what the device takes along each axis, at the ends of the sizes' ranges and in between.
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

static void takes(const LayerGrid& g) {
  CHECK(g.x >= 1 && g.x < (int64_t{1} << 31) && g.x * g.threads < (int64_t{1} << 32));
  CHECK(g.y >= 1 && g.y < (int64_t{1} << 16) && g.threads <= 1024);
}

static void walk(const LayerShape& s) {
  const LayerPlan p = layer_plan(s);
  const int64_t pairs = s.tokens * s.top;
  const LayerGrid up = layer_product_grid(p.up, p.slots, s.gated && p.up.mats == 1), down = layer_product_grid(p.down, p.slots, false),
                  act = layer_act_grid(s.inner, pairs), join = layer_join_grid(s.width, s.tokens);
  for (const LayerGrid& g : {up, down, act, join}) takes(g);
  CHECK(up.y == p.slots && down.y == p.slots && up.x == (int64_t)p.up.tiles * p.up.runs * p.up.mats && down.x == (int64_t)p.down.tiles * p.down.runs);
  CHECK(act.x * act.threads >= s.inner && (act.x - 1) * act.threads < s.inner && act.y == pairs);
  CHECK(join.x * kJoinColumns >= s.width && (join.x - 1) * kJoinColumns < s.width && join.y == s.tokens);
}

int main() {
  std::mt19937_64 rng(1);
  auto between = [&](double low, double high) { return (int64_t)std::llround(std::exp(std::uniform_real_distribution<>(std::log(low), std::log(high))(rng))); };
  for (bool gated : {false, true})
    for (bool f32 : {false, true})
      for (int n : {1, 2, 255, 4095, kLayerMaxExperts})
        for (int top : {1, 6, kLayerMaxTop})
          for (int64_t tokens : {int64_t{1}, int64_t{4096} / top, kLayerMaxPairs / top})
            for (int64_t width : {int64_t{1}, kLayerMaxWidth - 129, kLayerMaxWidth - 1, kLayerMaxWidth})
              for (int64_t inner : {int64_t{1}, kLayerMaxWidth - 65, kLayerMaxWidth - 1, kLayerMaxWidth}) walk({tokens, width, inner, top, n, gated, f32});
  for (int i = 0; i < 100000; ++i) {
    const int top = (int)between(1, 64);
    walk({between(1, (double)(kLayerMaxPairs / top)), between(1, (double)kLayerMaxWidth), between(1, (double)kLayerMaxWidth), top, (int)between(1, kLayerMaxExperts),
          rng() % 2 == 0, rng() % 2 == 0});
  }
  std::printf("ok\n");
}
