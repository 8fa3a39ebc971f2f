// Walks the plans of calls for log probabilities over their range of sizes and limits.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "score_plan.h"

using namespace muon;

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      std::printf("line %d: %s\n", __LINE__, #x);             \
      std::exit(1);                                           \
    }                                                         \
  } while (0)

static void walk(const HeadShape& s, bool best, size_t limit) {
  const size_t need = score_workspace(s, best, limit);
  CHECK(need % 256 == 0 && need > 0);
  ScorePlan p;
  const bool keep = !best && s.width % 2;
  CHECK(score_plan(s, best, keep, need, &p));
  CHECK(p.few == (!keep && p.shape.pack_weight && s.tokens <= (s.f32 ? 64 : 16)) && (!p.few || p.pieces == 1));
  CHECK(p.total <= need && p.piece >= 1 && p.piece <= kHeadPieceTokens);
  CHECK(p.pieces == (s.tokens ? (s.tokens + p.piece - 1) / p.piece : 1));
  CHECK(p.pieces == 1 || p.piece % 256 == 0);
  const int64_t row = p.shape.planes * p.shape.width_k * 2;
  size_t end = 0;
  auto section = [&](bool there, size_t at, int64_t bytes) {
    if (!there) return;
    CHECK(at % 256 == 0 && at >= end);
    end = at + (size_t)bytes;
  };
  section(p.shape.pack_weight, p.packed_weight, s.vocab * row);
  section(p.shape.pack_hidden, p.packed_hidden, p.piece * row);
  section(true, p.stats, p.shape.blocks * p.piece * 16);
  section(best, p.best, p.groups * p.piece * 8);
  CHECK(end <= p.total);
  CHECK(p.groups * kScoreGroup >= s.vocab && p.groups % 4 == 0);
  for (int i = 0; i < 2; ++i) {
    CHECK(p.logits[i].splits == 1 && p.logits[i].m == s.vocab && p.logits[i].k == p.shape.width_k);
    CHECK((int64_t)p.logits[i].tiles_n * p.logits[i].tile >= (i ? s.tokens - (p.pieces - 1) * p.piece : std::min(p.piece, s.tokens)));
    CHECK(p.logits[i].blocks() < (int64_t{1} << 24));
  }
  ScorePlan none;
  CHECK(!score_plan(s, best, false, 0, &none));
  if (limit) {
    CHECK(score_workspace(s, best, limit) <= std::max(limit, score_workspace(s, best, 1)));
    CHECK(score_workspace(s, best, limit) <= score_workspace(s, best, 0));
  }
}

int main() {
  std::mt19937_64 rng(1);
  auto between = [&](double low, double high) { return (int64_t)std::llround(std::exp(std::uniform_real_distribution<>(std::log(low), std::log(high))(rng))); };
  for (int i = 0; i < 30000; ++i) {
    const int64_t width = between(1, 8192), tokens = i % 17 == 0 ? (int64_t)(rng() % 4) : between(1, 200000);
    const HeadShape s{tokens, between(1, 1 << 21), width, width + (int64_t)(rng() % 3) * 4, width, rng() % 3 == 0, rng() % 2 == 0, rng() % 2 == 0, 1, false, false};
    walk(s, rng() % 2, rng() % 2 ? 0 : (size_t)between(1, 1e11));
    // a workspace for more tokens serves fewer
    HeadShape more = s;
    more.tokens += (int64_t)(rng() % 5000);
    CHECK(score_workspace(more, true, 0) >= score_workspace(s, true, 0));
  }
  std::printf("ok\n");
}
