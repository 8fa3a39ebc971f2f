// What the workspace of the head's losses (paper_2502_16982_amd/csrc/head_plan.cpp) promises: it serves every smaller call, a limit below what
// is answered without one never makes it larger, and no piece of tokens would do with less than the smallest.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "head_plan.h"

using namespace muon;

static int failures = 0;
static void fail(const char* what, const HeadShape& s, size_t limit, size_t got, size_t bar) {
  if (++failures <= 20)
    std::printf("%s: tokens %lld vocab %lld width %lld f32 %d top %d gradients %d%d limit %zu: %zu against %zu\n", what, (long long)s.tokens,
                (long long)s.vocab, (long long)s.width, s.f32, s.top, s.d_hidden, s.d_weight, limit, got, bar);
}

static HeadShape shape(int64_t t, int64_t v, int64_t d, bool f32 = false, int top = 1, bool dh = true, bool dw = true) {
  return {t, v, d, d, d, f32, true, true, top, dh, dw};
}

// The workspace of `large` serves `small`, which is no larger in anything.
static void serves(const HeadShape& large, const HeadShape& small, size_t limit) {
  const size_t have = head_workspace(large, limit), need = head_workspace(small, limit);
  if (need > have) fail("a smaller call needs more", small, limit, need, have);
  HeadPlan p;
  if (!head_plan(small, have, &p) || p.total > have) fail("a smaller call is refused", small, limit, p.total, have);
}

static void limited(const HeadShape& s, size_t limit) {
  const size_t whole = head_workspace(s, 0), got = head_workspace(s, limit), least = head_workspace(s, 1);
  HeadPlan p;
  if (limit <= whole && got > whole) fail("a limit makes it larger", s, limit, got, whole);
  if (got > limit && got != least) fail("beyond the limit, and not the smallest", s, limit, got, least);
  if (got < least) fail("below the smallest", s, limit, got, least);
  if (!head_plan(s, got, &p) || p.total > got) fail("the answer does not suffice", s, limit, p.total, got);
  if (least > 256 && head_plan(s, least - 256, &p)) fail("less than the smallest suffices", s, limit, p.total, least);
}

// "tokens vocab width f32 limit": how a call is cut that is given what a query with that limit answers.
static int describe(char** argv) {
  const HeadShape s = shape(std::atoll(argv[1]), std::atoll(argv[2]), std::atoll(argv[3]), std::atoi(argv[4]) != 0);
  HeadPlan p;
  head_plan(s, head_workspace(s, (size_t)std::atoll(argv[5])), &p);
  std::printf("pieces %lld of %lld\n", (long long)p.pieces, (long long)p.piece);
  for (int i = 0; i < 2; ++i)
    std::printf("weight %d splits %d quarters %lld hidden %d splits %d\n", p.weight[i].tile, p.weight[i].splits,
                (long long)(p.weight[i].tiles_m * (int64_t)p.weight[i].tiles_n - p.weight[i].whole), p.hidden[i].tile, p.hidden[i].splits);
  return 0;
}

int main(int argc, char** argv) {
  if (argc == 6) return describe(argv);
  // 1680 tokens in one run of K, 1260 in several
  serves(shape(1680, 3817, 4096), shape(1260, 3817, 4096), 0);
  serves(shape(1680, 3817, 4096), shape(1260, 3817, 4096), 27 << 20);
  // one piece is smaller than any number of pieces with the sum of d_weight
  for (const HeadShape& s : {shape(300, 131072, 4096), shape(4096, 131072, 4096), shape(512, 100003, 2048, true), shape(8193, 131072, 4096)}) {
    limited(s, head_workspace(s, 0) - 256);
    limited(s, head_workspace(s, 0) / 2);
  }
  std::mt19937_64 rng(1);
  auto between = [&](int64_t low, int64_t high) {        // even over the logarithm
    const double u = (double)(rng() >> 11) / 9007199254740992.0;
    return (int64_t)((double)low * std::exp(u * std::log((double)high / (double)low)));
  };
  for (int i = 0; i < 20000; ++i) {
    const bool f32 = rng() % 4 == 0, dh = rng() % 4 != 0, dw = rng() % 4 != 0;
    const int64_t t = between(1, 40000), v = between(1, 262144), d = between(8, 8192) / 8 * 8;
    const int top = 1 + (int)(rng() % 64);
    const HeadShape large = shape(t, v, d, f32, top, dh, dw);
    HeadShape small = shape(1 + (int64_t)(rng() % (uint64_t)t), rng() % 2 ? v : 1 + (int64_t)(rng() % (uint64_t)v), d, f32, 1 + (int)(rng() % (uint64_t)top),
                            dh && rng() % 4 != 0, dw && rng() % 4 != 0);
    const size_t whole = head_workspace(large, 0), limit = rng() % 2 ? 0 : (size_t)(rng() % (whole + whole / 4)) + 1;
    serves(large, small, limit);
    if (limit) limited(large, limit);
  }
  // without a limit the plan is the one that memory does not hold back
  for (int i = 0; i < 2000; ++i) {
    const HeadShape s = shape(between(1, 8192), between(1, 262144), between(8, 8192) / 8 * 8, rng() % 4 == 0);
    HeadPlan a, b;
    head_plan(s, head_workspace(s, 0), &a);
    head_plan(s, ~(size_t)0, &b);
    if (a.piece != b.piece || a.hidden[0].splits != b.hidden[0].splits || a.weight[0].splits != b.weight[0].splits || a.hidden[0].tile != b.hidden[0].tile)
      fail("held back", s, 0, a.total, b.total);
  }
  std::printf("%d failures\n", failures);
  return failures != 0;
}
