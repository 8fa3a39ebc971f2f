// Walks plans of the head's losses (paper_2502_16982_amd/csrc/head_plan.cpp) and checks what the launches rely on.  With arguments
// "tokens vocab width f32" prints the forms of that call's launches instead.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "head_plan.h"

using namespace muon;

static int failures = 0;
#define CHECK(c, ...)                                   \
  do {                                                  \
    if (!(c)) {                                         \
      ++failures;                                       \
      std::printf("line %d: %s: ", __LINE__, #c);       \
      std::printf(__VA_ARGS__);                         \
      std::printf("\n");                                \
    }                                                   \
  } while (0)

static HeadShape shape(int64_t t, int64_t v, int64_t d, bool f32, int top = 1, bool dh = true, bool dw = true) {
  return {t, v, d, d, d, f32, true, true, top, dh, dw};
}

static void check_product(const HeadProduct& p, int pairs) {
  CHECK(p.tile == 128 || p.tile == 256, "%d", p.tile);
  CHECK(!p.alone || p.tile == 128, "alone %d", p.tile);
  CHECK((int64_t)p.tiles_m * p.tile >= p.m && (int64_t)(p.tiles_m - 1) * p.tile < (p.m > 0 ? p.m : 1), "m");
  CHECK((int64_t)p.tiles_n * p.tile >= p.n, "n");
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n, slabs = (p.k + kHeadSlab - 1) / kHeadSlab * pairs;
  CHECK(p.whole <= tiles && (p.whole == tiles || (p.tile == 256 && p.splits == 1)), "whole %d of %lld", p.whole, (long long)tiles);
  CHECK(p.splits >= 1 && p.slabs_per_split >= 1, "splits");
  // every split has a slab of its own, and together they have all
  CHECK((int64_t)(p.splits - 1) * p.slabs_per_split < (slabs > 0 ? slabs : 1) && (int64_t)p.splits * p.slabs_per_split >= slabs, "runs");
  CHECK(p.blocks() < (1ll << 31), "grid");
}

static void check_plan(const HeadShape& s, const HeadPlan& p) {
  CHECK(p.piece >= 1 && p.pieces >= 1, "pieces");
  CHECK(s.tokens == 0 || (p.piece * p.pieces >= s.tokens && p.piece * (p.pieces - 1) < s.tokens), "pieces cover");
  CHECK(p.vocab_pitch % 256 == 0 && p.vocab_pitch >= s.vocab && p.width_k % 8 == 0 && p.width_k >= s.width, "pitches");
  CHECK(p.blocks * kHeadGrain >= s.vocab, "blocks");
  CHECK(p.piece * 256 < (1ll << 32) && p.piece * (p.vocab_pitch / 4096 + 1) * 256 < (1ll << 32) + (1ll << 28), "threads");
  const int64_t last = s.tokens - (p.pieces - 1) * p.piece, row = (int64_t)p.planes * p.width_k * 2;
  for (int i = 0; i < 2; ++i) {
    check_product(p.logits[i], p.pairs);
    check_product(p.hidden[i], p.pairs);
    check_product(p.weight[i], p.pairs);
    CHECK(p.logits[i].splits == 1, "logits are not split");
    const int64_t n = i ? last : p.piece;
    const bool grad = s.d_hidden || s.d_weight;
    // sections in order, each as large as what is put there, 256-byte aligned
    struct Section { size_t at; int64_t bytes; bool there; };
    const int64_t split_h = s.d_hidden && p.hidden[i].splits > 1 ? p.hidden[i].splits * n * s.width * 4 : 0;
    const int64_t split_w = s.d_weight && p.weight[i].splits > 1 ? p.weight[i].splits * s.vocab * s.width * 4 : 0;
    std::vector<Section> all = {
        {p.packed_weight, s.vocab * row, p.pack_weight},
        {p.sum, s.vocab * s.width * 4, s.d_weight && p.pieces > 1},
        {p.packed_hidden, p.piece * row, p.pack_hidden},
        {p.masked_hidden, p.piece * row, s.d_weight},
        {p.stats, p.blocks * p.piece * 8, true},
        {p.entry, p.piece * s.top * 4, true},
        {p.value, p.piece * s.top * 4, grad},
        {p.scale, p.piece * 4, true},
        {p.lse, p.piece * 8, true},
        {p.peak, 4, grad},
        {p.prob, p.piece * p.vocab_pitch * (s.f32 ? 4 : 2), grad},
        {p.grad, s.f32 ? 3 * p.piece * p.vocab_pitch * 2 : 0, grad && s.f32},
        {p.partial, split_h > split_w ? split_h : split_w, split_h + split_w > 0},
    };
    size_t end = 0;
    for (size_t k = 0; k < all.size(); ++k) {
      if (!all[k].there) continue;
      CHECK(all[k].at >= end && all[k].at % 256 == 0, "section %zu at %zu, the one before ends at %zu", k, all[k].at, end);
      end = all[k].at + (size_t)all[k].bytes;
    }
    CHECK(end <= p.total, "%zu of %zu", end, p.total);
  }
  if (!s.f32) CHECK(p.grad == p.prob, "in place");
  // offsets inside a tile: 256 rows, or 64 rows of K, of the widest pitch
  CHECK(256 * p.vocab_pitch * 2 <= (1ll << 30) && 256 * p.width_k * 2 <= (1ll << 30), "32-bit offsets");
  CHECK(p.pack_hidden || s.hidden_stride <= kHeadMaxPitch, "pitch of H");
}

static void print(const char* name, const HeadProduct& p) {
  std::printf("%s tile=%d alone=%d splits=%d quarters=%lld\n", name, p.tile, (int)p.alone, p.splits,
              (long long)(4 * ((int64_t)p.tiles_m * p.tiles_n - p.whole)));
}

int main(int argc, char** argv) {
  HeadPlan p;
  if (argc == 5) {
    head_plan(shape(std::atoll(argv[1]), std::atoll(argv[2]), std::atoll(argv[3]), std::atoi(argv[4]) != 0), 0, &p);
    print("logits", p.logits[0]);
    print("hidden", p.hidden[0]);
    print("weight", p.weight[0]);
    return 0;
  }
  const int64_t tokens[] = {0, 1, 2, 17, 255, 256, 257, 1000, 4096, 8192, 8193, 20000, 100000, kHeadMaxTokens};
  const int64_t vocab[] = {1, 2, 127, 128, 129, 1000, 5003, 32768, 65537, 131072, 256000, kHeadMaxVocab};
  const int64_t width[] = {1, 7, 8, 64, 65, 1024, 4096, 16384, kHeadMaxWidth};
  long plans = 0;
  for (int64_t t : tokens)
    for (int64_t v : vocab)
      for (int64_t d : width)
        for (int f32 = 0; f32 < 2; ++f32)
          for (int which = 0; which < 4; ++which) {
            HeadShape s = shape(t, v, d, f32 != 0, which == 3 ? 64 : 1, which & 1, which & 2);
            if (which == 2) s.hidden_aligned = false, s.hidden_stride = d + 3;
            CHECK(head_plan(s, 0, &p), "no limit");
            check_plan(s, p);
            CHECK(p.piece <= kHeadPieceTokens || t <= kHeadPieceTokens, "default pieces");
            const size_t whole = p.total;
            // a call finds a plan for what a query answered, also for a limit, and none below the smallest
            HeadPlan q;
            CHECK(head_plan(s, whole, &q) && q.total <= whole, "as much as the query said");
            check_plan(s, q);
            CHECK(head_plan(s, ~(size_t)0, &q), "all the memory there is");
            check_plan(s, q);
            if (t < 1000000) {
              HeadPlan least;
              const bool fits = head_plan(s, 1, &least);
              CHECK(!fits && least.piece <= 256, "the smallest pieces");
              check_plan(s, least);
              CHECK(head_plan(s, least.total, &q) && q.total <= least.total, "the smallest workspace");
              const size_t middle = (least.total + whole) / 2;
              if (middle >= least.total) {
                CHECK(head_plan(s, middle, &q) && q.total <= middle, "in between");
                check_plan(s, q);
                HeadPlan again;
                CHECK(head_plan(s, q.total, &again) && again.total <= q.total, "and again");
              }
            }
            ++plans;
          }
  std::printf("%ld plans, %d failures\n", plans, failures);
  return failures != 0;
}
