#include "head_plan.h"

#include <algorithm>

namespace muon {
namespace {

constexpr int64_t up(int64_t v, int64_t grain) { return (v + grain - 1) / grain * grain; }

void plan_piece(const HeadShape& s, int64_t piece, HeadPlan* p) {
  p->piece = piece;
  p->pieces = std::max<int64_t>(1, (s.tokens + piece - 1) / piece);
  const bool gradients = s.d_hidden || s.d_weight;
  const int64_t sizes[2] = {piece, s.tokens - (p->pieces - 1) * piece};
  int64_t partial = 0;
  for (int i = 0; i < 2; ++i) {
    p->logits[i] = head_product(s.vocab, sizes[i], p->width_k, p->pairs, false);
    p->hidden[i] = head_product(s.width, sizes[i], s.vocab, p->pairs, true);
    p->weight[i] = head_product(s.width, s.vocab, sizes[i], p->pairs, true);
    if (s.d_hidden && p->hidden[i].splits > 1) partial = std::max(partial, p->hidden[i].splits * sizes[i] * s.width * 4);
    if (s.d_weight && p->weight[i].splits > 1) partial = std::max(partial, p->weight[i].splits * s.vocab * s.width * 4);
  }
  size_t at = 0;
  auto take = [&](bool wanted, int64_t bytes) {
    const size_t here = at;
    if (wanted) at += (size_t)up(bytes, 256);
    return here;
  };
  const int64_t row = p->planes * p->width_k * 2;
  p->packed_weight = take(p->pack_weight, s.vocab * row);
  p->sum = take(s.d_weight && p->pieces > 1, s.vocab * s.width * 4);
  p->packed_hidden = take(p->pack_hidden, piece * row);
  p->masked_hidden = take(s.d_weight, piece * row);
  p->stats = take(true, p->blocks * piece * 8);
  p->entry = take(true, piece * s.top * 4);
  p->value = take(gradients, piece * s.top * 4);
  p->scale = take(true, piece * 4);
  p->lse = take(true, piece * 8);
  p->peak = take(gradients, 4);
  p->prob = take(gradients, piece * p->vocab_pitch * (s.f32 ? 4 : 2));
  p->grad = s.f32 ? take(gradients, 3 * piece * p->vocab_pitch * 2) : p->prob;      // bf16: in place of the probabilities
  p->partial = take(partial > 0, partial);
  p->total = std::max<size_t>(at, 256);
}

}  // namespace

namespace {

constexpr int64_t kUnits = 256;                  // compute units
// What a launch takes, in us, from the time of a slab of 64 of K: a 256-wide tile per compute unit 1.75; two 128-wide ones 1.17; one
// alone, on the longer ring, 0.58; and 10, 4 or 6 to start and to store.  Both sides of the choices that are near: gradient of H at 2048 x 32768 x 1024
// bf16, 256-wide in 8 runs of K 123 us + 14 to join, 128-wide alone in 2 runs 145 + 7; at 1000 x 20011 x 777 fp32 226 + 10 against 293 + 6;
// 4096 x 65537 x 2048 bf16 in 2 runs 899 + 21 against tiles of 128 in whole 1197; its gradient of W, 257 x 8 tiles, with the last round in
// quarters 991 against 1032.
double time_wide(int64_t blocks, double slabs) { return (double)((blocks + kUnits - 1) / kUnits) * (1.75 * slabs + 10); }
double time_narrow(int64_t blocks, double slabs) { return (double)((blocks + 2 * kUnits - 1) / (2 * kUnits)) * (1.17 * slabs + 4); }
double time_alone(int64_t blocks, double slabs) { return (double)((blocks + kUnits - 1) / kUnits) * (0.58 * slabs + 6); }

}  // namespace

// The fastest by the times above of: tiles of 256, with what the last round holds in tiles of 128 where that is quicker; tiles of 128;
// either with K in up to 64 runs of at least eight slabs, whose fp32 results are written and read once more (at 5 bytes per ps, and a launch).
HeadProduct head_product(int64_t m, int64_t n, int64_t k, int pairs, bool may_split) {
  HeadProduct p{};
  p.m = m;
  p.n = n;
  p.k = k;
  auto tiles = [&](int64_t tile) { return ((m + tile - 1) / tile) * ((n + tile - 1) / tile); };
  const int64_t wide = tiles(256), narrow = tiles(128), slabs = std::max<int64_t>(1, (k + kHeadSlab - 1) / kHeadSlab * pairs);
  double best = 0;
  int64_t splits = 1;
  auto offer = [&](double us, int tile, bool alone, int64_t whole, int64_t s) {
    if (p.tile && us >= best) return;
    best = us;
    p.tile = tile;
    p.alone = alone;
    p.whole = (int)whole;
    splits = s;
  };
  if (narrow <= kUnits) offer(time_alone(narrow, (double)slabs), 128, true, narrow, 1);
  offer(time_narrow(narrow, (double)slabs), 128, false, narrow, 1);
  offer(time_wide(wide, (double)slabs), 256, false, wide, 1);
  const int64_t rest = wide % kUnits;
  if (wide > kUnits && rest) offer(time_wide(wide - rest, (double)slabs) + time_alone(4 * rest, (double)slabs), 256, false, wide - rest, 1);
  if (may_split) {
    for (int64_t s = 2; s <= 64 && slabs / s >= 8; ++s) {
      const double each = (double)((slabs + s - 1) / s), join = 4 + (double)(s * m * n) * 8e-6 / 5;
      if (narrow * s <= kUnits) offer(time_alone(narrow * s, each) + join, 128, true, narrow, s);
      if (narrow * s <= 2 * kUnits) offer(time_narrow(narrow * s, each) + join, 128, false, narrow, s);
      if (wide * s <= 2 * kUnits) offer(time_wide(wide * s, each) + join, 256, false, wide, s);
    }
  }
  p.tiles_m = (int)((m + p.tile - 1) / p.tile);
  p.tiles_n = (int)((n + p.tile - 1) / p.tile);
  p.slabs_per_split = (int)((slabs + splits - 1) / splits);
  p.splits = (int)((slabs + p.slabs_per_split - 1) / p.slabs_per_split);
  return p;
}

bool head_plan(const HeadShape& s, size_t max_bytes, HeadPlan* p) {
  *p = HeadPlan{};
  p->planes = s.f32 ? 3 : 1;
  p->pairs = s.f32 ? 6 : 1;
  p->width_k = up(s.width, 8);
  p->vocab_pitch = up(s.vocab, 256);
  p->blocks = up(s.vocab, kHeadGrain) / kHeadGrain;
  // fp32 operands are split into planes; bf16 rows that do not come in whole aligned chunks of 16 bytes are copied
  const bool ragged = s.f32 || s.width % 8 != 0;
  p->pack_hidden = ragged || s.hidden_stride % 8 != 0 || s.hidden_stride > kHeadMaxPitch || !s.hidden_aligned;
  p->pack_weight = ragged || s.weight_stride % 8 != 0 || s.weight_stride > kHeadMaxPitch || !s.weight_aligned;
  // Equal pieces of whole tiles, ever more of them until the workspace fits: what a query answers is one of these, so that a call
  // that is given as many bytes finds it (or an earlier one).
  const int64_t all = std::max<int64_t>(1, s.tokens);
  const int64_t most = max_bytes == 0 ? kHeadPieceTokens : std::min(kHeadMaxPiece, kHeadMaxProbs / p->vocab_pitch / 256 * 256);
  for (int64_t pieces = (all + most - 1) / most;;) {
    const int64_t piece = std::min(all, up((all + pieces - 1) / pieces, 256));
    plan_piece(s, piece, p);
    if (max_bytes == 0 || p->total <= max_bytes) return true;
    const int64_t smaller = (piece - 1) / 256 * 256;
    if (smaller == 0) return false;
    pieces = (all + smaller - 1) / smaller;
  }
}

}  // namespace muon
