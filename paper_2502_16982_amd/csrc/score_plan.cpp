#include "score_plan.h"

#include <algorithm>

namespace muon {
namespace {

constexpr int64_t up(int64_t v, int64_t grain) { return (v + grain - 1) / grain * grain; }

void lay_out(const HeadShape& s, bool best, int64_t piece, ScorePlan* p) {
  const HeadPlan& h = p->shape;
  p->piece = piece;
  p->pieces = std::max<int64_t>(1, (s.tokens + piece - 1) / piece);
  p->groups = h.blocks * (kHeadGrain / kScoreGroup);
  size_t at = 0;
  auto take = [&](bool wanted, int64_t bytes) {
    const size_t here = at;
    if (wanted) at += (size_t)up(bytes, 256);
    return here;
  };
  const int64_t row = h.planes * h.width_k * 2;
  p->packed_weight = take(h.pack_weight, s.vocab * row);
  p->packed_hidden = take(h.pack_hidden, piece * row);
  p->stats = take(true, h.blocks * piece * 16);
  p->best = take(best, p->groups * piece * 8);
  p->total = at;
}

size_t bytes_of(const HeadShape& s, bool best, int64_t piece) {
  ScorePlan p{};
  p.shape = head_plan_shape(s);
  lay_out(s, best, piece, &p);
  return p.total;
}

// All tokens at once, or equal pieces of whole tiles of them; 0 where not even the smallest fit.
int64_t piece_of(const HeadShape& s, bool best, size_t bytes, int64_t most) {
  const int64_t all = std::max<int64_t>(1, s.tokens);
  if (all <= most && bytes_of(s, best, all) <= bytes) return all;
  int64_t low = 0, high = std::min(most, up(all, 256)) / 256;
  while (low < high) {
    const int64_t middle = (low + high + 1) / 2;
    if (bytes_of(s, best, middle * 256) <= bytes) low = middle;
    else high = middle - 1;
  }
  if (low == 0) return 0;
  const int64_t n = (all + low * 256 - 1) / (low * 256);
  return std::min(all, up((all + n - 1) / n, 256));
}

}  // namespace

size_t score_workspace(const HeadShape& s, bool best, size_t max_bytes) {
  const int64_t all = std::max<int64_t>(1, s.tokens);
  const size_t want = bytes_of(s, best, std::min(all, kHeadPieceTokens));
  if (max_bytes == 0 || want <= max_bytes) return want;
  return std::max(bytes_of(s, best, std::min<int64_t>(all, 256)), max_bytes / 256 * 256);
}

int64_t score_kept_values(const HeadShape& s) { return up(s.tokens * head_plan_shape(s).vocab_pitch * (s.f32 ? 4 : 2), 256); }
bool score_few(const HeadShape& s) { return head_plan_shape(s).pack_weight && s.tokens <= (s.f32 ? kScoreFewF32 : kScoreFew); }

size_t score_kept_bytes(const HeadShape& s) {
  if (score_few(s)) return 0;
  return (size_t)(score_kept_values(s) + (s.f32 ? 0 : up(s.tokens * head_plan_shape(s).blocks * 4, 256)));
}

bool score_plan(const HeadShape& s, bool best, bool keep, size_t bytes, ScorePlan* p) {
  *p = ScorePlan{};
  p->shape = head_plan_shape(s);
  p->few = !keep && score_few(s);
  const int64_t piece = piece_of(s, best, bytes, kHeadPieceTokens);
  if (piece == 0) return false;
  lay_out(s, best, piece, p);
  const int64_t sizes[2] = {piece, s.tokens - (p->pieces - 1) * piece};
  // The losses' choice of tiles, from times with their shorter epilogue, holds for these.  All tiles of 128 and all of 256, us, without and with 8
  // alternatives: 2048 x 32768 x 1024 140 and 134, 177 and 170; 4096 x 32768 x 1024 273 and 261, 347 and 329; 1024 x 50257 x 768 90 and 105, 118 and 132 (128 is
  // taken: 92, 117); 4096 x 100003 x 2048 1667 and 1408, 1770 and 1511; 512 x 100003 x 2048 249 and 230, 269 and 252 (256 with quarters: 204, 223).  With powers kept 2048 x 32768 x
  // 512 would be faster in 128 (104.5 against 112); 161 and 155, 362 and 324, 110 and 123 at the first three.
  for (int i = 0; i < 2; ++i) p->logits[i] = head_product(s.vocab, std::max<int64_t>(1, sizes[i]), p->shape.width_k, p->shape.pairs, 0);
  return true;
}

}  // namespace muon
