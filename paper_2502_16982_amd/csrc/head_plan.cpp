#include "head_plan.h"

#include <algorithm>

namespace muon {
namespace {

constexpr int64_t up(int64_t v, int64_t grain) { return (v + grain - 1) / grain * grain; }

constexpr int64_t kUnits = 256;                  // compute units
// What a launch takes, in us, from the time of a slab of 64 of K: a 256-wide tile per compute unit 1.75; two 128-wide ones 1.17; one
// alone, on the longer ring, 0.58; and 10, 4 or 6 to start and to store.  Both sides of the choices that are near: gradient of H at 2048 x 32768 x 1024
// bf16, 256-wide in 8 runs of K 123 us + 14 to join, 128-wide alone in 2 runs 145 + 7; at 1000 x 20011 x 777 fp32 226 + 10 against 293 + 6;
// 4096 x 65537 x 2048 bf16 in 2 runs 899 + 21 against tiles of 128 in whole 1197; its gradient of W, 257 x 8 tiles, with the last round in
// quarters 991 against 1032.  Held against the other forms (K in 1 to 64 runs) for each product of 15 calls that these times were not taken from (96 to
// 8192 tokens, vocabularies of 8000 to 100277, widths of 512 to 4096, three of them fp32), the choice is the fastest or within 2.5 % of the
// whole call in 41 of 45; the others: gradient of W at 200 x 32000 x 2048 in tiles of 256 (call 157 us) instead of 128 (144), of H at 2500 x 8192 x 4096 in 3
// runs (526) instead of one (488), at 6000 x 24000 x 640 128 alone (777) instead of 128 in 2 runs (748), at 700 x 12000 x 768 fp32 256 in 28
// runs (342) instead of 128 alone in 6 (316).
double time_wide(int64_t blocks, double slabs) { return (double)((blocks + kUnits - 1) / kUnits) * (1.75 * slabs + 10); }
double time_narrow(int64_t blocks, double slabs) { return (double)((blocks + 2 * kUnits - 1) / (2 * kUnits)) * (1.17 * slabs + 4); }
double time_alone(int64_t blocks, double slabs) { return (double)((blocks + kUnits - 1) / kUnits) * (0.58 * slabs + 6); }
// Runs of K, and slabs that a run has at least.
constexpr int64_t kMaxSplits = 64, kMinRun = 8;

}  // namespace

// The fastest by the times above of: tiles of 256, with what the last round holds in tiles of 128 where that is quicker; tiles of 128;
// either with K in up to 64 runs of at least eight slabs, whose fp32 results are written and read once more (at 5 bytes per ps, and a launch),
// where these take no more than partial_bytes.
HeadProduct head_product(int64_t m, int64_t n, int64_t k, int pairs, int64_t partial_bytes) {
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
  for (int64_t s = 2; s <= kMaxSplits && slabs / s >= kMinRun && s * m * n * 4 <= partial_bytes; ++s) {
    const double each = (double)((slabs + s - 1) / s), join = 4 + (double)(s * m * n) * 8e-6 / 5;
    if (narrow * s <= kUnits) offer(time_alone(narrow * s, each) + join, 128, true, narrow, s);
    if (narrow * s <= 2 * kUnits) offer(time_narrow(narrow * s, each) + join, 128, false, narrow, s);
    if (wide * s <= 2 * kUnits) offer(time_wide(wide * s, each) + join, 256, false, wide, s);
  }
  p.tiles_m = (int)((m + p.tile - 1) / p.tile);
  p.tiles_n = (int)((n + p.tile - 1) / p.tile);
  p.slabs_per_split = (int)((slabs + splits - 1) / splits);
  p.splits = (int)((slabs + p.slabs_per_split - 1) / p.slabs_per_split);
  return p;
}

namespace {

// What of a plan goes by the shape alone.
HeadPlan plan_shape(const HeadShape& s) {
  HeadPlan p{};
  p.planes = s.f32 ? 3 : 1;
  p.pairs = s.f32 ? 6 : 1;
  p.width_k = up(s.width, 8);
  p.vocab_pitch = up(s.vocab, 256);
  p.blocks = up(s.vocab, kHeadGrain) / kHeadGrain;
  // fp32 operands are split into planes; bf16 rows that do not come in whole aligned chunks of 16 bytes are copied
  const bool ragged = s.f32 || s.width % 8 != 0;
  p.pack_hidden = ragged || s.hidden_stride % 8 != 0 || s.hidden_stride > kHeadMaxPitch || !s.hidden_aligned;
  p.pack_weight = ragged || s.weight_stride % 8 != 0 || s.weight_stride > kHeadMaxPitch || !s.weight_aligned;
  return p;
}

// Lays out the sections for pieces of so many tokens; the splits' sums come last.
void lay_out(const HeadShape& s, int64_t piece, int64_t partial, HeadPlan* p) {
  p->piece = piece;
  p->pieces = std::max<int64_t>(1, (s.tokens + piece - 1) / piece);
  const bool gradients = s.d_hidden || s.d_weight;
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
  p->kept = take(gradients, piece * 4);
  p->prob = take(gradients, piece * p->vocab_pitch * (s.f32 ? 4 : 2));
  p->grad = s.f32 ? take(gradients, 3 * piece * p->vocab_pitch * 2) : p->prob;      // bf16: in place of the probabilities
  p->partial = take(partial > 0, partial);
  p->total = std::max<size_t>(at, 256);
}

// Bytes for pieces of so many tokens without any splits.  More tokens in a piece take more, but for the sum of d_weight, which one piece
// does without.
size_t bytes_unsplit(const HeadShape& s, int64_t piece) {
  HeadPlan p = plan_shape(s);
  lay_out(s, piece, 0, &p);
  return p.total;
}

// Bytes that the sums of splits may take: what no choice of head_product goes beyond, so that it is never held back.  Unlike the choice
// itself this grows with every size, which makes a workspace for more tokens one for fewer.
int64_t bytes_split(const HeadShape& s, int64_t piece) {
  auto product = [&](int64_t n, int64_t k) -> int64_t {
    const int64_t splits = std::min(kMaxSplits, (k + kHeadSlab - 1) / kHeadSlab * (s.f32 ? 6 : 1) / kMinRun);
    return splits < 2 ? 0 : std::min(2 * kUnits * 256 * 256 * 4, splits * s.width * n * 4);
  };
  return up(std::max(s.d_hidden ? product(piece, s.vocab) : 0, s.d_weight ? product(s.vocab, piece) : 0), 256);
}

// The most tokens of a piece that a launch takes.
int64_t most_tokens(const HeadShape& s) { return std::min(kHeadMaxPiece, kHeadMaxProbs / up(s.vocab, 256) / 256 * 256); }

}  // namespace

size_t head_workspace(const HeadShape& s, size_t max_bytes) {
  const int64_t all = std::max<int64_t>(1, s.tokens);
  size_t want = ~(size_t)0, least = ~(size_t)0;
  if (all <= most_tokens(s)) {                     // one piece
    least = bytes_unsplit(s, all);
    want = least + bytes_split(s, all);
  }
  if (max_bytes == 0) return all <= kHeadPieceTokens ? want : std::min(want, bytes_unsplit(s, kHeadPieceTokens) + bytes_split(s, kHeadPieceTokens));
  if (want <= max_bytes) return want;
  if (all > 256) least = std::min(least, bytes_unsplit(s, 256));
  return std::max(least, max_bytes / 256 * 256);
}

bool head_plan(const HeadShape& s, size_t max_bytes, HeadPlan* p) {
  *p = plan_shape(s);
  const int64_t all = std::max<int64_t>(1, s.tokens), most = max_bytes == 0 ? kHeadPieceTokens : most_tokens(s);
  const size_t limit = max_bytes == 0 ? (size_t)1 << 62 : std::min(max_bytes, (size_t)1 << 62);
  // The products for pieces of so many tokens with so many bytes for the splits' sums, of which it answers what they take.
  auto products = [&](int64_t piece, int64_t room) {
    const int64_t before_last = (std::max<int64_t>(1, (s.tokens + piece - 1) / piece) - 1) * piece, sizes[2] = {piece, s.tokens - before_last};
    int64_t partial = 0;
    for (int i = 0; i < 2; ++i) {
      p->logits[i] = head_product(s.vocab, sizes[i], p->width_k, p->pairs, 0);
      p->hidden[i] = head_product(s.width, sizes[i], s.vocab, p->pairs, room);
      p->weight[i] = head_product(s.width, s.vocab, sizes[i], p->pairs, room);
      if (s.d_hidden && p->hidden[i].splits > 1) partial = std::max(partial, p->hidden[i].splits * sizes[i] * s.width * 4);
      if (s.d_weight && p->weight[i].splits > 1) partial = std::max(partial, p->weight[i].splits * s.vocab * s.width * 4);
    }
    return up(partial, 256);
  };
  // All tokens in one piece, or equal pieces of as many whole tiles of them as fit.
  auto equal = [&](int64_t most_each) {
    const int64_t n = (all + most_each - 1) / most_each;
    return up((all + n - 1) / n, 256);
  };
  int64_t piece = all;
  bool fits = all <= most && bytes_unsplit(s, all) <= limit;
  if (!fits) {
    int64_t low = 0, high = std::min(most, (all - 1) / 256 * 256) / 256;
    while (low < high) {
      const int64_t middle = (low + high + 1) / 2;
      if (bytes_unsplit(s, middle * 256) <= limit) low = middle;
      else high = middle - 1;
    }
    fits = low > 0;
    piece = fits ? equal(low * 256) : std::min<int64_t>(all, 256);
    // smaller ones where these leave no room for the splits, but not by half: a piece more reads the weight three times and the sum twice
    for (int64_t less = piece; fits && 2 * less > low * 256; less = equal(less - 256)) {
      if (bytes_unsplit(s, less) + (size_t)products(less, bytes_split(s, less)) <= limit) {
        piece = less;
        break;
      }
      if (less <= 256) break;
    }
  }
  const int64_t partial = products(piece, fits ? (int64_t)((limit - bytes_unsplit(s, piece)) / 256 * 256) : 0);
  lay_out(s, piece, partial, p);
  return fits;
}

}  // namespace muon
