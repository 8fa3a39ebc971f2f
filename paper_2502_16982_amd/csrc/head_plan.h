// How a call of the head's losses is cut up: tokens in pieces, the workspace's sections, tiles and splits of the three products
// (plain C++, no HIP include).
#pragma once
#include <cstddef>
#include <cstdint>

namespace muon {

constexpr int64_t kHeadMaxTokens = 1ll << 30, kHeadMaxVocab = 1ll << 21, kHeadMaxWidth = 1ll << 20;
constexpr int kHeadMaxTop = 4096;
// Rows further apart than this are copied first: offsets in a tile of 256 rows stay below 2^30 bytes.
constexpr int64_t kHeadMaxPitch = 1ll << 21;
// Tokens of a piece where the caller sets no limit to the workspace.
constexpr int64_t kHeadPieceTokens = 8192;
// The most of a piece, and of a piece times the row pitch of its probabilities: a launch has fewer than 2^32 threads.
constexpr int64_t kHeadMaxPiece = 1ll << 18, kHeadMaxProbs = 1ll << 35;

struct HeadShape {
  int64_t tokens, vocab, width;
  int64_t hidden_stride, weight_stride;     // elements
  bool f32;
  bool hidden_aligned, weight_aligned;      // to 16 bytes
  int top;                                  // sparse entries of a token's target
  bool d_hidden, d_weight;
};

// One of the three products as it is launched: T = L R^T in tiles of tile x tile, the slabs of K in `splits` equal runs.  Of the tiles of
// 256 the first `whole` run as they are and the others, too few for the chip, as four of 128 each.
struct HeadProduct {
  int64_t m, n, k;          // rows of L, rows of R
  int tile;
  bool alone;               // tiles of 128, a compute unit each
  int tiles_m, tiles_n;
  int whole;
  int splits;
  int slabs_per_split;      // of kHeadSlab elements of K, over all pairs of planes
  int64_t blocks() const { return ((int64_t)whole + 4 * ((int64_t)tiles_m * tiles_n - whole)) * splits; }
};

constexpr int kHeadSlab = 64;

// Vocabulary entries that one pair of statistics of the logits' product stands for.
constexpr int kHeadGrain = 128;

struct HeadPlan {
  int planes;               // bf16 planes that an operand is the sum of: 1, or 3 for fp32
  int pairs;                // pairs of planes that are multiplied: 1 or 6
  int64_t width_k;          // columns of packed operands; K of the logits' product
  int64_t vocab_pitch;      // row pitch of the probabilities and of the logits' gradient
  int64_t piece, pieces;    // tokens per piece
  bool pack_hidden, pack_weight;
  int64_t blocks;           // pairs of statistics per token
  HeadProduct logits[2], hidden[2], weight[2];      // of a whole piece; of the last one
  // byte offsets of the workspace's sections
  size_t packed_weight, packed_hidden, masked_hidden, stats, entry, value, scale, lse, peak, kept, prob, grad, partial, sum;
  size_t total;
};

// The product of an m x k by a k x n operand for a device of 256 compute units; the sums of K's runs may take partial_bytes (0: one run).
HeadProduct head_product(int64_t m, int64_t n, int64_t k, int pairs, int64_t partial_bytes);
// Workspace to give a call: what the fastest plan takes with pieces of kHeadPieceTokens (max_bytes 0), or with one piece of all tokens; where that is
// more than max_bytes, all of these; the smallest workspace at least.  Never less for more tokens, vocabulary or entries, or for a higher limit.
size_t head_workspace(const HeadShape& shape, size_t max_bytes);
// The plan of a call that has so many bytes (0: pieces of kHeadPieceTokens, whatever they take): the largest pieces that fit, K in runs where
// there is room for their sums.  False, with the plan of the smallest pieces, where nothing fits.
bool head_plan(const HeadShape& shape, size_t max_bytes, HeadPlan* out);

}  // namespace muon
