// How a call for log probabilities is cut up: tokens in pieces, the workspace's sections (plain C++, no HIP include).
#pragma once
#include "head_plan.h"

namespace muon {

constexpr int kScoreMaxTop = 64;
// Alternatives are picked among so many more than are asked for: fp32 sums may order logits otherwise that are nearly alike.
constexpr int kScoreMargin = 4;
// Vocabulary entries of a group, of which the largest logit is kept.
constexpr int kScoreGroup = 32;

struct ScorePlan {
  HeadPlan shape;           // planes, pairs, width_k, pack_*, blocks
  int64_t groups;           // per token, whole blocks of them
  int64_t piece, pieces;
  HeadProduct logits[2];    // of a whole piece; of the last one
  // byte offsets of the workspace's sections
  size_t packed_weight, packed_hidden, stats, best;
  size_t total;
};

// Bytes for a call: pieces of up to kHeadPieceTokens (max_bytes 0), or the largest that fit, the smallest there are at least.
size_t score_workspace(const HeadShape& s, bool best, size_t max_bytes);
// Bytes of what a call keeps for its backward call: values of all tokens, then (bf16) the blocks' tops.
int64_t score_kept_values(const HeadShape& s);
size_t score_kept_bytes(const HeadShape& s);
// The largest pieces that fit into so many bytes; false where none do.
bool score_plan(const HeadShape& s, bool best, size_t bytes, ScorePlan* p);

}  // namespace muon
