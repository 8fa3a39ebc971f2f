// How a call for log probabilities is cut up: tokens in pieces, the workspace's sections (plain C++, no HIP include).
#pragma once
#include "head_plan.h"

namespace muon {

constexpr int kScoreMaxTop = 64;
// Alternatives are picked among so many more than are asked for: fp32 sums may order logits otherwise that are nearly alike.  With none, 4 and 12 more: 4096 x
// 100003 x 2048, top 8, 1495, 1507, 1530 us; 8 x 32768 x 1024, top 5, 23.3, 25.0, 25.9.
constexpr int kScoreMargin = 4;
// Vocabulary entries of a group, of which the largest logit is kept.
constexpr int kScoreGroup = 32;

// Calls of so few tokens, fp32 or of rows that would be copied first, go through W's rows as they are.  Both sides in us, with 5 alternatives: fp32
// 100003 x 2048 with 1, 64, 96 tokens 892, 935, 940 in planes, 200, 481, 789 so; 32768 x 1024 125, 137, 142 and 47, 71, 138; 20000 x 777 77, 88,
// 90 and 28, 63, 116.  bf16 20000 x 777 with 1, 16, 32 tokens 40, 41, 49 copied, 31, 39, 49 so; 32768 x 1024, not copied, 25, 31, 29 and 25, 27,
// 34: the tiles stay.
constexpr int64_t kScoreFew = 16, kScoreFewF32 = 64;

struct ScorePlan {
  HeadPlan shape;           // planes, pairs, width_k, pack_*, blocks
  bool few;
  int64_t groups;           // per token, whole blocks of them
  int64_t piece, pieces;
  HeadProduct logits[2];    // of a whole piece; of the last one
  // byte offsets of the workspace's sections
  size_t packed_weight, packed_hidden, stats, best;
  size_t total;
};

// Bytes for a call: pieces of up to kHeadPieceTokens (max_bytes 0), or the largest that fit, the smallest there are at least.
size_t score_workspace(const HeadShape& s, bool best, size_t max_bytes);
bool score_few(const HeadShape& s);
// Bytes of what a call keeps for its backward call: values of all tokens, then (bf16) the blocks' tops.  0 for few tokens that go through W's rows as
// they are: both calls would copy W where now one does (fp32 8 x 20011 x 2048, forward and backward, 394 us kept, 362 not).
int64_t score_kept_values(const HeadShape& s);
size_t score_kept_bytes(const HeadShape& s);
// The largest pieces that fit into so many bytes; false where none do.  keep: the call leaves something for a backward one.
bool score_plan(const HeadShape& s, bool best, bool keep, size_t bytes, ScorePlan* p);

}  // namespace muon
