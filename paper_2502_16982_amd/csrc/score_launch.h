// Device-side arguments and host-callable launchers of the head's log probabilities (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include "head_launch.h"

namespace muon {

// The given tokens; index null: none.
struct ScoreTarget {
  const void* index;
  int index64;
};

// What the logits' product leaves behind, y = unit z (units of log 2).  Per token and block of kHeadGrain vocabulary entries: its largest y as `top`,
// sum of 2^(y - top), sum of 2^(y - top) (y - top).  With `best`, per token and group of kScoreGroup entries: its largest z, and its second largest
// as a bound from above whose low five bits are the largest one's place in the group.
struct ScoreStats {
  float top, sum, slope, unused;
};
struct ScoreBest {
  float z;
  unsigned second;
};
// What a forward call keeps for the backward one, [tokens, pitch]: powers 2^(15 + y - top) in f16, up to 2^15 in a block, with each block's top per
// token; or, tops null, z in fp32.  values null: nothing.  Not together with `best`.  (f16: its step is an eighth of the one that dz is rounded by;
// fp32 would double what both calls move most of.)
struct ScoreKept {
  void* values;
  long long pitch;
  float* tops;
};
hipError_t launch_score_logits(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, ScoreStats* stats,
                               ScoreBest* best, const ScoreKept& kept, hipStream_t s);

// The same statistics for few tokens (16, fp32 64 at most), from the rows themselves.
hipError_t launch_score_few(const HeadRows& rows, long long tokens, long long vocab, float unit, ScoreStats* stats, ScoreBest* best, hipStream_t s);

struct ScoreOut {
  float *log_prob, *entropy, *lse, *lse_rest;      // log_prob null where there are no targets
  long long* top_index;
  float* top_log_prob;                             // [tokens, top]
};
// Joins the blocks; log probability of the given token and of the `top` largest logits, both from logits that are summed in double.
hipError_t launch_score_finish(const ScoreTarget& t, float inv_tau, float unit, const ScoreStats* stats, long long blocks,
                               const ScoreBest* best, long long groups, int top, const HeadRows& rows, long long tokens, long long vocab, const ScoreOut& out,
                               hipStream_t s);

// Per token of a piece: dz_v = -p_v (a + b log2 p_v) + [v = target] ..., whose whole value at the target is `value`; all over *peak.
struct ScoreCoef {
  float *a, *b, *value;
  float2* log2sum;                                 // of 2^y over the vocabulary, in two floats; infinite where the token has no gradient
};
struct ScoreGrads {
  const float *lse, *lse_rest, *entropy;           // of the forward call
  const float *d_log_prob, *d_entropy;             // d_entropy null: 0
};
// *peak = the largest finite |gradient| of the piece, or 1: by a launch of its own, or, for few tokens, by the preparation.
hipError_t launch_score_peak(const ScoreTarget& t, const ScoreGrads& d, long long tokens, long long vocab, float* peak, hipStream_t s);
// The coefficients, and, with `masked`, hidden states as operand planes, zeros where the token has no gradient.
hipError_t launch_score_prepare(const ScoreTarget& t, float inv_tau, float unit, const ScoreGrads& d, float* peak, const HeadRows& rows,
                                long long tokens, long long vocab, const ScoreCoef& c, uint16_t* masked, long long ld, long long plane, hipStream_t s);
// The logits' gradient over *peak, in bf16 or three planes, from the logits' product done again.
hipError_t launch_score_grad(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, const ScoreTarget& t,
                             const ScoreCoef& c, bool f32, uint16_t* grad, long long pitch, long long plane, hipStream_t s);
// The same from what the forward call kept.
hipError_t launch_score_dz(const ScoreTarget& t, float unit, const ScoreKept& kept, long long blocks, const ScoreCoef& c, long long tokens, long long vocab, bool f32,
                           uint16_t* grad, long long pitch, long long plane, hipStream_t s);

}  // namespace muon
