// Device-side arguments and host-callable launchers of the head's losses (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "head_plan.h"

namespace muon {

// One operand of a product: `rows` of K contiguous elements at a pitch of ld, or, K-major, K rows of `rows` contiguous ones.  16-byte
// aligned, pitch a multiple of 8; elements up to the next multiple of 8 behind a row's end may be read, and are zero where the row
// runs along K.  An fp32 operand is the sum of three bf16 arrays, `plane` elements apart.
struct HeadOperand {
  const uint16_t* p;
  long long ld, plane;
  long long rows;
};

struct HeadTiles {
  long long k;
  int pairs;
  int tiles_m, tiles_n, whole;
  int splits, slabs_per_split;
};

inline HeadTiles tiles_of(const HeadProduct& g, int pairs) { return {g.k, pairs, g.tiles_m, g.tiles_n, g.whole, g.splits, g.slabs_per_split}; }

// Where a gradient's tiles go.  out: n rows of m elements, dense.  partial (splits > 1): [split][n][m] in fp32.  sum: fp32 [n][m],
// the pieces of tokens before (add) and with this one (keep).  Results are times `scale` and *peak (null: 1).
struct HeadOut {
  void* out;
  int f32;
  float* partial;
  float* sum;
  int add, keep;
  float scale;
  const float* peak;
};

// logits: L = weight, R = hidden, in units of log 2: y = unit z, unit = log2(e) / tau.  Per block of kHeadGrain vocabulary entries and token
// the pair (bias, sum of 2^(y + bias)), the largest of these powers being 2^15; with `prob` what the gradient needs: these powers in f16,
// or, fp32, z.
hipError_t launch_head_logits(const HeadOperand& weight, const HeadOperand& hidden, const HeadProduct& g, int pairs, float unit, float2* stats,
                              long long stats_pitch, void* prob, long long prob_pitch, int prob_f32, hipStream_t s);
// out = L R^T with L K-major; R plain or K-major.
hipError_t launch_head_product(const HeadOperand& l, const HeadOperand& r, int r_kmajor, const HeadProduct& g, int pairs,
                               const HeadOut& out, hipStream_t s);

// Rows [0, n) of a bf16 or fp32 matrix as operand planes of pitch ld, zero from `width` on.
hipError_t launch_head_pack(const void* src, long long stride, int f32, long long n, long long width, uint16_t* dst, long long ld,
                            long long plane, hipStream_t s);

// What the target of a token is.  Cross entropy: `index` of one entry (targets); distillation: `top` entries with the teacher's logits.
struct HeadTarget {
  const void* index;
  int index64;
  const void* logits;       // null: cross entropy
  int logits_bf16;
  int top;
  float inv_tau, tau;
  const float* token_scale;
};
// The logits (over tau) of the tokens' entries, and, with `masked`, the tokens' hidden states as operand planes, zeros where the token has no gradient;
// with `kept`, the tokens' scales, 0 where there is no gradient.
hipError_t launch_head_entries(const HeadTarget& t, const void* hidden, long long hidden_stride, const void* weight,
                               long long weight_stride, int f32, long long tokens, long long vocab, long long width, float* entry,
                               uint16_t* masked, long long ld, long long plane, float* kept, hipStream_t s);
// *peak = the largest finite |kept|, or 1: by a launch of its own, or, for few tokens, by the join.
hipError_t launch_head_peak(const float* kept, long long tokens, float* peak, hipStream_t s);
// Joins the pairs: loss and, if wanted, lse per token; with `value`, the gradients at the entries over tau and *peak, the scale of the others, and
// log2 of the sum of 2^y in two floats.  peak null: all scales count as they are.  entry null (one entry per token): the entries' logits
// are computed here, from the rows themselves.
struct HeadRows {
  const void *hidden, *weight;
  long long hidden_stride, weight_stride, width;
  int f32;
};
hipError_t launch_head_join(const HeadTarget& t, float unit, const float* kept, float* peak, const float2* stats,
                            long long stats_pitch, long long blocks, const float* entry, const HeadRows& rows, long long tokens, long long vocab,
                            float* loss, float* lse, float* value, float* scale, float2* log2sum, hipStream_t s);
// The logits' gradient in bf16 (in place of the probabilities) or three planes.
hipError_t launch_head_grad(const HeadTarget& t, float unit, const float2* stats, long long stats_pitch, const float2* log2sum,
                            const float* value, const float* scale, long long tokens, long long vocab, const void* prob, long long pitch,
                            int f32, uint16_t* grad, long long plane, hipStream_t s);
// Sums the splits of a product.
hipError_t launch_head_sum_splits(const HeadOut& out, int splits, long long count, hipStream_t s);
hipError_t launch_fill_zero(void* p, size_t bytes, hipStream_t s);

}  // namespace muon
