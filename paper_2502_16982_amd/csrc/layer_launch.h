// Device-side arguments and host-callable launchers of a mixture's layer for few tokens (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include "layer_plan.h"

namespace muon {

// The pairs (token, choice) of a call and their experts.
struct LayerPairs {
  const void* expert;       // [tokens, top], -1 or beyond the experts: no pair
  int index64;
  int pairs, top, experts;
  int slots, slot_is_pair;
};

// One matrix of each expert: K x N, rows contiguous.
struct LayerMatrix {
  const void* w;
  long long expert_stride, row_stride;     // elements
};

// Rows that are multiplied: pair p's at row p / per (per = top: the token's row).
struct LayerRows {
  const void* x;
  long long stride;
  int per;
};

// Rows that the first product left as sums of its runs, [run][pair][matrix][n]; `act` is still to be applied.
struct LayerSums {
  const float* part;
  long long n;
  int runs, mats, act;
};

// out[run][pair][matrix][N] in fp32, or, one run and `act` >= 0, the activated rows [pair][N] in the inputs' type.  from: the rows instead of x; runs
// of the summed axis of up to kLayerStage bytes for 2 x 16 pairs.
hipError_t launch_layer_product(const LayerPairs& p, const LayerProduct& g, const LayerRows& x, const LayerMatrix& w, const LayerMatrix* gate,
                                const LayerSums* from, bool f32, int act, void* out, hipStream_t s);
// The activated rows from the sums of the runs.
hipError_t launch_layer_act(const LayerPairs& p, int runs, long long n, bool gated, bool f32, int act, const float* part, void* inner, hipStream_t s);
// out[t] = sum_j weights[t, j] sum_run rows[run][t, j].
hipError_t launch_layer_join(const LayerPairs& p, int runs, long long n, bool f32, const float* rows, const float* weights, void* out, hipStream_t s);

}  // namespace muon
