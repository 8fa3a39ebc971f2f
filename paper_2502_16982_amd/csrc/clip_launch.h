// Host-callable launchers of the gradients' norm and scaling (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "clip_batch.h"

namespace muon {

// One partial sum of squares per block.  stream: with the streaming hint.
hipError_t launch_grad_squares(const GradBatch& b, int blocks, bool stream, double* partial, hipStream_t s);
// *norm and, if wanted, *scale from n partial sums; up to n / kGradJoin + 1 more are written behind them.
hipError_t launch_grad_norm(double* partial, int64_t n, double max_norm, double* norm, float* scale, hipStream_t s);
// The same and the scaling for a list of one launch with up to kGradFew partial sums.
constexpr int kGradFew = 256;
hipError_t launch_grad_norm_scale(const GradBatch& b, int blocks, const double* partial, int n, double max_norm, double* norm, float* scale, hipStream_t s);
// Nothing is touched where *scale is 1.
hipError_t launch_grad_scale(const GradBatch& b, int blocks, const float* scale, hipStream_t s);

}  // namespace muon
