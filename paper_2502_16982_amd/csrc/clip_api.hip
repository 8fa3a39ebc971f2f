// C ABI of the gradients' norm and clipping (include/muon.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "api_guard.h"
#include "clip_launch.h"

using namespace muon;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_sizes(const muon_grad* grads, int32_t n) {
  if (n < 0 || (n && !grads)) return MUON_E_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i) {
    const muon_grad& q = grads[i];
    if (q.dtype != MUON_F32 && q.dtype != MUON_BF16) return MUON_E_UNSUPPORTED_DTYPE;
    if (q.reserved != 0 || q.numel < 0 || q.numel > kGradMaxNumel) return MUON_E_INVALID_ARG;
  }
  return MUON_OK;
}

int check_list(const muon_grad* grads, int32_t n) {
  if (int st = check_sizes(grads, n)) return st;
  for (int32_t i = 0; i < n; ++i) {
    if (grads[i].numel && !grads[i].g) return MUON_E_INVALID_ARG;
    if (!aligned(grads[i].g, grads[i].dtype == MUON_BF16 ? 2 : 4)) return MUON_E_MISALIGNED;
  }
  return MUON_OK;
}

// Whether two tensors share memory: what is scaled twice, by two blocks at a time, would have no defined value.
bool overlap(const muon_grad* grads, int32_t n) {
  struct Range {
    uintptr_t from, to;
  };
  auto range = [&](int32_t i) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(grads[i].g);
    return Range{p, p + (uintptr_t)grads[i].numel * (grads[i].dtype == MUON_BF16 ? 2 : 4)};
  };
  bool rising = true;                            // as slices of one buffer are
  uintptr_t end = 0;
  for (int32_t i = 0; i < n && rising; ++i) {
    const Range r = range(i);
    if (r.from == r.to) continue;
    rising = r.from >= end;
    end = r.to;
  }
  if (rising) return false;
  std::vector<Range> all;
  all.reserve((size_t)n);
  for (int32_t i = 0; i < n; ++i)
    if (grads[i].numel) all.push_back(range(i));
  std::sort(all.begin(), all.end(), [](const Range& x, const Range& y) { return x.from < y.from; });
  for (size_t i = 1; i < all.size(); ++i)
    if (all[i].from < all[i - 1].to) return true;
  return false;
}

// in_place: and scales the gradients.
int run_norm(const muon_grad* grads, int32_t n, double max_norm, double* norm, float* scale, bool in_place, void* workspace, size_t workspace_bytes,
             hipStream_t s) {
  if (!(max_norm >= 0.0) || !norm) return MUON_E_INVALID_ARG;
  if (!aligned(norm, 8) || !aligned(scale, 4) || !aligned(workspace, 8)) return MUON_E_MISALIGNED;
  const int64_t partials = grad_partials(grads, n);
  if (!workspace || workspace_bytes < grad_workspace(partials)) return MUON_E_WORKSPACE_TOO_SMALL;
  double* partial = static_cast<double*>(workspace);
  GradBatch b{};
  GradCursor at;
  int64_t done = 0;
  while (const int blocks = grad_next_batch(grads, n, at, b)) {
    MUON_HIP(launch_grad_squares(b, blocks, in_place, partial + done, s));
    done += blocks;
    if (in_place && blocks == partials && blocks <= kGradFew) {
      MUON_HIP(launch_grad_norm_scale(b, blocks, partial, blocks, max_norm, norm, scale, s));
      return MUON_OK;
    }
  }
  MUON_HIP(launch_grad_norm(partial, partials, max_norm, norm, scale, s));
  if (!in_place) return MUON_OK;
  at = GradCursor{};
  while (const int blocks = grad_next_batch(grads, n, at, b)) MUON_HIP(launch_grad_scale(b, blocks, scale, s));
  return MUON_OK;
}

}  // namespace

extern "C" {

int muon_grad_norm_bytes(const muon_grad* grads, int32_t n, size_t* out) {
  return guarded([&]() -> int {
    if (!out) return MUON_E_INVALID_ARG;
    if (int st = check_sizes(grads, n)) return st;
    *out = grad_workspace(grad_partials(grads, n));
    return MUON_OK;
  });
}

int muon_grad_norm(const muon_grad* grads, int32_t n, double max_norm, double* norm, float* scale, void* workspace, size_t workspace_bytes,
                   void* hip_stream) {
  return guarded([&]() -> int {
    if (int st = check_list(grads, n)) return st;
    return run_norm(grads, n, max_norm, norm, scale, false, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
  });
}

int muon_grad_scale(const muon_grad* grads, int32_t n, const float* scale, void* hip_stream) {
  return guarded([&]() -> int {
    if (int st = check_list(grads, n)) return st;
    if (!scale || overlap(grads, n)) return MUON_E_INVALID_ARG;
    if (!aligned(scale, 4)) return MUON_E_MISALIGNED;
    GradBatch b{};
    GradCursor at;
    while (const int blocks = grad_next_batch(grads, n, at, b)) MUON_HIP(launch_grad_scale(b, blocks, scale, static_cast<hipStream_t>(hip_stream)));
    return MUON_OK;
  });
}

int muon_grad_clip(const muon_grad* grads, int32_t n, double max_norm, double* norm, float* scale, void* workspace, size_t workspace_bytes,
                   void* hip_stream) {
  return guarded([&]() -> int {
    if (int st = check_list(grads, n)) return st;
    if (!scale || overlap(grads, n)) return MUON_E_INVALID_ARG;
    return run_norm(grads, n, max_norm, norm, scale, true, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
  });
}

}  // extern "C"
