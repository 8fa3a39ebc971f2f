// C ABI of the experts' sort, dispatch and combine (include/muon.h).
#include <hip/hip_runtime.h>

#include "api_guard.h"
#include "experts_launch.h"

using namespace muon;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_sizes(int64_t tokens, int32_t top, int32_t experts) {
  if (tokens < 0 || top < 1 || top > kMaxExpertTop || experts < 1 || experts > kMaxExperts || tokens > kMaxExpertPairs / top)
    return MUON_E_INVALID_ARG;
  return MUON_OK;
}

int expert_rows(const muon_routing* g, int64_t width, int32_t dtype, ExpertRows* r) {
  if (!g) return MUON_E_INVALID_ARG;
  if (int st = check_sizes(g->tokens, g->top, g->experts)) return st;
  if (dtype != MUON_F32 && dtype != MUON_BF16) return MUON_E_UNSUPPORTED_DTYPE;
  if (width < 1 || width > (1ll << 30) || (g->tokens && (!g->position || !g->offsets))) return MUON_E_INVALID_ARG;
  if (!aligned(g->position, 4) || !aligned(g->offsets, 4)) return MUON_E_MISALIGNED;
  *r = {g->position, g->offsets ? g->offsets + g->experts : nullptr, g->tokens, width, g->top, dtype == MUON_F32};
  return MUON_OK;
}

}  // namespace

extern "C" {

int muon_expert_sort_bytes(int64_t tokens, int32_t top, int32_t experts, size_t* out) {
  return guarded([&]() -> int {
    if (!out) return MUON_E_INVALID_ARG;
    if (int st = check_sizes(tokens, top, experts)) return st;
    const int blocks = sort_blocks(tokens * top);
    *out = blocks > 1 ? sizeof(int) * (size_t)blocks * experts : 0;
    return MUON_OK;
  });
}

int muon_expert_sort(const void* expert, int32_t expert_bytes, int64_t tokens, int32_t top, int32_t experts, int32_t* position, int32_t* source,
                     int32_t* offsets, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    if (expert_bytes != 4 && expert_bytes != 8) return MUON_E_INVALID_ARG;
    size_t need = 0;
    if (int st = muon_expert_sort_bytes(tokens, top, experts, &need)) return st;
    if (!offsets || (tokens && (!expert || !position || !source))) return MUON_E_INVALID_ARG;
    if (!aligned(expert, expert_bytes) || !aligned(position, 4) || !aligned(source, 4) || !aligned(offsets, 4) || !aligned(workspace, 4))
      return MUON_E_MISALIGNED;
    if (need && (!workspace || workspace_bytes < need)) return MUON_E_WORKSPACE_TOO_SMALL;
    MUON_HIP(launch_expert_sort(expert, expert_bytes == 8, tokens * top, experts, position, source, offsets, static_cast<int*>(workspace),
                                static_cast<hipStream_t>(hip_stream)));
    return MUON_OK;
  });
}

int muon_expert_dispatch(const muon_routing* routing, const void* x, int64_t x_stride, int64_t width, int32_t dtype, void* rows, void* hip_stream) {
  return guarded([&]() -> int {
    ExpertRows r;
    if (int st = expert_rows(routing, width, dtype, &r)) return st;
    if (r.tokens == 0) return MUON_OK;
    const uintptr_t size = r.f32 ? 4 : 2;
    if (!x || !rows || x_stride < width) return MUON_E_INVALID_ARG;
    if (!aligned(x, size) || !aligned(rows, size)) return MUON_E_MISALIGNED;
    MUON_HIP(launch_expert_dispatch(r, x, x_stride, rows, static_cast<hipStream_t>(hip_stream)));
    return MUON_OK;
  });
}

int muon_expert_combine(const muon_routing* routing, const void* rows, const float* weights, int64_t width, int32_t dtype, void* out,
                        void* hip_stream) {
  return guarded([&]() -> int {
    ExpertRows r;
    if (int st = expert_rows(routing, width, dtype, &r)) return st;
    if (r.tokens == 0) return MUON_OK;
    const uintptr_t size = r.f32 ? 4 : 2;
    if (!rows || !out) return MUON_E_INVALID_ARG;
    if (!aligned(rows, size) || !aligned(out, size) || !aligned(weights, 4)) return MUON_E_MISALIGNED;
    MUON_HIP(launch_expert_combine(r, rows, weights, out, static_cast<hipStream_t>(hip_stream)));
    return MUON_OK;
  });
}

int muon_expert_combine_backward(const muon_routing* routing, const void* d_out, int64_t d_out_stride, const void* rows, const float* weights,
                                 int64_t width, int32_t dtype, void* d_rows, float* d_weights, void* hip_stream) {
  return guarded([&]() -> int {
    ExpertRows r;
    if (int st = expert_rows(routing, width, dtype, &r)) return st;
    if (r.tokens == 0) return MUON_OK;
    const uintptr_t size = r.f32 ? 4 : 2;
    if (!d_out || !rows || !weights || !d_rows || !d_weights || d_out_stride < width) return MUON_E_INVALID_ARG;
    if (!aligned(d_out, size) || !aligned(rows, size) || !aligned(weights, 4) || !aligned(d_rows, size) || !aligned(d_weights, 4))
      return MUON_E_MISALIGNED;
    MUON_HIP(launch_expert_combine_backward(r, d_out, d_out_stride, rows, weights, d_rows, d_weights, static_cast<hipStream_t>(hip_stream)));
    return MUON_OK;
  });
}

}  // extern "C"
