// C ABI of the experts' sort, dispatch and combine and of a mixture's layer for few tokens (include/muon.h).
#include <hip/hip_runtime.h>

#include "api_guard.h"
#include "experts_launch.h"
#include "layer_launch.h"

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

int layer_shape(const muon_layer* l, LayerShape* s) {
  if (!l || l->reserved != 0) return MUON_E_INVALID_ARG;
  if (l->dtype != MUON_F32 && l->dtype != MUON_BF16) return MUON_E_UNSUPPORTED_DTYPE;
  if (l->activation != MUON_ACT_SILU && l->activation != MUON_ACT_RELU) return MUON_E_INVALID_ARG;
  if (l->tokens < 0 || l->top < 1 || l->top > kLayerMaxTop || l->experts < 1 || l->experts > kLayerMaxExperts || l->tokens > kLayerMaxPairs / l->top ||
      l->width < 1 || l->width > kLayerMaxWidth || l->inner < 1 || l->inner > kLayerMaxWidth)
    return MUON_E_INVALID_ARG;
  *s = {l->tokens, l->width, l->inner, l->top, l->experts, l->gate.w != nullptr, l->dtype == MUON_F32};
  return MUON_OK;
}

}  // namespace

extern "C" {

int muon_expert_layer_bytes(const muon_layer* layer, size_t* out) {
  return guarded([&]() -> int {
    if (!out) return MUON_E_INVALID_ARG;
    LayerShape s;
    if (int st = layer_shape(layer, &s)) return st;
    *out = layer_plan(s).total;
    return MUON_OK;
  });
}

int muon_expert_layer(const muon_layer* layer, const void* x, int64_t x_stride, const void* expert, int32_t expert_bytes, const float* weights,
                      void* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    LayerShape s;
    if (int st = layer_shape(layer, &s)) return st;
    if (expert_bytes != 4 && expert_bytes != 8) return MUON_E_INVALID_ARG;
    if (s.tokens == 0) return MUON_OK;
    const uintptr_t size = s.f32 ? 4 : 2;
    const muon_matrices *up = &layer->up, *gate = &layer->gate, *down = &layer->down;
    if (!x || !expert || !out || !up->w || !down->w || x_stride < s.width || up->row_stride < s.inner || down->row_stride < s.width ||
        up->row_stride > kLayerMaxStride || down->row_stride > kLayerMaxStride || up->expert_stride < 0 || down->expert_stride < 0 ||
        (s.gated && (gate->row_stride < s.inner || gate->row_stride > kLayerMaxStride || gate->expert_stride < 0)))
      return MUON_E_INVALID_ARG;
    if (!aligned(x, size) || !aligned(expert, expert_bytes) || !aligned(weights, 4) || !aligned(out, size) || !aligned(up->w, size) ||
        !aligned(gate->w, size) || !aligned(down->w, size) || !aligned(workspace, 256))
      return MUON_E_MISALIGNED;
    const LayerPlan plan = layer_plan(s);
    if (!workspace || workspace_bytes < plan.total) return MUON_E_WORKSPACE_TOO_SMALL;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const LayerPairs pairs{expert, expert_bytes == 8, (int)(s.tokens * s.top), s.top, s.experts, plan.slots, plan.slot_is_pair};
    const LayerMatrix wu{up->w, up->expert_stride, up->row_stride}, wg{gate->w, gate->expert_stride, gate->row_stride},
        wd{down->w, down->expert_stride, down->row_stride};
    const LayerRows tokens{x, x_stride, s.top}, inner{ws + plan.inner, s.inner, 1};
    const int act = layer->activation;
    const bool runs = plan.up.runs > 1;
    const LayerSums sums{reinterpret_cast<const float*>(ws + plan.part), s.inner, plan.up.runs, s.gated ? 2 : 1, act};
    MUON_HIP(launch_layer_product(pairs, plan.up, tokens, wu, s.gated ? &wg : nullptr, nullptr, s.f32, runs ? -1 : act,
                                  runs ? ws + plan.part : ws + plan.inner, stream));
    if (runs && !plan.staged) MUON_HIP(launch_layer_act(pairs, plan.up.runs, s.inner, s.gated, s.f32, act, sums.part, ws + plan.inner, stream));
    MUON_HIP(launch_layer_product(pairs, plan.down, inner, wd, nullptr, plan.staged ? &sums : nullptr, s.f32, -1, ws + plan.rows, stream));
    MUON_HIP(launch_layer_join(pairs, plan.down.runs, s.width, s.f32, reinterpret_cast<const float*>(ws + plan.rows), weights, out, stream));
    return MUON_OK;
  });
}

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
