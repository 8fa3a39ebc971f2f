// C ABI of the head's losses (include/muon.h): checks, the sequence of launches of each piece of tokens.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api_guard.h"
#include "head_launch.h"

using namespace muon;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Sizes and types of a call; fills in what the plan goes by.
int head_shape(const muon_head* h, int32_t top, bool d_hidden, bool d_weight, HeadShape* s) {
  if (!h || h->reserved != 0) return MUON_E_INVALID_ARG;
  if (h->dtype != MUON_F32 && h->dtype != MUON_BF16) return MUON_E_UNSUPPORTED_DTYPE;
  if (h->tokens < 0 || h->tokens > kHeadMaxTokens || h->vocab < 1 || h->vocab > kHeadMaxVocab || h->width < 1 || h->width > kHeadMaxWidth ||
      top < 1 || top > kHeadMaxTop || h->hidden_stride < h->width || h->weight_stride < h->width)
    return MUON_E_INVALID_ARG;
  const uintptr_t size = h->dtype == MUON_F32 ? 4 : 2;
  if (!aligned(h->hidden, size) || !aligned(h->weight, size)) return MUON_E_MISALIGNED;
  *s = {h->tokens, h->vocab, h->width, h->hidden_stride, h->weight_stride, h->dtype == MUON_F32, aligned(h->hidden, 16),
        aligned(h->weight, 16), top, d_hidden, d_weight};
  return MUON_OK;
}

struct HeadOutputs {
  float *loss, *lse;
  void *d_hidden, *d_weight;
};

int run_head(const muon_head* h, const HeadTarget& target, const HeadOutputs& out, void* workspace, size_t workspace_bytes, hipStream_t s) {
  HeadShape shape;
  if (int st = head_shape(h, target.top, out.d_hidden != nullptr, out.d_weight != nullptr, &shape)) return st;
  const uintptr_t size = shape.f32 ? 4 : 2;
  if (!h->weight || (shape.tokens && (!h->hidden || !target.index || !out.loss))) return MUON_E_INVALID_ARG;
  if (!aligned(target.index, target.index64 ? 8 : 4) || !aligned(target.logits, target.logits_bf16 ? 2 : 4) ||
      !aligned(target.token_scale, 4) || !aligned(out.loss, 4) || !aligned(out.lse, 4) || !aligned(out.d_hidden, size) ||
      !aligned(out.d_weight, size) || !aligned(workspace, 256))
    return MUON_E_MISALIGNED;
  const size_t elem = shape.f32 ? 4 : 2;
  if (shape.tokens == 0) {
    if (out.d_weight) MUON_HIP(launch_fill_zero(out.d_weight, elem * shape.vocab * shape.width, s));
    return MUON_OK;
  }
  HeadPlan p;
  if (!workspace || workspace_bytes == 0 || !head_plan(shape, workspace_bytes, &p)) return MUON_E_WORKSPACE_TOO_SMALL;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  auto u16_at = [&](size_t at) { return reinterpret_cast<uint16_t*>(ws + at); };
  auto f32_at = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  const bool gradients = shape.d_hidden || shape.d_weight;
  const float unit = (float)(1.44269504088896340736 * (double)target.inv_tau);
  // dz goes through the products over the largest scale of the piece's tokens that have a gradient: where all are alike the target's entries
  // stay near -1, which bf16 holds exactly
  float *peak = nullptr, *kept = nullptr;
  if (gradients && target.token_scale) peak = f32_at(p.peak), kept = f32_at(p.kept);

  HeadOperand weight{static_cast<const uint16_t*>(h->weight), h->weight_stride, 0, shape.vocab};
  if (p.pack_weight) {
    weight = {u16_at(p.packed_weight), p.width_k, shape.vocab * p.width_k, shape.vocab};
    MUON_HIP(launch_head_pack(h->weight, h->weight_stride, shape.f32, shape.vocab, shape.width, u16_at(p.packed_weight), weight.ld,
                              weight.plane, s));
  }
  for (int64_t piece = 0; piece < p.pieces; ++piece) {
    const int last = piece == p.pieces - 1;
    const int64_t t0 = piece * p.piece, n = std::min(p.piece, shape.tokens - t0);
    const unsigned char* rows = static_cast<const unsigned char*>(h->hidden) + elem * t0 * h->hidden_stride;
    HeadTarget t = target;
    t.index = static_cast<const unsigned char*>(target.index) + (size_t)(target.index64 ? 8 : 4) * t0 * target.top;
    if (t.logits) t.logits = static_cast<const unsigned char*>(target.logits) + (size_t)(target.logits_bf16 ? 2 : 4) * t0 * target.top;
    if (t.token_scale) t.token_scale += t0;
    HeadOperand hidden{reinterpret_cast<const uint16_t*>(rows), h->hidden_stride, 0, n};
    if (p.pack_hidden) {
      hidden = {u16_at(p.packed_hidden), p.width_k, p.piece * p.width_k, n};
      MUON_HIP(launch_head_pack(rows, h->hidden_stride, shape.f32, n, shape.width, u16_at(p.packed_hidden), hidden.ld, hidden.plane, s));
    }
    uint16_t* masked = shape.d_weight ? u16_at(p.masked_hidden) : nullptr;
    const int64_t masked_plane = p.piece * p.width_k;
    // forward only with one entry: the join makes its logit, a launch less (16 x 32768 x 1024: 23.5 -> 22.5 us on the device, 64 x 50257 x 768:
    // 26.2 -> 25.2, 8192 x 16000 x 512: 163 -> 159); with two, one after the other, they take as long as the launch or longer (23.7 against 24.7)
    const bool entries = gradients || t.top > 1;
    if (entries)
      MUON_HIP(launch_head_entries(t, rows, h->hidden_stride, h->weight, h->weight_stride, shape.f32, n, shape.vocab, shape.width,
                                   f32_at(p.entry), masked, p.width_k, masked_plane, kept, s));
    if (peak) MUON_HIP(launch_head_peak(kept, n, peak, s));
    float2* stats = reinterpret_cast<float2*>(ws + p.stats);
    MUON_HIP(launch_head_logits(weight, hidden, p.logits[last], p.pairs, unit, stats, p.piece, gradients ? ws + p.prob : nullptr,
                                p.vocab_pitch, shape.f32, s));
    float2* log2sum = reinterpret_cast<float2*>(ws + p.lse);
    const HeadRows both{rows, h->weight, h->hidden_stride, h->weight_stride, shape.width, shape.f32};
    MUON_HIP(launch_head_join(t, unit, kept, peak, stats, p.piece, p.blocks, entries ? f32_at(p.entry) : nullptr,
                              both, n, shape.vocab, out.loss + t0, out.lse ? out.lse + t0 : nullptr, gradients ? f32_at(p.value) : nullptr,
                              f32_at(p.scale), log2sum, s));
    if (!gradients) continue;
    const int64_t grad_plane = p.piece * p.vocab_pitch;
    MUON_HIP(launch_head_grad(t, unit, stats, p.piece, log2sum, f32_at(p.value), f32_at(p.scale), n, shape.vocab, ws + p.prob,
                              p.vocab_pitch, shape.f32, u16_at(p.grad), grad_plane, s));
    if (shape.d_hidden) {
      const HeadOut o{static_cast<unsigned char*>(out.d_hidden) + elem * t0 * shape.width, shape.f32, f32_at(p.partial), nullptr, 0, 0, target.tau, peak};
      const HeadOperand l{weight.p, weight.ld, weight.plane, shape.width}, r{u16_at(p.grad), p.vocab_pitch, grad_plane, n};
      const HeadProduct& g = p.hidden[last];
      MUON_HIP(launch_head_product(l, r, 0, g, p.pairs, o, s));
      if (g.splits > 1) MUON_HIP(launch_head_sum_splits(o, g.splits, n * shape.width, s));
    }
    if (shape.d_weight) {
      const HeadOut o{out.d_weight, shape.f32, f32_at(p.partial), f32_at(p.sum), piece > 0, !last, target.tau, peak};
      const HeadOperand l{masked, p.width_k, masked_plane, shape.width}, r{u16_at(p.grad), p.vocab_pitch, grad_plane, shape.vocab};
      const HeadProduct& g = p.weight[last];
      MUON_HIP(launch_head_product(l, r, 1, g, p.pairs, o, s));
      if (g.splits > 1) MUON_HIP(launch_head_sum_splits(o, g.splits, shape.vocab * shape.width, s));
    }
  }
  return MUON_OK;
}

}  // namespace

extern "C" {

int muon_head_workspace_bytes(const muon_head* head, int32_t top, int32_t gradients, size_t max_bytes, size_t* out) {
  return guarded([&]() -> int {
    if (!out || gradients < 0 || gradients > 3) return MUON_E_INVALID_ARG;
    HeadShape shape;
    if (int st = head_shape(head, top, (gradients & MUON_HEAD_D_HIDDEN) != 0, (gradients & MUON_HEAD_D_WEIGHT) != 0, &shape)) return st;
    *out = head_workspace(shape, max_bytes);
    return MUON_OK;
  });
}

int muon_cross_entropy(const muon_head* head, const void* targets, int32_t targets_bytes, const float* token_scale, float* loss, float* lse,
                       void* d_hidden, void* d_weight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    if (targets_bytes != 4 && targets_bytes != 8) return MUON_E_INVALID_ARG;
    const HeadTarget t{targets, targets_bytes == 8, nullptr, 0, 1, 1.f, 1.f, token_scale};
    return run_head(head, t, {loss, lse, d_hidden, d_weight}, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
  });
}

int muon_distill(const muon_head* head, const void* index, int32_t index_bytes, const void* teacher_logits, int32_t teacher_dtype, int32_t top,
                 double temperature, const float* token_scale, float* loss, float* lse, void* d_hidden, void* d_weight, void* workspace,
                 size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    if ((index_bytes != 4 && index_bytes != 8) || !(temperature > 0.0) || !std::isfinite((float)temperature) ||
        !std::isfinite((float)(1.0 / temperature)) || (float)(1.0 / temperature) == 0.f || (float)temperature == 0.f)
      return MUON_E_INVALID_ARG;
    if (teacher_dtype != MUON_F32 && teacher_dtype != MUON_BF16) return MUON_E_UNSUPPORTED_DTYPE;
    if (!teacher_logits && head && head->tokens > 0) return MUON_E_INVALID_ARG;
    const HeadTarget t{index, index_bytes == 8, teacher_logits, teacher_dtype == MUON_BF16, top, (float)(1.0 / temperature), (float)temperature,
                       token_scale};
    return run_head(head, t, {loss, lse, d_hidden, d_weight}, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
  });
}

}  // extern "C"
