// C ABI of the head's log probabilities (include/muon.h): checks, the sequence of launches of each piece of tokens.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api_guard.h"
#include "score_launch.h"
#include "score_plan.h"

using namespace muon;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int score_shape(const muon_head* h, bool d_hidden, bool d_weight, HeadShape* s) {
  if (!h || h->reserved != 0) return MUON_E_INVALID_ARG;
  if (h->dtype != MUON_F32 && h->dtype != MUON_BF16) return MUON_E_UNSUPPORTED_DTYPE;
  if (h->tokens < 0 || h->tokens > kHeadMaxTokens || h->vocab < 1 || h->vocab > kHeadMaxVocab || h->width < 1 || h->width > kHeadMaxWidth ||
      h->hidden_stride < h->width || h->weight_stride < h->width)
    return MUON_E_INVALID_ARG;
  const uintptr_t size = h->dtype == MUON_F32 ? 4 : 2;
  if (!aligned(h->hidden, size) || !aligned(h->weight, size)) return MUON_E_MISALIGNED;
  *s = {h->tokens, h->vocab, h->width, h->hidden_stride, h->weight_stride, h->dtype == MUON_F32, aligned(h->hidden, 16), aligned(h->weight, 16),
        1, d_hidden, d_weight};
  return MUON_OK;
}

bool temperature_fits(double tau) {
  return tau > 0.0 && std::isfinite((float)tau) && std::isfinite((float)(1.0 / tau)) && (float)(1.0 / tau) != 0.f && (float)tau != 0.f;
}

const void* behind(const void* p, int64_t bytes) { return p ? static_cast<const unsigned char*>(p) + bytes : nullptr; }

ScoreKept kept_from(const HeadShape& s, const HeadPlan& p, void* kept, int64_t t0) {
  if (!kept) return {nullptr, 0, nullptr};
  unsigned char* at = static_cast<unsigned char*>(kept);
  float* tops = s.f32 ? nullptr : reinterpret_cast<float*>(at + score_kept_values(s)) + t0 * p.blocks;
  return {at + t0 * p.vocab_pitch * (s.f32 ? 4 : 2), p.vocab_pitch, tops};
}

struct Scale {
  float inv_tau, unit;
};
Scale scale_of(double tau) { return {(float)(1.0 / tau), (float)(1.44269504088896340736 * (double)(float)(1.0 / tau))}; }

// The operands of the logits' product, copied first where their rows ask for it.
int pack(const muon_head* h, const HeadShape& s, const HeadPlan& p, unsigned char* to, HeadOperand* weight, hipStream_t stream) {
  *weight = {static_cast<const uint16_t*>(h->weight), h->weight_stride, 0, s.vocab};
  if (!p.pack_weight) return MUON_OK;
  uint16_t* at = reinterpret_cast<uint16_t*>(to);
  *weight = {at, p.width_k, s.vocab * p.width_k, s.vocab};
  MUON_HIP(launch_head_pack(h->weight, h->weight_stride, s.f32, s.vocab, s.width, at, weight->ld, weight->plane, stream));
  return MUON_OK;
}
int pack_rows(const muon_head* h, const HeadShape& s, const HeadPlan& p, const void* rows, int64_t n, int64_t piece, unsigned char* to, HeadOperand* hidden,
              hipStream_t stream) {
  *hidden = {static_cast<const uint16_t*>(rows), h->hidden_stride, 0, n};
  if (!p.pack_hidden) return MUON_OK;
  uint16_t* at = reinterpret_cast<uint16_t*>(to);
  *hidden = {at, p.width_k, piece * p.width_k, n};
  MUON_HIP(launch_head_pack(rows, h->hidden_stride, s.f32, n, s.width, at, hidden->ld, hidden->plane, stream));
  return MUON_OK;
}

}  // namespace

extern "C" {

int muon_log_probs_bytes(const muon_head* head, int32_t top, size_t max_bytes, size_t* out) {
  return guarded([&]() -> int {
    HeadShape s;
    if (!out) return MUON_E_INVALID_ARG;
    if (int st = score_shape(head, false, false, &s)) return st;
    if (top < 0 || top > kScoreMaxTop || top > s.vocab) return MUON_E_INVALID_ARG;
    *out = score_workspace(s, top > 0, max_bytes);
    return MUON_OK;
  });
}

int muon_log_probs_kept_bytes(const muon_head* head, size_t* out) {
  return guarded([&]() -> int {
    HeadShape s;
    if (!out) return MUON_E_INVALID_ARG;
    if (int st = score_shape(head, false, false, &s)) return st;
    *out = score_kept_bytes(s);
    return MUON_OK;
  });
}

int muon_log_probs(const muon_head* h, const void* targets, int32_t targets_bytes, int32_t top, double temperature, float* log_prob, float* entropy,
                   float* lse, float* lse_rest, int64_t* top_index, float* top_log_prob, void* kept, size_t kept_bytes, void* workspace,
                   size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    HeadShape s;
    if (int st = score_shape(h, false, false, &s)) return st;
    if ((targets_bytes != 4 && targets_bytes != 8) || top < 0 || top > kScoreMaxTop || top > s.vocab || !temperature_fits(temperature) || (top && kept))
      return MUON_E_INVALID_ARG;
    if (s.tokens == 0) return MUON_OK;
    if (!h->weight || !h->hidden || !entropy || !lse || !lse_rest || (targets != nullptr) != (log_prob != nullptr) || (top && (!top_index || !top_log_prob)))
      return MUON_E_INVALID_ARG;
    if (!aligned(targets, targets_bytes) || !aligned(log_prob, 4) || !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(lse_rest, 4) ||
        !aligned(top_index, 8) || !aligned(top_log_prob, 4) || !aligned(kept, 256) || !aligned(workspace, 256))
      return MUON_E_MISALIGNED;
    if (kept && kept_bytes < score_kept_bytes(s)) return MUON_E_WORKSPACE_TOO_SMALL;
    if (score_kept_bytes(s) == 0) kept = nullptr;
    ScorePlan p;
    if (!workspace || !score_plan(s, top > 0, kept != nullptr, workspace_bytes, &p)) return MUON_E_WORKSPACE_TOO_SMALL;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const Scale scale = scale_of(temperature);
    const int64_t elem = s.f32 ? 4 : 2;
    HeadOperand weight{};
    if (!p.few)
      if (int st = pack(h, s, p.shape, ws + p.packed_weight, &weight, stream)) return st;
    ScoreStats* stats = reinterpret_cast<ScoreStats*>(ws + p.stats);
    ScoreBest* best = top ? reinterpret_cast<ScoreBest*>(ws + p.best) : nullptr;
    for (int64_t piece = 0; piece < p.pieces; ++piece) {
      const int64_t t0 = piece * p.piece, n = std::min(p.piece, s.tokens - t0);
      const HeadRows rows{behind(h->hidden, elem * t0 * h->hidden_stride), h->weight, h->hidden_stride, h->weight_stride, s.width, s.f32};
      if (p.few) {
        MUON_HIP(launch_score_few(rows, n, s.vocab, scale.unit, stats, best, stream));
      } else {
        HeadOperand hidden;
        if (int st = pack_rows(h, s, p.shape, rows.hidden, n, p.piece, ws + p.packed_hidden, &hidden, stream)) return st;
        MUON_HIP(launch_score_logits(weight, hidden, p.logits[piece == p.pieces - 1], p.shape.pairs, scale.unit, stats, best,
                                     kept_from(s, p.shape, kept, t0), stream));
      }
      const ScoreTarget t{behind(targets, targets_bytes * t0), targets_bytes == 8};
      const ScoreOut out{log_prob ? log_prob + t0 : nullptr, entropy + t0, lse + t0, lse_rest + t0,
                         top ? reinterpret_cast<long long*>(top_index) + t0 * top : nullptr, top ? top_log_prob + t0 * top : nullptr};
      MUON_HIP(launch_score_finish(t, scale.inv_tau, scale.unit, stats, p.shape.blocks, best, p.groups, top, rows, n, s.vocab, out, stream));
    }
    return MUON_OK;
  });
}

int muon_log_probs_backward(const muon_head* h, const void* targets, int32_t targets_bytes, double temperature, const float* lse, const float* lse_rest,
                            const float* entropy, const float* d_log_prob, const float* d_entropy, const void* kept, size_t kept_bytes, void* d_hidden,
                            void* d_weight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return guarded([&]() -> int {
    HeadShape s;
    if (int st = score_shape(h, d_hidden != nullptr, d_weight != nullptr, &s)) return st;
    if ((targets_bytes != 4 && targets_bytes != 8) || !temperature_fits(temperature) || !h->weight ||
        (s.tokens && (!h->hidden || !lse || !lse_rest || !entropy || (targets != nullptr) != (d_log_prob != nullptr) || (!d_log_prob && !d_entropy))))
      return MUON_E_INVALID_ARG;
    const uintptr_t size = s.f32 ? 4 : 2;
    if (!aligned(targets, targets_bytes) || !aligned(lse, 4) || !aligned(lse_rest, 4) || !aligned(entropy, 4) || !aligned(d_log_prob, 4) ||
        !aligned(d_entropy, 4) || !aligned(kept, 256) || !aligned(d_hidden, size) || !aligned(d_weight, size) || !aligned(workspace, 256))
      return MUON_E_MISALIGNED;
    if (kept && kept_bytes < score_kept_bytes(s)) return MUON_E_WORKSPACE_TOO_SMALL;
    if (score_kept_bytes(s) == 0) kept = nullptr;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (s.tokens == 0) {
      if (d_weight) MUON_HIP(launch_fill_zero(d_weight, size * s.vocab * s.width, stream));
      return MUON_OK;
    }
    if (!d_hidden && !d_weight) return MUON_OK;
    HeadPlan p;
    if (!workspace || workspace_bytes == 0 || !head_plan(s, workspace_bytes, &p)) return MUON_E_WORKSPACE_TOO_SMALL;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    auto u16_at = [&](size_t at) { return reinterpret_cast<uint16_t*>(ws + at); };
    auto f32_at = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
    const Scale scale = scale_of(temperature);
    HeadOperand weight;
    weight = {};
    if (!kept || s.d_hidden)
      if (int st = pack(h, s, p, ws + p.packed_weight, &weight, stream)) return st;
    for (int64_t piece = 0; piece < p.pieces; ++piece) {
      const int last = piece == p.pieces - 1;
      const int64_t t0 = piece * p.piece, n = std::min(p.piece, s.tokens - t0);
      const HeadRows rows{behind(h->hidden, (int64_t)size * t0 * h->hidden_stride), h->weight, h->hidden_stride, h->weight_stride, s.width, s.f32};
      const ScoreTarget t{behind(targets, targets_bytes * t0), targets_bytes == 8};
      const ScoreGrads d{lse + t0, lse_rest + t0, entropy + t0, d_log_prob ? d_log_prob + t0 : nullptr, d_entropy ? d_entropy + t0 : nullptr};
      const ScoreCoef c{f32_at(p.scale), f32_at(p.kept), f32_at(p.value), reinterpret_cast<float2*>(ws + p.lse)};
      float* peak = f32_at(p.peak);
      uint16_t* masked = s.d_weight ? u16_at(p.masked_hidden) : nullptr;
      const int64_t masked_plane = p.piece * p.width_k, grad_plane = p.piece * p.vocab_pitch;
      MUON_HIP(launch_score_peak(t, d, n, s.vocab, peak, stream));
      MUON_HIP(launch_score_prepare(t, scale.inv_tau, scale.unit, d, peak, rows, n, s.vocab, c, masked, p.width_k, masked_plane, stream));
      if (kept) {
        MUON_HIP(launch_score_dz(t, scale.unit, kept_from(s, p, const_cast<void*>(kept), t0), p.blocks, c, n, s.vocab, s.f32, u16_at(p.grad), p.vocab_pitch,
                                 grad_plane, stream));
      } else {
        HeadOperand hidden;
        if (int st = pack_rows(h, s, p, rows.hidden, n, p.piece, ws + p.packed_hidden, &hidden, stream)) return st;
        MUON_HIP(launch_score_grad(weight, hidden, p.logits[last], p.pairs, scale.unit, t, c, s.f32, u16_at(p.grad), p.vocab_pitch, grad_plane, stream));
      }
      if (s.d_hidden) {
        const HeadOut o{static_cast<unsigned char*>(d_hidden) + size * t0 * s.width, s.f32, f32_at(p.partial), nullptr, 0, 0, scale.inv_tau, peak};
        const HeadOperand l{weight.p, weight.ld, weight.plane, s.width}, r{u16_at(p.grad), p.vocab_pitch, grad_plane, n};
        const HeadProduct& g = p.hidden[last];
        MUON_HIP(launch_head_product(l, r, 0, g, p.pairs, o, stream));
        if (g.splits > 1) MUON_HIP(launch_head_sum_splits(o, g.splits, n * s.width, stream));
      }
      if (s.d_weight) {
        const HeadOut o{d_weight, s.f32, f32_at(p.partial), f32_at(p.sum), piece > 0, !last, scale.inv_tau, peak};
        const HeadOperand l{masked, p.width_k, masked_plane, s.width}, r{u16_at(p.grad), p.vocab_pitch, grad_plane, s.vocab};
        const HeadProduct& g = p.weight[last];
        MUON_HIP(launch_head_product(l, r, 1, g, p.pairs, o, stream));
        if (g.splits > 1) MUON_HIP(launch_head_sum_splits(o, g.splits, s.vocab * s.width, stream));
      }
    }
    return MUON_OK;
  });
}

}  // extern "C"
