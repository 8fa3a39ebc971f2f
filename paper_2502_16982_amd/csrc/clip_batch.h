// How the gradients' list is cut into launches: plain C++, no HIP include, so that the tests build it with the host compiler alone.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "../../include/muon.h"

namespace muon {

constexpr int kGradSlots = 192;                  // tensors (or pieces of one) per launch: 3.9 KB of kernel arguments
constexpr int kGradSpan = 16384;                 // elements per block of 256 threads
constexpr int64_t kGradMaxBlocks = (int64_t{1} << 24) - 1;     // a launch holds less than 2^32 work-items
constexpr int64_t kGradMaxNumel = int64_t{1} << 42;            // per tensor
constexpr uint64_t kGradIsF32 = uint64_t{1} << 63;

// Travels by value in the kernel arguments.
struct GradBatch {
  void* g[kGradSlots];
  uint64_t size[kGradSlots];                     // elements; kGradIsF32 for fp32 ones
  int block_start[kGradSlots + 1];               // first block of each tensor; [n] = total blocks
  int n;
};
static_assert(sizeof(GradBatch) <= 3968, "kernel arguments");

// Tensors before `tensor` and the first `element` elements of that one are in earlier launches.
struct GradCursor {
  int32_t tensor = 0;
  int64_t element = 0;                           // a multiple of kGradSpan
};

inline int64_t grad_blocks(int64_t numel) { return (numel + kGradSpan - 1) / kGradSpan; }

// Fills `b` with the next launch's pieces and moves the cursor behind them.  Returns the launch's blocks (0: list done).
inline int grad_next_batch(const muon_grad* grads, int32_t n, GradCursor& at, GradBatch& b) {
  int64_t blocks = 0;
  b.n = 0;
  while (at.tensor < n && b.n < kGradSlots && blocks < kGradMaxBlocks) {
    const muon_grad& q = grads[at.tensor];
    const int64_t e = at.element, len = std::min<int64_t>(q.numel - e, (kGradMaxBlocks - blocks) * kGradSpan);
    if (len > 0) {
      const int k = b.n++;
      b.g[k] = static_cast<char*>(q.g) + e * (q.dtype == MUON_BF16 ? 2 : 4);
      b.size[k] = (uint64_t)len | (q.dtype == MUON_F32 ? kGradIsF32 : 0);
      b.block_start[k] = (int)blocks;
      blocks += grad_blocks(len);
    }
    if (e + len == q.numel) {
      ++at.tensor;
      at.element = 0;
    } else {
      at.element = e + len;
    }
  }
  b.block_start[b.n] = (int)blocks;
  return (int)blocks;
}

// One partial sum per block; more than kGradJoin of them are joined in groups of so many first, whose sums follow behind.  (A launch of 5 us; one
// block sums 12 000 of them in as many, 32 768 in 9.)
constexpr int64_t kGradJoin = 32768;
inline int64_t grad_partials(const muon_grad* grads, int32_t n) {
  int64_t blocks = 0;
  for (int32_t i = 0; i < n; ++i) blocks += grad_blocks(grads[i].numel);
  return blocks;
}
inline size_t grad_workspace(int64_t partials) {
  const int64_t groups = partials > kGradJoin ? (partials + kGradJoin - 1) / kGradJoin : 0;
  return std::max<size_t>(256, ((size_t)(partials + groups) * 8 + 255) / 256 * 256);
}

}  // namespace muon
