// Host-callable launchers of the experts' sort, dispatch and combine (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace muon {

constexpr int kMaxExperts = 4096, kMaxExpertTop = 64;
constexpr int64_t kMaxExpertPairs = (1ll << 31) - (1 << 16);      // positions are 32-bit, and so is the last block's end
// Pairs per block of the sort, a multiple of 256 (its four waves take whole 64s): one block for few, otherwise 512 and never more than kSortBlocks
// blocks.  One block is a launch less, but takes the pairs one wave's 64 after the other: 64 experts, 512 pairs 3.7 us, 1024 5.5 against 6.5
// in two launches, 2048 9.0 against 6.5.  Blocks of 256 pairs are quicker for 16384 pairs of 64 experts (6.2 against 6.9) and slower for
// 49152 of 512 (27 against 19), blocks of 1024 the other way round (9.4; 16.5).
constexpr int kSortAlone = 1024, kSortChunk = 512, kSortBlocks = 256;
inline int64_t sort_chunk(int64_t pairs) {
  if (pairs <= kSortAlone) return pairs <= 256 ? 256 : (pairs + 255) / 256 * 256;
  const int64_t even = (pairs + kSortBlocks - 1) / kSortBlocks;
  return even <= kSortChunk ? kSortChunk : (even + 255) / 256 * 256;
}
inline int sort_blocks(int64_t pairs) { return pairs <= kSortAlone ? 1 : (int)((pairs + sort_chunk(pairs) - 1) / sort_chunk(pairs)); }

hipError_t launch_expert_sort(const void* expert, int index64, int64_t pairs, int experts, int* position, int* source, int* offsets,
                              int* counts, hipStream_t s);
// The tokens' way to their rows and back.  `count`: device address of the number of rows that belong to a pair.
struct ExpertRows {
  const int* position;      // [tokens, top]
  const int* count;
  long long tokens, width;
  int top;
  int f32;
};
hipError_t launch_expert_dispatch(const ExpertRows& r, const void* x, long long x_stride, void* rows, hipStream_t s);
hipError_t launch_expert_combine(const ExpertRows& r, const void* rows, const float* weights, void* out, hipStream_t s);
hipError_t launch_expert_combine_backward(const ExpertRows& r, const void* d_out, long long d_out_stride, const void* rows,
                                          const float* weights, void* d_rows, float* d_weights, hipStream_t s);

}  // namespace muon
