// Walks the launches that lists of gradients are cut into and checks that each element is covered once.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2502_16982_amd/csrc/clip_batch.h"

using namespace muon;

#define CHECK(x)                                              \
  do {                                                        \
    if (!(x)) {                                               \
      std::printf("line %d: %s\n", __LINE__, #x);             \
      std::exit(1);                                           \
    }                                                         \
  } while (0)

static void walk(const std::vector<int64_t>& sizes, uint64_t seed) {
  std::mt19937_64 rng(seed);
  std::vector<muon_grad> list(sizes.size());
  for (size_t i = 0; i < sizes.size(); ++i)
    list[i] = {reinterpret_cast<void*>((uintptr_t{1} << 50) * (i % 7 + 1)), sizes[i], rng() % 2 ? MUON_BF16 : MUON_F32, 0};
  GradBatch b{};
  GradCursor at;
  size_t tensor = 0;
  int64_t element = 0, blocks = 0;
  auto skip_empty = [&] {
    while (tensor < list.size() && list[tensor].numel == element) ++tensor, element = 0;
  };
  skip_empty();
  while (const int n = grad_next_batch(list.data(), (int32_t)list.size(), at, b)) {
    CHECK(b.n >= 1 && b.n <= kGradSlots && n <= kGradMaxBlocks && b.block_start[0] == 0 && b.block_start[b.n] == n);
    for (int k = 0; k < b.n; ++k) {
      const int64_t len = (int64_t)(b.size[k] & ~kGradIsF32);
      CHECK(tensor < list.size() && len >= 1 && element % kGradSpan == 0);
      const muon_grad& q = list[tensor];
      CHECK(((b.size[k] & kGradIsF32) != 0) == (q.dtype == MUON_F32));
      CHECK(b.g[k] == static_cast<char*>(q.g) + element * (q.dtype == MUON_F32 ? 4 : 2));
      CHECK(b.block_start[k + 1] - b.block_start[k] == grad_blocks(len));
      element += len;
      CHECK(element <= q.numel);
      skip_empty();
    }
    blocks += n;
  }
  CHECK(tensor == list.size());
  CHECK(blocks == grad_partials(list.data(), (int32_t)list.size()));
  const int64_t groups = blocks > kGradJoin ? (blocks + kGradJoin - 1) / kGradJoin : 0;
  CHECK(grad_workspace(blocks) >= (size_t)(blocks + groups) * 8);
}

int main() {
  walk({}, 1);
  walk({0}, 2);
  walk({0, 0, 1, 0}, 3);
  walk({kGradSpan - 1, kGradSpan, kGradSpan + 1}, 4);
  walk(std::vector<int64_t>(1000, 5), 5);
  walk(std::vector<int64_t>(kGradSlots, 1), 6);
  walk({kGradMaxNumel, 3, kGradMaxNumel}, 7);
  walk({kGradMaxBlocks * kGradSpan, 1}, 8);
  walk({kGradMaxBlocks * kGradSpan + 1, 1, 0}, 9);
  std::mt19937_64 rng(10);
  for (int i = 0; i < 200; ++i) {
    std::vector<int64_t> sizes(rng() % 600);
    for (auto& s : sizes) s = (int64_t)(rng() % (uint64_t{1} << (rng() % 32)));
    walk(sizes, 100 + i);
  }
  std::printf("ok\n");
}
