// Index arithmetic of the cache's kernels in plain constant functions, so that
// the host can check it for every page and head size that is taken.
#pragma once

namespace palq {

constexpr int kPages[] = {16, 32, 64, 128};   // tokens of a page
constexpr int kDims[] = {64, 96, 128, 256};   // channels of a head

// cache_append_kernel: a block goes by items of 4 tokens x 8 channels, one for a
// thread at a time, and a thread holds all of its items at once (1, 2 or 4).
constexpr int kAppendThreads = 256;
constexpr int append_items(int page, int dim) { return page / 4 * (dim / 8); }
constexpr int append_rounds(int page, int dim) {
  const int n = (append_items(page, dim) + kAppendThreads - 1) / kAppendThreads;
  return n <= 2 ? n : 4;
}
// Values turned in LDS: page / 4 words a channel, and one that keeps banks apart.
constexpr int turned_stride(int page) { return page / 4 + 1; }
constexpr int turned_words(int rounds) { return rounds * kAppendThreads * 8 + 256; }

constexpr bool append_holds_every_block() {
  for (const int page : kPages)
    for (const int dim : kDims) {
      const int n = append_rounds(page, dim);
      if (n > 4 || append_items(page, dim) > n * kAppendThreads || dim * turned_stride(page) > turned_words(n)) return false;
    }
  return true;
}
static_assert(append_holds_every_block(), "a block that the append's threads or LDS do not hold");

}  // namespace palq
