// Tasks of the page bounds (sparse.cu), one a warp: sequence, layer, place of the page among those that the call may look
// at, KV head.  Plain C++, so that the split is checked at its limits without a GPU.
#pragma once

#include <cstdint>

namespace starkv {

// Pages that `tokens` tokens at the end of a row may lie in: as many as they can spread over, and no more than a row has.
__host__ __device__ __forceinline__ int bounds_pages(int tokens, int shift, int max_pages) {
  const int spread = ((tokens + (1 << shift) - 2) >> shift) + 1;
  return spread < max_pages ? spread : max_pages;
}

struct BoundsTask {
  int seq, layer, page, g;
  // (The tasks of one sequence pass 31 bits: 2^20 pages, 64 layers and 32 KV heads are 2^31.)
  __host__ __device__ __forceinline__ BoundsTask(int64_t task, int pages, int layers, int G) {
    const int64_t each = static_cast<int64_t>(pages) * layers * G;
    seq = static_cast<int>(task / each);
    int64_t rem = task - seq * each;
    g = static_cast<int>(rem % G);
    rem /= G;
    page = static_cast<int>(rem % pages);
    layer = static_cast<int>(rem / pages);
  }
};

}  // namespace starkv
