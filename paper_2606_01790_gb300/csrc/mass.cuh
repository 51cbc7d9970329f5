// Launch interface of the attention mass and the eviction by it (mass.cu).
#pragma once

#include "common.cuh"
#include "pages.cuh"

namespace starkv {

// Mass of one layer (starkv_mass): token j of row r, KV head g at m + r row_stride + g group_stride + j.
struct MassView {
  float* m;
  int64_t layer_stride, row_stride, group_stride;   // elements
};

struct MassParams {
  const __nv_bfloat16* k;   // of the layer
  int64_t page_stride;      // elements
  const int32_t* table;
  const int32_t* len;
  int n_pages, n_rows, max_pages, shift;
  // queries (starkv_queries); strides in elements
  const __nv_bfloat16* q;
  const float* lse;         // [n][T][H]
  const uint64_t* mask;     // tree: [n][T]
  const int32_t* rows;      // [n], or NULL = 0, 1, ...
  const int32_t* n_tokens;  // [n], or NULL
  int n, T;
  int64_t q_seq, q_token, q_head;
  int H, G, hg;             // hg = H / G
  int tree;                 // 1: mask, 0: n_sink and window
  int n_sink, window;
  float scale2;             // log2(e) / sqrt(d)
  MassView mass;
  float decay;
  uint32_t* err;
};

cudaError_t mass_launch(const MassParams& p, int num_sms, cudaStream_t stream);

// Picks the tokens of an eviction whose bookkeeping (`plan`) was carried out, and moves their mass.
cudaError_t mass_select_launch(const PagesView& pg, const SeqBatch& b, const int32_t* rows, int row0, int w, int per_head,
                               const PagePlan* plan, const MassView& mass, cudaStream_t stream);

}  // namespace starkv
