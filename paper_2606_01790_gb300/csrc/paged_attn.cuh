// Launch interface of the attention over a paged cache (paged_attn.cu).
#pragma once

#include "common.cuh"

namespace starkv {

constexpr int kMaxDraft = 64;   // drafted tokens of a tree (bits of a mask word)

struct PagedAttnParams {
  const __nv_bfloat16* k;   // the layer's pages
  const __nv_bfloat16* v;
  int64_t page_stride;      // elements
  const int32_t* table;
  const int32_t* len;
  int n_pages, n_rows, max_pages, shift;
  // queries (starkv_queries); strides in elements
  const __nv_bfloat16* q;
  __nv_bfloat16* o;
  float* lse;               // [n][T][H], or NULL
  const uint64_t* mask;     // tree: [n][T]
  const int32_t* rows;      // [n], or NULL
  const int32_t* n_tokens;  // [n], or NULL
  int n, T;
  int64_t q_seq, q_token, q_head, o_seq, o_token, o_head;
  int H, G;
  int tree;                 // 1: mask, 0: n_sink and window
  int n_sink, window;
  float scale2;             // log2(e) / sqrt(d)
  uint32_t* err;
};

cudaError_t paged_attn_launch(const PagedAttnParams& p, int num_sms, cudaStream_t stream);

}  // namespace starkv
