// Launch interface of the attention over a paged cache (paged_attn.cu).
#pragma once

#include "common.cuh"

namespace starkv {

constexpr int kMaxDraft = 64;        // drafted tokens of a tree (bits of a mask word)
constexpr int kPagedRows = 128;      // query rows of a block: (token, head of the group) pairs
constexpr int kPagedUnitKeys = 64;   // keys per pipeline unit
constexpr int kPagedItems = 1024;    // query blocks of a launch, at most

// The (query block, group) that a CTA's range begins and does not finish: the ranges up to
// `last` hold the rest of it.
struct PagedSplit {
  int64_t total;   // units of the launch
  int valid, gang; // CTAs of a gang (1: none): range c is that of CTAs c * gang ..
  int seq, row0, nrows, g, last, pad_;
};

struct PagedAttnParams {
  CUtensorMap tmk, tmv;     // the layer's pages: dims (d, P, G, n_pages), box (64, min(P, 64), 1, 1), 128B swizzle
  const __nv_bfloat16* k;
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
  const int32_t* rows;      // [n], or NULL = row0, row0 + 1, ...
  const int32_t* n_tokens;  // [n], or NULL
  int row0, n, T;
  int64_t q_seq, q_token, q_head, o_seq, o_token, o_head;
  int H, G, hg;             // hg = H / G
  int nblk;                 // query blocks of a sequence
  uint32_t inv_hg, inv_nblk;   // ceil(2^32 / n), 0 for n = 1
  int tree;                 // 1: mask, 0: n_sink and window
  int n_sink, window;
  float scale2;             // log2(e) / sqrt(d)
  int grid;                 // CTAs of the main kernel
  PagedSplit* split;        // [grid]
  float2* part_ml;          // [2 * grid][128] reference and sum of a part
  float* part_o;            // [2 * grid][128][128] unnormalised output of a part
  uint32_t* err;
  uint64_t wait_ns;
};

cudaError_t paged_attn_configure();
cudaError_t paged_attn_launch(const PagedAttnParams& p, cudaStream_t stream);
cudaError_t paged_combine_launch(const PagedAttnParams& p, cudaStream_t stream);

}  // namespace starkv
