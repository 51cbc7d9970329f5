// Launch interface of the page bounds and of the choice of pages (sparse.cu).
#pragma once

#include "common.cuh"
#include "pages.cuh"

namespace starkv {

// Bounds of pages (starkv_bounds), one layer: [page][G][2][d].
struct BoundsView {
  __nv_bfloat16* b;
  int64_t layer_stride, page_stride;   // elements
};

// The pages that hold the last n_tokens tokens of the call's rows.
struct BoundsParams {
  PagesView pg;
  BoundsView out;
  const int32_t* rows;
  const int32_t* n_tokens;
  int n, T, layer0, nlayers;
  uint32_t* err;
};

cudaError_t page_bounds_launch(const BoundsParams& p, cudaStream_t stream);

// Query v of a call's n * T: its position in its row.
struct SparseQuery {
  int row;
  int pos;      // -1: the row does not fit the call, nothing is seen
  bool live;    // one of the sequence's n_tokens
  bool wrong;   // to be reported
};

__device__ __forceinline__ SparseQuery sparse_query(const int32_t* rows, const int32_t* n_tokens, const int32_t* len, int n_rows,
                                                    int max_pages, int shift, int T, int v) {
  SparseQuery q;
  const int seq = v / T, t = v - seq * T;
  q.row = rows ? rows[seq] : seq;
  const int n = n_tokens ? n_tokens[seq] : T;
  const int L = q.row >= 0 && q.row < n_rows ? len[q.row] : -1;
  const bool counted = n >= 0 && n <= T;
  const bool fits = L >= n && L <= static_cast<int64_t>(max_pages) << shift;
  q.live = counted && t < n;
  q.pos = fits ? L - n + t : -1;
  q.wrong = !counted || (n > 0 && !fits);
  return q;
}

struct ChooseParams {
  PagesView pg;
  const __nv_bfloat16* bounds;   // of the layer
  int64_t bounds_page;           // elements
  const __nv_bfloat16* q;        // bf16, strides in elements
  int64_t q_seq, q_token, q_head;
  const int32_t* rows;
  const int32_t* n_tokens;
  int T, item0, items;           // queries item0 .. item0 + items - 1 of the call's n * T
  int G, hg;
  int n_first, n_last, n_list;   // n_list: pages taken, at most max_pages
  int32_t* list;                 // [items][G][n_list] page numbers
  int2* tokens;                  // [items] tokens that the chosen pages hold up to the query (-1: the row does not fit), 1 for a query
  uint32_t* err;
  int32_t* chosen;               // [n * T][G][n_chosen] places in the row, or NULL
  int n_chosen;
  int ctas;                      // of a cluster: 1, 2, 4 or 8
  uint64_t* keys;                // [items][G][max_pages]: scores in 64 bits, where many are close
  uint32_t* scores;              // the same, in 32: rows of more than kChoosePages pages
};

constexpr int kChoosePages = 8192;   // scores that shared memory holds

cudaError_t page_choose_configure();
cudaError_t page_choose_launch(const ChooseParams& p, cudaStream_t stream);

}  // namespace starkv
