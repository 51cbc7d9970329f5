// Launch interface of the paged cache's kernels (pages.cu).
#pragma once

#include "common.cuh"

namespace starkv {

constexpr int kMaxPages = 1 << 20;       // pages of a pool (the free-page bits of a cluster CTA: 16 KB)
constexpr int kMaxTableRows = 1 << 16;   // rows of a page table
constexpr int kMaxCallRows = 1024;       // rows of one call (one per thread of a bookkeeping block)

// The pool and its table as the kernels see them (starkv_pages).
struct PagesView {
  __nv_bfloat16* k;
  __nv_bfloat16* v;
  int64_t layer_stride, page_stride;   // elements
  int32_t* table;   // [n_rows][max_pages]
  int32_t* len;     // [n_rows]
  int32_t* refs;    // [n_pages]
  int n_pages, n_rows, max_pages;
  int shift;        // log2 of the tokens of a page
  int n_layers, G;
};

// Workspace of a bookkeeping call: what the copy and gather kernels after it do.
struct PagePlan {
  int32_t ok;         // 1: the call was carried out
  int32_t n_copies;   // entries of the copy list
  int32_t pad_[2];
};

enum BookOp : int { kBookExtend, kBookFork, kBookForkDeep, kBookFree, kBookCompact };

struct BookParams {
  PagesView pg;
  const int32_t* rows;    // [n] (fork: the new rows), or NULL = 0, 1, ...
  const int32_t* src;     // fork: [n], or NULL
  const int32_t* n_new;   // extend: [n]
  int n;
  PagePlan* plan;
  int4* copies;           // (from, to, tokens, 0): extend [n], deep fork [n * max_pages]
  int32_t* old_table;     // compact: [n][max_pages], the rows' pages before the call
  uint32_t* err;
};

// Compaction only: each row's tokens before and after.
struct BookLens {
  int32_t L[kMaxCallRows], kept[kMaxCallRows];
};

cudaError_t pages_configure();
// `lens`: with kBookCompact.
cudaError_t book_launch(BookOp op, const BookParams& p, const BookLens* lens, cudaStream_t stream);
// Copies the plan's pages in every layer; at most max_copies entries.
cudaError_t page_copy_launch(const PagesView& pg, const PagePlan* plan, const int4* copies, int64_t max_copies,
                             int num_sms, cudaStream_t stream);
// The gather of a compaction: rows of old_table to the pages that the table names now,
// for the call's sequences row0, row0 + 1, ... of the batch.
cudaError_t page_gather_launch(const PagesView& pg, const SeqBatch& b, const int32_t* rows, int row0, int w, int per_head,
                               const PagePlan* plan, const int32_t* old_table, int rows_out_max, uint32_t* err,
                               cudaStream_t stream);

// Tokens outside the pages (starkv_tokens); strides in elements.
struct TokensView {
  __nv_bfloat16* k;
  __nv_bfloat16* v;   // NULL: keys only
  const int32_t* rows;
  const int32_t* n_tokens;
  int n, T, layer0, nlayers;
  int64_t seq_stride, layer_stride, token_stride, head_stride;
};

cudaError_t page_move_launch(bool store, const PagesView& pg, const TokensView& t, uint32_t* err, cudaStream_t stream);

}  // namespace starkv
