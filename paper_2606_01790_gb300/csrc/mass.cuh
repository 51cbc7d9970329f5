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

constexpr int kMassTile = 128;   // keys of a tile, (token, head) pairs of a query block at most
constexpr int kMassSpan = 4;     // tiles of a group, at most
constexpr int kMassQueryStep = 8;   // rows of a query block that are copied at a time

// The group that a CTA's range begins and does not finish: the ranges up to `last` hold the rest.  `failed`: a wait of this
// CTA ran out, or it was held back, and its parts may not be there.
struct MassSplit {
  int valid, seq, g, k0, keys, last, failed, pad_;
};

struct MassParams {
  CUtensorMap tmk;          // the layer's pages: dims (d, P, G, n_pages), box (64, min(P, 64), 1, 1), 128B swizzle
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
  int tpb, heads, chunks;   // tokens and heads of a block; blocks that the heads of a group take
  int cut;                  // 1: a group's blocks may be cut between ranges (more than stay in shared memory)
  uint32_t inv_tpb, inv_heads, inv_chunks;   // ceil(2^32 / n), 0 for n = 1
  int64_t step, wrap;       // elements from a block's pair to the one kMassQueryStep on; more where that passes `heads` heads
  int step_h;               // kMassQueryStep mod heads
  int64_t span_from;        // tiles of a launch from which groups have kMassSpan of them (else 1)
  int tree;                 // 1: mask, 0: n_sink and window
  int n_sink, window;
  float scale2;             // log2(e) / sqrt(d)
  MassView mass;
  float decay;
  int grid;                 // CTAs of the main kernel
  MassSplit* split;         // [grid]
  float* part;              // [2 * grid][span * 128]
  uint32_t* err;
  uint64_t wait_ns;
};

cudaError_t mass_configure();
cudaError_t mass_launch(const MassParams& p, cudaStream_t stream);
// The parts of the groups that were cut: with p.cut only.
cudaError_t mass_sum_launch(const MassParams& p, cudaStream_t stream);

cudaError_t mass_select_configure();
// Picks the tokens of an eviction whose bookkeeping (`plan`) was carried out, and moves their mass.
cudaError_t mass_select_launch(const PagesView& pg, const SeqBatch& b, const int32_t* rows, int row0, int w, int per_head,
                               const PagePlan* plan, const MassView& mass, cudaStream_t stream);

}  // namespace starkv
