// Bounds of the keys of a page, and the pages that a query takes by them.
//
// Bounds: per layer, page, KV head g and channel c, over the slots that hold tokens,
//   lo_c = min K_c,  hi_c = max K_c.
// Score of a page for a query (the heads h of group g together): the most that its keys'
// logits can come to,
//   s = sum_h sum_c max(q_hc lo_c, q_hc hi_c) = sum_c up_c hi_c + down_c lo_c,
//   up_c = sum_h max(q_hc, 0),  down_c = sum_h min(q_hc, 0),
// so that the heads of a group cost one product of 256 terms a page.  A query takes the
// first pages, the last ones up to its own and the best of the others; equal scores go to
// the lower page.  Which of two pages is taken hangs on the last bit of their scores: the
// products of two bf16 numbers and their sums are formed in 64 bits.
#include <algorithm>

#include "common.cuh"
#include "ptx.cuh"
#include "sparse.cuh"

namespace starkv {

namespace {

constexpr uint32_t kFull = 0xffffffffu;

cudaLaunchConfig_t config(cudaLaunchAttribute* attr, dim3 grid, int threads, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // starts under the previous kernel's tail
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

// ---------------------------------------------------------------- bounds

constexpr int kBoundsThreads = 256;
constexpr int kBoundsWarps = kBoundsThreads / 32;
constexpr int kInFlight = 4;

struct Pair8 {   // eight channels
  __nv_bfloat162 v[4];
};

__device__ __forceinline__ Pair8 as_pairs(const uint4& x) {
  Pair8 p;
  *reinterpret_cast<uint4*>(&p) = x;
  return p;
}

}  // namespace

// Warp tasks: (sequence, layer, page, KV head); half a warp a slot, 16 bytes a lane.  A NaN
// among the keys is a NaN in both bounds.
__global__ void __launch_bounds__(kBoundsThreads) k_page_bounds(const __grid_constant__ BoundsParams p) {
  griddep_launch_dependents();
  griddep_wait();
  const PagesView& pg = p.pg;
  const int lane = threadIdx.x & 31, half = lane >> 4, hl = lane & 15;
  const int P = 1 << pg.shift;
  const int most = ((p.T + P - 2) >> pg.shift) + 1;   // pages that T tokens may lie in
  const int64_t per_seq = static_cast<int64_t>(most) * p.nlayers * pg.G, ntask = per_seq * p.n;
  for (int64_t task = static_cast<int64_t>(blockIdx.x) * kBoundsWarps + (threadIdx.x >> 5); task < ntask;
       task += static_cast<int64_t>(gridDim.x) * kBoundsWarps) {
    const int seq = static_cast<int>(task / per_seq);
    int rem = static_cast<int>(task - seq * per_seq);
    const int g = rem % pg.G;
    rem /= pg.G;
    const int j = rem % most, l = rem / most;
    const int row = p.rows ? p.rows[seq] : seq;
    const int count = p.n_tokens ? p.n_tokens[seq] : p.T;
    const int L = row >= 0 && row < pg.n_rows ? pg.len[row] : -1;
    if (count < 0 || count > p.T || L < count || L > static_cast<int64_t>(pg.max_pages) << pg.shift) {
      if (lane == 0) atomicOr(p.err, kErrRow);
      continue;
    }
    const int at = ((L - count) >> pg.shift) + j;   // the page's place in the row
    const int fill = min(P, L - (at << pg.shift));
    if (count == 0 || fill <= 0) continue;
    const int page = pg.table[static_cast<int64_t>(row) * pg.max_pages + at];
    if (page < 0 || page >= pg.n_pages) {
      if (lane == 0) atomicOr(p.err, kErrRow);
      continue;
    }
    const uint4* k = reinterpret_cast<const uint4*>(pg.k + (p.layer0 + l) * pg.layer_stride + page * pg.page_stride +
                                                    (static_cast<int64_t>(g) << pg.shift) * kHeadDim);
    const __nv_bfloat162 inf = __float2bfloat162_rn(INFINITY), ninf = __float2bfloat162_rn(-INFINITY);
    Pair8 lo, hi;
#pragma unroll
    for (int c = 0; c < 4; ++c) lo.v[c] = inf, hi.v[c] = ninf;
    for (int s0 = 0; s0 < fill; s0 += 2 * kInFlight) {
      uint4 x[kInFlight];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {   // (behind the last slot: the last one again)
        const int s = min(s0 + 2 * u + half, fill - 1);
        x[u] = ld_stream(k + s * (kHeadDim / 8) + hl);
      }
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const Pair8 y = as_pairs(x[u]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          lo.v[c] = __hmin2_nan(lo.v[c], y.v[c]);
          hi.v[c] = __hmax2_nan(hi.v[c], y.v[c]);
        }
      }
    }
    // the halves' bounds: the lower lanes write the least keys, the upper ones the greatest
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      lo.v[c] = __hmin2_nan(lo.v[c], __shfl_xor_sync(kFull, lo.v[c], 16));
      hi.v[c] = __hmax2_nan(hi.v[c], __shfl_xor_sync(kFull, hi.v[c], 16));
    }
    uint4* out = reinterpret_cast<uint4*>(p.out.b + (p.layer0 + l) * p.out.layer_stride + page * p.out.page_stride +
                                          static_cast<int64_t>(g) * 2 * kHeadDim);
    out[lane] = *reinterpret_cast<const uint4*>(half ? &hi : &lo);
  }
}

cudaError_t page_bounds_launch(const BoundsParams& p, int num_sms, cudaStream_t stream) {
  const int P = 1 << p.pg.shift;
  const int64_t tasks = static_cast<int64_t>(((p.T + P - 2) >> p.pg.shift) + 1) * p.nlayers * p.pg.G * p.n;
  if (tasks <= 0) return cudaSuccess;
  const int64_t blocks = (tasks + kBoundsWarps - 1) / kBoundsWarps;
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(static_cast<unsigned>(std::min<int64_t>(blocks, int64_t(1) << 30))), kBoundsThreads, stream);
  return cudaLaunchKernelEx(&cfg, k_page_bounds, p);
}

// ---------------------------------------------------------------- choice

namespace {

constexpr int kChooseThreads = 256;
constexpr int kChooseWarps = kChooseThreads / 32;

// Ascending order of the scores; a NaN (a bound that is none) comes with the greatest, so that
// its page is not passed over.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) s = INFINITY;
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(s + 0.0));   // (-0 is 0)
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

// Sum over the block of 0 / 1 flags in front of this thread's, and all of them.
__device__ int2 count_before(bool flag, int* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t m = __ballot_sync(kFull, flag);
  if (lane == 0) warp_sum[warp] = __popc(m);
  __syncthreads();
  int before = __popc(m & ((1u << lane) - 1)), all = 0;
#pragma unroll
  for (int w = 0; w < kChooseWarps; ++w) {
    if (w < warp) before += warp_sum[w];
    all += warp_sum[w];
  }
  __syncthreads();
  return make_int2(before, all);
}

}  // namespace

// Block (item, KV head): scores, the threshold by eight bits at a time, the list in order.
__global__ void __launch_bounds__(kChooseThreads) k_page_choose(const __grid_constant__ ChooseParams p) {
  __shared__ double s_up[kHeadDim], s_down[kHeadDim];
  __shared__ int hist[256], warp_sum[kChooseWarps];
  __shared__ uint64_t s_prefix;
  __shared__ int s_need;
  griddep_launch_dependents();
  griddep_wait();
  const PagesView& pg = p.pg;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int item = blockIdx.x, g = blockIdx.y, v = p.item0 + item;
  const SparseQuery sq = sparse_query(p.rows, p.n_tokens, pg.len, pg.n_rows, pg.max_pages, pg.shift, p.T, v);
  if (!sq.live) return;
  int32_t* list = p.list + (static_cast<int64_t>(item) * p.G + g) * p.n_list;
  int32_t* chosen = p.chosen ? p.chosen + (static_cast<int64_t>(v) * p.G + g) * p.n_chosen : nullptr;
  const int pages = sq.pos < 0 ? 0 : (sq.pos >> pg.shift) + 1;
  const int take = min(pages, p.n_list);
  const int32_t* entries = pg.table + static_cast<int64_t>(sq.row) * pg.max_pages;
  if (chosen)
    for (int i = take + tid; i < p.n_chosen; i += kChooseThreads) chosen[i] = -1;
  // pages lo .. hi - 1 compete for `need` places; the others are taken anyway
  const int lo = take == pages ? pages : p.n_first, hi = take == pages ? pages : pages - p.n_last;
  int need = take - (pages - (hi - lo));
  uint64_t* keys = p.keys + (static_cast<int64_t>(item) * p.G + g) * pg.max_pages;
  uint64_t least = 0;   // pages with greater keys are taken, and `need` of those that have this one
  if (need > 0) {
    const int seq = v / p.T, t = v - seq * p.T;
    if (tid < kHeadDim) {
      const __nv_bfloat16* q = p.q + seq * p.q_seq + t * p.q_token + static_cast<int64_t>(g) * p.hg * p.q_head + tid;
      double up = 0, down = 0;
      for (int h = 0; h < p.hg; ++h) {
        const double x = __bfloat162float(q[h * p.q_head]);
        up += x < 0 ? 0 : x;   // (a NaN goes into both)
        down += x > 0 ? 0 : x;
      }
      s_up[tid] = up;
      s_down[tid] = down;
    }
    __syncthreads();
    for (int j = lo + warp; j < hi; j += kChooseWarps) {
      const int page = entries[j];
      double s = 0;
      if (page >= 0 && page < pg.n_pages) {
        const __nv_bfloat16* b = p.bounds + page * p.bounds_page + static_cast<int64_t>(g) * 2 * kHeadDim;
#pragma unroll
        for (int c = lane; c < kHeadDim; c += 32)
          s += s_down[c] * static_cast<double>(__bfloat162float(b[c])) + s_up[c] * static_cast<double>(__bfloat162float(b[kHeadDim + c]));
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
      if (lane == 0) keys[j] = score_key(s);
    }
    if (tid == 0) s_prefix = 0, s_need = need;
    __syncthreads();
    for (int bit = 56; bit >= 0; bit -= 8) {
      hist[tid] = 0;
      __syncthreads();
      const uint64_t prefix = s_prefix;
      for (int j = lo + tid; j < hi; j += kChooseThreads)
        if (bit == 56 || (keys[j] ^ prefix) >> (bit + 8) == 0) atomicAdd(&hist[keys[j] >> bit & 255], 1);
      __syncthreads();
      if (tid == 0) {
        int left = s_need, d = 255;
        while (d > 0 && hist[d] < left) left -= hist[d--];
        s_prefix = prefix | static_cast<uint64_t>(d) << bit;
        s_need = left;
      }
      __syncthreads();
    }
    least = s_prefix;
    need = s_need;
  }
  int at = 0, equal = 0;   // taken so far, and of those that have the least key
  for (int j0 = 0; j0 < pages; j0 += kChooseThreads) {
    const int j = j0 + tid;
    const bool rival = j >= lo && j < hi;
    const uint64_t key = rival && need > 0 ? keys[j] : 0;
    const int2 e = count_before(rival && need > 0 && key == least, warp_sum);
    const bool in = j < pages && (!rival || (need > 0 && (key > least || (key == least && equal + e.x < need))));
    const int2 n = count_before(in, warp_sum);
    if (in) {
      list[at + n.x] = entries[j];
      if (chosen) chosen[at + n.x] = j;
    }
    equal += e.y;
    at += n.y;
  }
}

cudaError_t page_choose_launch(const ChooseParams& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.items, p.G), kChooseThreads, stream);
  return cudaLaunchKernelEx(&cfg, k_page_choose, p);
}

}  // namespace starkv
