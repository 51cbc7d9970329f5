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
// the lower page.  Which of two pages is taken hangs on the last bit of their scores, which
// are those of 64 bits.
//
// What bounds them.  Bounds: the keys' bytes, read once (28 layers of 14,032 tokens, 415 MB, 66 us: 93 % of the copy rate; one new
// token of 64 rows in 28 layers 15 us, of which the pages' 68 MB 10).  Choice: the bounds' bytes (64 rows of 14k ragged
// tokens in pages of 32: 72 MB of them in 12 us), and behind them a chain of about 10 us (row, length, query, numbers and bounds
// of pages, the border, the list).  Scores in 64 bits throughout took 590 us there.
#include <algorithm>

#include "bounds_task.cuh"
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
  const int most = bounds_pages(p.T, pg.shift, pg.max_pages);
  const int64_t ntask = static_cast<int64_t>(most) * p.nlayers * pg.G * p.n;
  for (int64_t task = static_cast<int64_t>(blockIdx.x) * kBoundsWarps + (threadIdx.x >> 5); task < ntask;
       task += static_cast<int64_t>(gridDim.x) * kBoundsWarps) {
    const BoundsTask of(task, most, p.nlayers, pg.G);
    const int seq = of.seq, g = of.g, l = of.layer;
    const int row = p.rows ? p.rows[seq] : seq;
    const int count = p.n_tokens ? p.n_tokens[seq] : p.T;
    const int L = row >= 0 && row < pg.n_rows ? pg.len[row] : -1;
    if (count < 0 || count > p.T || L < count || L > static_cast<int64_t>(pg.max_pages) << pg.shift) {
      if (lane == 0) atomicOr(p.err, kErrRow);
      continue;
    }
    const int at = ((L - count) >> pg.shift) + of.page;   // the page's place in the row
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

cudaError_t page_bounds_launch(const BoundsParams& p, cudaStream_t stream) {
  const int64_t tasks = static_cast<int64_t>(bounds_pages(p.T, p.pg.shift, p.pg.max_pages)) * p.nlayers * p.pg.G * p.n;
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
constexpr int kPagesAtOnce = 8;        // of a warp
constexpr int kFew = 256;              // close pages that are ranked by comparing each with each
constexpr int kRun = 4;                // competing pages of a thread, at most, where one pass over bins finds the border
constexpr int kBins = 2048;

// Ascending order as unsigned numbers.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
// (A NaN, of a bound that is none, comes with infinity, so that its page is not passed over; -0 is 0.)
__device__ __forceinline__ uint64_t order_of(double x) {
  if (x != x) x = INFINITY;
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

// a + b rounded, with what the rounding left out (Knuth's two-sum) added to *rest
__device__ __forceinline__ float sum_and_rest(float a, float b, float* rest) {
  const float s = a + b, t = s - a;
  *rest += (a - (s - t)) + (b - t);
  return s;
}

struct ChooseSmem {
  uint32_t key[kChoosePages];
  float up[kHeadDim], down[kHeadDim], up_rest[kHeadDim], down_rest[kHeadDim];
  uint32_t size[kMaxCluster][kChooseWarps];   // largest sum of terms' sizes that a warp met
  int hist[256];
  int warp_sum[kChooseWarps];
  uint64_t prefix;
  int need, few;
  uint32_t least, most;
  int bin, bin_sum[2][kChooseWarps];
  int bins[kBins];
  uint64_t close[kFew];
  int close_page[kFew];
};

// Sum over the block of a count per thread, in front of this thread's; the total to everybody.  AGAIN: warp_sum is
// free for another use afterwards.
template <bool AGAIN = true>
__device__ __forceinline__ int block_before(int x, int* warp_sum, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(kFull, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  int before = inc - x, all = 0;
#pragma unroll
  for (int w = 0; w < kChooseWarps; ++w) {
    if (w < warp) before += warp_sum[w];
    all += warp_sum[w];
  }
  if (AGAIN) __syncthreads();
  *total = all;
  return before;
}

// The k-th greatest of key(lo) .. key(hi - 1), eight bits at a time; *of_it: how many of those that have
// it are among the k greatest.
template <typename Key, typename F>
__device__ Key kth_greatest(ChooseSmem& s, int lo, int hi, int k, F key, int* of_it) {
  const int tid = threadIdx.x, lane = tid & 31;
  Key prefix = 0;
  for (int bit = static_cast<int>(sizeof(Key)) * 8 - 8; bit >= 0; bit -= 8) {
    if (tid < 256) s.hist[tid] = 0;
    __syncthreads();
    for (int j0 = lo; j0 < hi; j0 += kChooseThreads) {   // (scores share their first bits: one addition for all of a warp that meet)
      const Key x = j0 + tid < hi ? key(j0 + tid) : 0;
      const bool counts = j0 + tid < hi && (bit == static_cast<int>(sizeof(Key)) * 8 - 8 || (x ^ prefix) >> (bit + 8) == 0);
      const int digit = counts ? static_cast<int>(x >> bit & 255) : -1;
      const uint32_t same = __match_any_sync(kFull, digit);
      if (counts && lane == __ffs(same) - 1) atomicAdd(&s.hist[digit], __popc(same));
    }
    __syncthreads();
    if (tid < 32) {   // lane l: the digits 255 - 8 l downwards
      int sum = 0, n[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += n[i] = s.hist[255 - 8 * lane - i];
      int inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, inc, o);
        if (lane >= o) inc += y;
      }
      int left = k - (inc - sum);
      if (left > 0 && left <= sum) {
        int i = 0;
        while (i < 7 && n[i] < left) left -= n[i++];
        s.prefix = prefix | static_cast<Key>(255 - 8 * lane - i) << bit;
        s.need = left;
      }
    }
    __syncthreads();
    prefix = static_cast<Key>(s.prefix);
    k = s.need;
  }
  *of_it = k;
  return prefix;
}

}  // namespace

static_assert(kChooseThreads >= 256, "a thread a digit and a close page");

// Cluster (item, KV head): its CTAs score a share of the pages each, in fp32, into the first one's shared
// memory (rows of more pages than it holds: into the workspace); the first CTA takes the best.
//
// A lane has 8 of the 256 terms; sums over the lanes are taken for eight pages together, halving the pages with every
// step.  With u = 2^-24 a score is off by at most (8 + 5 + hg) u times the sum of its terms' sizes (the products' sums, the
// sums over lanes, the weights' sums over heads), plus what underflows: at most E, with the lanes' largest sizes added up for
// all pages.  With the k-th greatest score between t0 and t1, a page 2 E above t1 is among the k best and one 2 E below t0 is not; those between are
// scored again in 64 bits where they are more than the places left: usually none or a few, all of them where scores are equal
// or sizes are past what 32 bits hold.
__global__ void __launch_bounds__(kChooseThreads) k_page_choose(const __grid_constant__ ChooseParams p) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  ChooseSmem& s = *reinterpret_cast<ChooseSmem*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x & (p.ctas - 1), g = blockIdx.y, item = blockIdx.x / p.ctas, v = p.item0 + item;
  cluster_arrive();   // waited for before the first write into the first CTA's shared memory
  griddep_launch_dependents();
  griddep_wait();
  const PagesView& pg = p.pg;
  const int seq = v / p.T, t = v - seq * p.T;
  const __nv_bfloat16* q = p.q + seq * p.q_seq + t * p.q_token + static_cast<int64_t>(g) * p.hg * p.q_head;
  // the weights of the terms, on their way with the row's length (a query that is none is not read)
  const int count = p.n_tokens ? p.n_tokens[seq] : p.T;
  float up = 0.f, down = 0.f, up_rest = 0.f, down_rest = 0.f;
  if (tid < kHeadDim && t < count && count <= p.T)
#pragma unroll 4
    for (int h = 0; h < p.hg; ++h) {
      const float x = __bfloat162float(q[h * p.q_head + tid]);
      up = sum_and_rest(up, x < 0.f ? 0.f : x, &up_rest);   // (a NaN goes into both)
      down = sum_and_rest(down, x > 0.f ? 0.f : x, &down_rest);
    }
  const SparseQuery sq = sparse_query(p.rows, p.n_tokens, pg.len, pg.n_rows, pg.max_pages, pg.shift, p.T, v);
  const int pages = !sq.live || sq.pos < 0 ? 0 : (sq.pos >> pg.shift) + 1;
  const int take = min(pages, p.n_list);
  const int32_t* entries = pg.table + static_cast<int64_t>(sq.row) * pg.max_pages;
  // pages lo .. hi - 1 compete for `need` places; the others are taken anyway
  const int lo = take == pages ? pages : p.n_first, hi = take == pages ? pages : pages - p.n_last;
  const int need = take - (pages - (hi - lo));
  const bool here = hi - lo <= kChoosePages;   // the scores fit shared memory
  const int64_t place = (static_cast<int64_t>(item) * p.G + g) * pg.max_pages;
  uint32_t* far = p.scores + place - lo;
  if (tid == 0 && g == 0 && rank == 0) {   // what the attention has to know of the query
    if (sq.wrong) atomicOr(p.err, kErrRow);
    const int last = sq.pos & ((1 << pg.shift) - 1);
    p.tokens[item] = make_int2(sq.live && sq.pos >= 0 ? ((take - 1) << pg.shift) + last + 1 : -1, sq.live);
  }
  const int per = p.ctas * kChooseWarps * kPagesAtOnce, own = (rank * kChooseWarps + warp) * kPagesAtOnce;
  if (tid == 0) s.least = ~0u, s.most = 0, s.few = 0;
  if (rank == 0)
    for (int i = tid; i < kBins; i += kChooseThreads) s.bins[i] = 0;
  if (need > 0) {
    int id = lo + own + (lane & 7) < hi ? entries[lo + own + (lane & 7)] : -1;   // lane l: page l of the eight
    if (tid < kHeadDim) {
      s.up[tid] = up;
      s.down[tid] = down;
      s.up_rest[tid] = fabsf(up) < INFINITY ? up_rest : 0.f;
      s.down_rest[tid] = fabsf(down) < INFINITY ? down_rest : 0.f;
    }
    __syncthreads();
    float w[8];   // this lane's terms: eight channels, the least keys (lanes 0 .. 15) or the greatest
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = lane < 16 ? s.down[lane * 8 + i] : s.up[lane * 8 + i - kHeadDim];
    uint32_t size = 0;
    cluster_wait();
    const uint32_t first_cta = dsmem_map(s.key, 0);
    for (int j0 = lo + own; j0 < hi; j0 += per) {
      if (j0 + (lane & 7) < hi && (id < 0 || id >= pg.n_pages)) atomicOr(p.err, kErrRow);   // (its score is 0)
      uint4 x[kPagesAtOnce];
#pragma unroll
      for (int u = 0; u < kPagesAtOnce; ++u) {
        const int page = __shfl_sync(kFull, id, u);
        x[u] = make_uint4(0u, 0u, 0u, 0u);
        if (page >= 0 && page < pg.n_pages)
          x[u] = ld_stream(reinterpret_cast<const uint4*>(p.bounds + page * p.bounds_page + static_cast<int64_t>(g) * 2 * kHeadDim) + lane);
      }
      const int next = j0 + per + (lane & 7);
      id = next < hi ? entries[next] : -1;
      float sum[kPagesAtOnce];
#pragma unroll
      for (int u = 0; u < kPagesAtOnce; ++u) {
        const uint32_t words[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y0 = __uint_as_float(words[i] << 16), y1 = __uint_as_float(words[i] & 0xFFFF0000u);
          a = fmaf(w[2 * i], y0, a);
          a = fmaf(w[2 * i + 1], y1, a);
          b = fmaf(fabsf(w[2 * i]), fabsf(y0), b);
          b = fmaf(fabsf(w[2 * i + 1]), fabsf(y1), b);
        }
        sum[u] = a;
        size = max(size, __float_as_uint(b));   // (sizes are not negative; a NaN is above infinity)
      }
      // the sum of page (lane & 7), in every lane
#pragma unroll
      for (int o = 4; o; o >>= 1)
#pragma unroll
        for (int u = 0; u < o; ++u) {
          const bool upper = lane & o;
          const float mine = upper ? sum[u + o] : sum[u], theirs = upper ? sum[u] : sum[u + o];
          sum[u] = mine + __shfl_xor_sync(kFull, theirs, o);
        }
      sum[0] += __shfl_xor_sync(kFull, sum[0], 8);
      sum[0] += __shfl_xor_sync(kFull, sum[0], 16);
      const int j = j0 + (lane & 7);
      if (lane < 8 && j < hi) {
        const uint32_t k = order_of(sum[0] + 0.f);   // (-0 is 0)
        if (here) dsmem_st_u32(first_cta + (j - lo) * 4, k);
        else far[j] = k;
      }
    }
    float total = __uint_as_float(size);
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kFull, total, o);
    if (lane == 0) dsmem_st_u32(dsmem_map(&s.size[rank][warp], 0), __float_as_uint(total));
  } else {
    cluster_wait();
  }
  cluster_sync();   // (every CTA of the cluster has the same `need`, or leaves from here as well)
  if (rank != 0 || !sq.live) return;

  int32_t* list = p.list + (static_cast<int64_t>(item) * p.G + g) * p.n_list;
  int32_t* chosen = p.chosen ? p.chosen + (static_cast<int64_t>(v) * p.G + g) * p.n_chosen : nullptr;
  if (chosen)
    for (int i = take + tid; i < p.n_chosen; i += kChooseThreads) chosen[i] = -1;
  uint32_t* keys = here ? s.key - lo : far;   // from here on: 0 (not taken) or 1
  if (need > 0) {
    int of_it;
    const int n = hi - lo, run = (n + kChooseThreads - 1) / kChooseThreads;
    const bool ranked = run <= kRun;   // (shared memory holds them)
    uint32_t mine[kRun];               // pages lo + tid run ..
    int number[kRun];                  // and theirs in the pool, on their way
    float top, bottom;                 // the k-th greatest score lies between them
    if (ranked) {
      // bins of equal width between the least key and the greatest: the one that the k-th greatest is in holds
      // hardly any other (digits of eight bits took four rounds, 3 us)
      uint32_t least = ~0u, most = 0;
#pragma unroll
      for (int r = 0; r < kRun; ++r) {
        const bool real = r < run && tid * run + r < n;
        mine[r] = real ? s.key[tid * run + r] : 0;
        number[r] = real ? entries[lo + tid * run + r] : 0;
        if (real) least = min(least, mine[r]), most = max(most, mine[r]);
      }
      least = __reduce_min_sync(kFull, least);
      most = __reduce_max_sync(kFull, most);
      if (lane == 0) {
        atomicMin(&s.least, least);
        atomicMax(&s.most, most);
      }
      __syncthreads();
      least = s.least;
      most = s.most;
      const int shift = max(0, 32 - __clz(most - least) - 11);   // (kBins = 2^11)
#pragma unroll
      for (int r = 0; r < kRun; ++r)
        if (r < run && tid * run + r < n) atomicAdd(&s.bins[(mine[r] - least) >> shift], 1);
      __syncthreads();
      constexpr int kOwn = kBins / kChooseThreads;   // bins of a thread, from the greatest down
      int count[kOwn], sum = 0, total;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) sum += count[i] = s.bins[kBins - 1 - tid * kOwn - i];
      int left = need - block_before<false>(sum, s.bin_sum[0], &total);
      if (left > 0 && left <= sum) {
        int i = 0;
#pragma unroll
        for (int u = 0; u < kOwn - 1; ++u)
          if (i == u && count[u] < left) left -= count[u], ++i;
        s.bin = kBins - 1 - tid * kOwn - i;
      }
      __syncthreads();
      const uint32_t from = least + (static_cast<uint32_t>(s.bin) << shift);
      bottom = value_of(from);
      top = value_of(min(most, from + ((1u << shift) - 1)));
    } else {
      top = bottom = value_of(kth_greatest<uint32_t>(s, lo, hi, need, [&](int j) { return keys[j]; }, &of_it));
    }
    uint32_t size = 0;
    for (int i = lane; i < p.ctas * kChooseWarps; i += 32) size = max(size, s.size[i / kChooseWarps][i % kChooseWarps]);
    const float E = __uint_as_float(__reduce_max_sync(kFull, size)) * ((16 + p.hg) * 1.001f * 0x1p-24f) + 0x1p-140f;
    const float above = top + 2.1f * E, below = bottom - 2.1f * E;
    int sure = 0, close = 0;
    if (ranked) {
#pragma unroll
      for (int r = 0; r < kRun; ++r) {
        const float x = value_of(mine[r]);
        const bool real = r < run && tid * run + r < n, in = x > above;
        sure += real && in;
        close += real && !in && !(x < below);
      }
      int total;   // (both counts in one sum: neither passes 1,024)
      const int before = block_before<false>(sure << 16 | close, s.bin_sum[1], &total);
      if (need - (total >> 16) == (total & 0xffff)) {   // the usual case: as many as there are places
        int to = (before >> 16) + (before & 0xffff) + lo;
#pragma unroll
        for (int r = 0; r < kRun; ++r)
          if (r < run && tid * run + r < n && !(value_of(mine[r]) < below)) {
            const int j = lo + tid * run + r;
            list[to] = number[r];
            if (chosen) chosen[to] = j;
            ++to;
          }
        for (int i = tid; i < lo + pages - hi; i += kChooseThreads) {   // the first pages and the last ones
          const int j = i < lo ? i : hi + i - lo, to_j = i < lo ? i : lo + need + i - lo;
          list[to_j] = entries[j];
          if (chosen) chosen[to_j] = j;
        }
        return;
      }
      sure = close = 0;
    }
    for (int j = lo + tid; j < hi; j += kChooseThreads) {
      const float x = value_of(keys[j]);
      const bool in = x > above, out = x < below;   // (where E is not a number: neither)
      sure += in;
      close += !in && !out;
    }
    int n_sure, n_close;
    block_before(sure, s.warp_sum, &n_sure);
    block_before(close, s.warp_sum, &n_close);
    const int left = need - n_sure;
    const bool all = left == n_close, few = n_close <= kFew;
    uint64_t* wide = p.keys + place - lo;
    for (int j = lo + tid; j < hi; j += kChooseThreads) {
      const float x = value_of(keys[j]);
      const bool in = x > above, near = !in && !(x < below);
      if (few || all) {
        if (near && !all) s.close_page[atomicAdd(&s.few, 1)] = j;
        keys[j] = in || (near && all);
      } else {
        wide[j] = in ? ~uint64_t(0) : near ? 1 : 0;   // (scores are above 1, and below ~0)
      }
    }
    __syncthreads();
    if (!all) {
      // the same terms in 64 bits (of which the weights have 47: what 32 left out is known), by the warps that have a page:
      // the unit for them is slow, and all warps' weights from the queries again took 12 us
      double wd[8];
      if (!few || warp < n_close)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = (lane & 15) * 8 + i;
          wd[i] = lane < 16 ? static_cast<double>(s.down[c]) + static_cast<double>(s.down_rest[c])
                            : static_cast<double>(s.up[c]) + static_cast<double>(s.up_rest[c]);
        }
      auto score = [&](int j) {   // by the whole warp
        const int page = entries[j];
        double a = 0;
        if (page >= 0 && page < pg.n_pages) {
          const uint4 x = ld_stream(reinterpret_cast<const uint4*>(p.bounds + page * p.bounds_page + static_cast<int64_t>(g) * 2 * kHeadDim) + lane);
          const uint32_t words[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a = fma(wd[2 * i], static_cast<double>(__uint_as_float(words[i] << 16)), a);
            a = fma(wd[2 * i + 1], static_cast<double>(__uint_as_float(words[i] & 0xFFFF0000u)), a);
          }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(kFull, a, o);
        return order_of(a);
      };
      if (few) {
        for (int i = warp; i < n_close; i += kChooseWarps) {
          const uint64_t k = score(s.close_page[i]);
          if (lane == 0) s.close[i] = k;
        }
        __syncthreads();
        if (tid < n_close) {
          const uint64_t k = s.close[tid];
          const int j = s.close_page[tid];
          int better = 0;
          for (int i = 0; i < n_close; ++i) better += s.close[i] > k || (s.close[i] == k && s.close_page[i] < j);
          keys[j] = better < left;
        }
        __syncthreads();
      } else {
        for (int j = lo + warp; j < hi; j += kChooseWarps)
          if (wide[j] == 1) {
            const uint64_t k = score(j);
            __syncwarp();
            if (lane == 0) wide[j] = k;
          }
        __syncthreads();
        const uint64_t least = kth_greatest<uint64_t>(s, lo, hi, need, [&](int j) { return wide[j]; }, &of_it);
        // of the pages that have the least key the lowest `of_it`: every thread a run of pages
        const int run = (hi - lo + kChooseThreads - 1) / kChooseThreads, b = min(lo + tid * run, hi), e = min(b + run, hi);
        int equal = 0, total;
        for (int j = b; j < e; ++j) equal += wide[j] == least;
        int before = block_before(equal, s.warp_sum, &total);
        for (int j = b; j < e; ++j) keys[j] = wide[j] > least || (wide[j] == least && before++ < of_it);
        __syncthreads();
      }
    }
  }
  // the list, in the order of the pages: every thread a run of them
  const int run = (pages + kChooseThreads - 1) / kChooseThreads, b = min(tid * run, pages), e = min(b + run, pages);
  __syncthreads();
  auto taken = [&](int j) { return j < lo || j >= hi || (need > 0 && keys[j]); };
  int mine = 0, total;
  for (int j = b; j < e; ++j) mine += taken(j);
  int at = block_before(mine, s.warp_sum, &total);
  for (int j = b; j < e; ++j)
    if (taken(j)) {
      list[at] = entries[j];
      if (chosen) chosen[at] = j;
      ++at;
    }
}

cudaError_t page_choose_configure() {
  return cudaFuncSetAttribute(k_page_choose, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(ChooseSmem));
}

cudaError_t page_choose_launch(const ChooseParams& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.items * p.ctas, p.G), kChooseThreads, stream);
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.numAttrs = 2;
  cfg.dynamicSmemBytes = sizeof(ChooseSmem);
  return cudaLaunchKernelEx(&cfg, k_page_choose, p);
}

}  // namespace starkv
