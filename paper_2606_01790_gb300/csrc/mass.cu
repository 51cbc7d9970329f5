// Attention mass of cached tokens, and the choice of those that stay by it.
//
// Mass: token j of a row, KV head g, after a call whose queries (the row's last n tokens)
// have normalisers lse:
//   mass_j = (j < L - n ? decay mass_j : 0) + sum_t sum_{h in g} [t sees j] exp(q_th . k_j / sqrt(d) - lse_th).
#include <algorithm>

#include "common.cuh"
#include "mass.cuh"
#include "ptx.cuh"

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

constexpr int kThreads = 256;
constexpr int kKeys = 64;       // keys of a tile
constexpr int kQueries = 32;    // (token, head) pairs at a time
constexpr int kKeyStride = kHeadDim + 8;   // (rows 16 bytes apart in the banks)

}  // namespace

// Block (x, sequence, KV head): tiles x, x + gridDim.x, ... of 64 keys, thread (key, a quarter
// of the pairs).
__global__ void __launch_bounds__(kThreads) k_mass(const __grid_constant__ MassParams p) {
  __shared__ __align__(16) __nv_bfloat16 s_k[kKeys][kKeyStride];
  __shared__ float s_q[kQueries][kHeadDim];
  __shared__ float s_lse[kQueries];
  __shared__ float s_sum[4][kKeys];
  griddep_launch_dependents();
  griddep_wait();
  const int tid = threadIdx.x, seq = blockIdx.y, g = blockIdx.z;
  const int row = p.rows ? p.rows[seq] : seq;
  const int n = p.n_tokens ? p.n_tokens[seq] : p.T;
  const int L = row >= 0 && row < p.n_rows ? p.len[row] : -1;
  bool bad = n < 0 || n > p.T || (n > 0 && (L < n || L > static_cast<int64_t>(p.max_pages) << p.shift));
  if (p.rows && n != 0)   // a row that two sequences with queries name would get one's or the other's
    for (int i = tid; i < p.n; i += kThreads) bad = bad || (i != seq && p.rows[i] == row && !(p.n_tokens && p.n_tokens[i] == 0));
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(p.err, kErrRow);
    return;
  }
  if (n == 0) return;
  const int32_t* entries = p.table + static_cast<int64_t>(row) * p.max_pages;
  float* mass = p.mass.m + row * p.mass.row_stride + g * p.mass.group_stride;
  const int P = 1 << p.shift, ctx = L - n;
  const int key = tid & (kKeys - 1), quarter = tid >> 6;
  for (int k0 = blockIdx.x * kKeys; k0 < L; k0 += gridDim.x * kKeys) {
    __syncthreads();
    for (int i = tid; i < kKeys * (kHeadDim / 8); i += kThreads) {
      const int r = i / (kHeadDim / 8), c = i % (kHeadDim / 8), j = k0 + r;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (j < L) {
        const int page = entries[j >> p.shift];
        if (page >= 0 && page < p.n_pages)
          x = *reinterpret_cast<const uint4*>(p.k + page * p.page_stride + ((static_cast<int64_t>(g) << p.shift) + (j & (P - 1))) * kHeadDim + c * 8);
        else atomicOr(p.err, kErrRow);
      }
      *reinterpret_cast<uint4*>(&s_k[r][c * 8]) = x;
    }
    const int j = k0 + key;
    float sum = 0.f;
    for (int c0 = 0; c0 < n * p.hg; c0 += kQueries) {
      __syncthreads();
      for (int i = tid; i < kQueries * kHeadDim; i += kThreads) {
        const int c = c0 + i / kHeadDim, t = c / p.hg, h = g * p.hg + c - t * p.hg;
        s_q[i / kHeadDim][i % kHeadDim] =
            t < n ? __bfloat162float(p.q[seq * p.q_seq + t * p.q_token + h * p.q_head + i % kHeadDim]) : 0.f;
        if (i % kHeadDim == 0) s_lse[i / kHeadDim] = t < n ? p.lse[(static_cast<int64_t>(seq) * p.T + t) * p.H + h] * 1.4426950408889634f : 0.f;
      }
      __syncthreads();
      float acc[kQueries / 4] = {};
      for (int d = 0; d < kHeadDim; d += 8) {
        float k[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = __bfloat162float(s_k[key][d + e]);
#pragma unroll
        for (int u = 0; u < kQueries / 4; ++u)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[u] = fmaf(k[e], s_q[quarter * 8 + u][d + e], acc[u]);
      }
#pragma unroll
      for (int u = 0; u < kQueries / 4; ++u) {
        const int c = c0 + quarter * 8 + u, t = c / p.hg, i = ctx + t;
        bool seen = t < n && j <= i && (j < p.n_sink || j > i - p.window);
        if (p.tree) seen = t < n && (j < ctx || (j < L && (p.mask[static_cast<int64_t>(seq) * p.T + t] >> (j - ctx) & 1)));
        if (seen) sum += exp2f(fmaf(acc[u], p.scale2, -s_lse[quarter * 8 + u]));
      }
    }
    s_sum[quarter][key] = sum;
    __syncthreads();
    if (tid < kKeys && j < L) {
      const float had = j < ctx ? p.decay * mass[j] : 0.f;
      mass[j] = had + ((s_sum[0][key] + s_sum[1][key]) + (s_sum[2][key] + s_sum[3][key]));
    }
  }
}

cudaError_t mass_launch(const MassParams& p, int num_sms, cudaStream_t stream) {
  const int64_t tiles = ((static_cast<int64_t>(p.max_pages) << p.shift) + kKeys - 1) / kKeys;
  const int64_t most = std::max<int64_t>(1, 8 * num_sms / (static_cast<int64_t>(p.n) * p.G));
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(static_cast<unsigned>(std::min(tiles, most)), p.n, p.G), kThreads, stream);
  return cudaLaunchKernelEx(&cfg, k_mass, p);
}

// ---------------------------------------------------------------- eviction

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;

// Ascending order; a NaN (a mass that is none) comes with the greatest, infinity, so that its token stays.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) x = INFINITY;
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0 is 0)
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(double x) {
  if (x != x) x = INFINITY;
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

// Sum over the block of 0 / 1 flags in front of this thread's, and all of them.
__device__ int2 count_before(bool flag, int* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t m = __ballot_sync(kFull, flag);
  if (lane == 0) warp_sum[warp] = __popc(m);
  __syncthreads();
  int s = warp_sum[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kFull, s, o);
    if (lane >= o) s += x;
  }
  const int all = __shfl_sync(kFull, s, 31), in_front = __shfl_sync(kFull, s, max(warp - 1, 0));
  __syncthreads();
  return make_int2((warp ? in_front : 0) + __popc(m & ((1u << lane) - 1)), all);
}

}  // namespace

// Block (set, layer, sequence): the budget tokens j < L - w of greatest mass (PER_HEAD: of one
// KV head, else of all of them added up in 64 bits, which 32-bit masses fill without a
// rounding where they lie within 2^24 of each other), equal ones the lowest first, in ascending
// order; then the mass of the kept ones and of the window moves to their new places.
template <bool PER_HEAD>
__global__ void __launch_bounds__(kSelThreads)
    k_mass_select(const __grid_constant__ PagesView pg, const __grid_constant__ SeqBatch b, const int32_t* rows, int row0, int w,
                  const PagePlan* plan, const __grid_constant__ MassView mv) {
  using Value = typename std::conditional<PER_HEAD, float, double>::type;
  using Key = typename std::conditional<PER_HEAD, uint32_t, uint64_t>::type;
  __shared__ int hist[256], warp_sum[kSelWarps];
  __shared__ Key s_prefix;
  __shared__ int s_need;
  griddep_launch_dependents();
  griddep_wait();
  if (!plan->ok) return;
  const int tid = threadIdx.x, set = blockIdx.x, layer = blockIdx.y, seq = blockIdx.z;
  const SeqView& sv = b.s[seq];
  const int B = sv.budget, Lp = sv.Lp;
  const int row = rows ? rows[row0 + seq] : row0 + seq;
  const int g0 = PER_HEAD ? set : 0, g1 = PER_HEAD ? set + 1 : pg.G;
  float* mass = mv.m + layer * mv.layer_stride + row * mv.row_stride;
  int32_t* idx = sv.idx + (static_cast<int64_t>(layer) * (PER_HEAD ? pg.G : 1) + set) * B;
  auto key_of = [&](int j) {
    Value x = mass[g0 * mv.group_stride + j];
    for (int g = g0 + 1; g < g1; ++g) x += static_cast<Value>(mass[g * mv.group_stride + j]);
    return order_key(x);
  };
  if (tid == 0) s_prefix = 0, s_need = B;
  __syncthreads();
  if (B > 0 && B < Lp)
    for (int bit = static_cast<int>(sizeof(Key)) * 8 - 8; bit >= 0; bit -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const Key prefix = s_prefix;
      for (int j = tid; j < Lp; j += kSelThreads) {
        const Key key = key_of(j);
        if (bit + 8 == static_cast<int>(sizeof(Key)) * 8 || (key ^ prefix) >> (bit + 8) == 0) atomicAdd(&hist[key >> bit & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int left = s_need, d = 255;
        while (d > 0 && hist[d] < left) left -= hist[d--];
        s_prefix = prefix | static_cast<Key>(d) << bit;
        s_need = left;
      }
      __syncthreads();
    }
  const Key least = s_prefix;
  const int need = s_need;   // of the tokens that have the least key
  int at = 0, equal = 0;
  if (B > 0)
    for (int j0 = 0; j0 < Lp; j0 += kSelThreads) {
      const int j = j0 + tid;
      const Key key = j < Lp ? key_of(j) : 0;
      const int2 e = count_before(j < Lp && key == least, warp_sum);
      const bool in = j < Lp && (B == Lp || key > least || (key == least && equal + e.x < need));
      const int2 c = count_before(in, warp_sum);
      if (in) idx[at + c.x] = j;
      equal += e.y;
      at += c.y;
    }
  __syncthreads();   // the indices are written
  // A token's new place is never behind its old one: what a round writes has been read.
  for (int r0 = 0; r0 < B + w; r0 += kSelThreads) {
    const int r = r0 + tid;
    const int from = r < B ? idx[r] : Lp + (r - B);
    for (int g = g0; g < g1; ++g) {
      float* m = mass + g * mv.group_stride;
      const float x = r < B + w ? m[from] : 0.f;
      __syncthreads();
      if (r < B + w) m[r] = x;
    }
    __syncthreads();
  }
}

cudaError_t mass_select_launch(const PagesView& pg, const SeqBatch& b, const int32_t* rows, int row0, int w, int per_head,
                               const PagePlan* plan, const MassView& mass, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(per_head ? pg.G : 1, b.nlayers, b.nseq), kSelThreads, stream);
  return cudaLaunchKernelEx(&cfg, per_head ? k_mass_select<true> : k_mass_select<false>, pg, b, rows, row0, w, plan, mass);
}

}  // namespace starkv
