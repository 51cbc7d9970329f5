// Attention of new tokens over a paged cache.  Query t of sequence s is the token
// at position i = L - n + t of its row (L tokens, n queries) and sees
//   tree:  the keys j < L - n, and the drafted token j = L - n + b where bit b of
//          mask[t] is set;
//   sink:  the keys j <= i with j < n_sink or j > i - window.
//   o[t,h]   = sum_j softmax_j(q[t,h] . K[g(h),j] / sqrt(d)) V[g(h),j]
//   lse[t,h] = log sum_j exp(q[t,h] . K[g(h),j] / sqrt(d))
// over the keys seen; a query that sees none has o = 0 and lse = -inf.  One warp
// per (sequence, token, head), one key at a time, all sums in fp32.
#include "common.cuh"
#include "paged_attn.cuh"
#include "ptx.cuh"

namespace starkv {

namespace {

constexpr int kThreads = 128;
constexpr uint32_t kFull = 0xffffffffu;

__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xFFFF0000u));
}

}  // namespace

__global__ void __launch_bounds__(kThreads) k_paged_attn(const __grid_constant__ PagedAttnParams p) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t nwarp = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  const int64_t total = static_cast<int64_t>(p.n) * p.T * p.H;
  for (int64_t w = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); w < total; w += nwarp) {
    const int h = static_cast<int>(w % p.H);
    const int t = static_cast<int>(w / p.H % p.T);
    const int s = static_cast<int>(w / p.H / p.T);
    const int g = h / (p.H / p.G);
    const int row = p.rows ? p.rows[s] : s;
    const int n = p.n_tokens ? p.n_tokens[s] : p.T;
    if (n < 0 || n > p.T) {
      if (lane == 0) atomicOr(p.err, kErrRow);
      continue;
    }
    if (t >= n) continue;
    int L = row >= 0 && row < p.n_rows ? p.len[row] : -1;
    if (L < n || L > static_cast<int64_t>(p.max_pages) << p.shift) {
      if (lane == 0) atomicOr(p.err, kErrRow);
      L = 0;   // nothing is seen
    }
    const int i = L - n + t;
    const uint64_t mask = p.tree ? p.mask[static_cast<int64_t>(s) * p.T + t] : 0;
    const float4 q = load4(p.q + s * p.q_seq + t * p.q_token + h * p.q_head + lane * 4);
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const int32_t* table = p.table + static_cast<int64_t>(row) * p.max_pages;
    const int end = p.tree ? L : min(L, i + 1);
    for (int j = 0; j < end; ++j) {
      const bool seen = p.tree ? j < L - n || (mask >> (j - (L - n)) & 1) : j < p.n_sink || j > i - p.window;
      if (!seen) continue;
      const int page = table[j >> p.shift];
      if (page < 0 || page >= p.n_pages) {
        if (lane == 0) atomicOr(p.err, kErrRow);
        continue;
      }
      const int64_t at = page * p.page_stride + ((static_cast<int64_t>(g) << p.shift) + (j & ((1 << p.shift) - 1))) * kHeadDim + lane * 4;
      const float4 k = load4(p.k + at);
      float z = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
      for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(kFull, z, o);
      z *= p.scale2;
      const float4 v = load4(p.v + at);
      const float top = fmaxf(m, z), ref = top == -INFINITY ? 0.f : top;
      const float keep = exp2f(m - ref), e = exp2f(z - ref);
      m = top;
      l = l * keep + e;
      acc = make_float4(acc.x * keep + e * v.x, acc.y * keep + e * v.y, acc.z * keep + e * v.z, acc.w * keep + e * v.w);
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    __nv_bfloat162 out[2] = {__floats2bfloat162_rn(acc.x * inv, acc.y * inv), __floats2bfloat162_rn(acc.z * inv, acc.w * inv)};
    *reinterpret_cast<uint2*>(p.o + s * p.o_seq + t * p.o_token + h * p.o_head + lane * 4) = *reinterpret_cast<uint2*>(out);
    if (p.lse && lane == 0)
      p.lse[(static_cast<int64_t>(s) * p.T + t) * p.H + h] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  }
}

cudaError_t paged_attn_launch(const PagedAttnParams& p, int num_sms, cudaStream_t stream) {
  const int64_t warps = static_cast<int64_t>(p.n) * p.T * p.H;
  if (warps <= 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(min((warps + 3) / 4, static_cast<int64_t>(num_sms) * 16)));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_paged_attn, p);
}

}  // namespace starkv
