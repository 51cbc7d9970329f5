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

// ---------------------------------------------------------------- mass: units and their order

constexpr int kMassWarps = 22;
constexpr int kThreads = 32 * kMassWarps;
constexpr int kQueryWarp = 2, kSoftWarp = 6;      // first of the query warps (4) and of the weighing warps (16)
constexpr int kTileBytes = kMassTile * 256;       // 128 keys x 128 bf16, or as many (token, head) pairs: 32 KB
constexpr int kHalfBytes = kTileBytes / 2;
constexpr int kKeySlots = 4, kQuerySlots = 2;     // rings; a tile of keys has an accumulator and a warpgroup of its own
constexpr int kTmemCols = 512;
constexpr uint64_t kDrainWaitNs = 2000000000ull;

struct Item {
  int L, n;   // tokens of the row and queries; n = 0: nothing to do
};

// A block of (token, head) pairs as the weighing warps see it.
struct Pairs {
  alignas(16) float lse[kMassTile];   // -lse in base 2
  int pos[kMassTile];                 // position of the token
  uint64_t bits[kMassTile];           // tree: drafted tokens seen
};

struct Start {
  int seq, g, s, b;
};

struct Ctl {
  uint64_t k_full[kKeySlots], k_empty[kKeySlots];
  uint64_t q_full[kQuerySlots], q_empty[kQuerySlots];
  uint64_t s_full[kKeySlots], s_empty[kKeySlots];   // accumulators
  uint64_t drain;
  uint32_t tmem_base;
  volatile int abort;
  int span;             // tiles of a group
  Start start;
  Pairs pairs[kQuerySlots];
  int64_t before[kMaxCallRows + 1];   // units before a sequence
  Item item[kMaxCallRows];
};

// The tiles of one group of a row and the query blocks that see some of it.
struct Group {
  int k0, tiles, lo, hi;   // first key; tiles of 128; blocks lo .. hi - 1

  __device__ __forceinline__ Group(const MassParams& p, const Item& it, int span, int s) {
    k0 = s * span * kMassTile;
    const int end = min(it.L, k0 + span * kMassTile), ctx = it.L - it.n;
    tiles = (end - k0 + kMassTile - 1) / kMassTile;
    int t0 = 0, t1 = it.n;
    if (!p.tree) {
      t0 = max(0, k0 - ctx);
      if (k0 >= p.n_sink) t1 = min(it.n, end - 1 + p.window - ctx);
    }
    if (!p.cut && t0 < t1) t0 = 0, t1 = it.n;   // (blocks that stay in shared memory stay whole)
    lo = t0 / p.tpb * p.chunks;
    hi = t1 <= t0 ? lo : (t1 + p.tpb - 1) / p.tpb * p.chunks;
  }
  // a group that nothing sees is a unit all the same: its mass may fade
  __device__ __forceinline__ int units(const MassParams& p) const { return p.cut ? max(1, hi - lo) : 1; }
};

__device__ __forceinline__ int groups_of(int L, int span) { return (L + span * kMassTile - 1) / (span * kMassTile); }

// Runs of blocks of one group, in the order of a CTA's range.
struct PieceIter {
  int seq, g, s;
  int b0, b1;        // blocks b0 .. b1 - 1
  int64_t rem;       // units of the range from here on
  Group grp;
  Item it;
  __device__ __forceinline__ PieceIter(const MassParams& p, const Ctl* ctl, int64_t units)
      : seq(ctl->start.seq), g(ctl->start.g), s(ctl->start.s), rem(units), grp(p, Item{0, 0}, 1, 0), it{0, 0} {
    if (rem <= 0) return;
    it = ctl->item[seq];
    take(p, ctl, ctl->start.b);
  }
  __device__ __forceinline__ bool valid() const { return rem > 0; }
  __device__ __forceinline__ bool whole() const { return b0 == grp.lo && b1 == grp.hi; }
  __device__ __forceinline__ void take(const MassParams& p, const Ctl* ctl, int from) {
    grp = Group(p, it, ctl->span, s);
    b0 = grp.lo + from;
    b1 = p.cut ? static_cast<int>(min(static_cast<int64_t>(grp.hi), b0 + rem)) : grp.hi;
  }
  // the last group of this row and KV head that the range has
  __device__ __forceinline__ bool last_of_head(const Ctl* ctl) const {
    return rem <= 1 || s + 1 == groups_of(it.L, ctl->span);
  }
  __device__ __forceinline__ void next(const MassParams& p, const Ctl* ctl) {
    rem -= p.cut ? max(1, b1 - b0) : 1;
    if (rem <= 0) return;
    if (++s == groups_of(it.L, ctl->span)) {
      s = 0;
      if (++g == p.G) {
        g = 0;
        do ++seq;
        while (ctl->before[seq + 1] == ctl->before[seq]);
        it = ctl->item[seq];
      }
    }
    take(p, ctl, 0);
  }
};

__device__ __forceinline__ int64_t range_begin(int64_t T, int c, int P) { return c < P ? T * c / P : T; }
// Ranges of a launch of T units on P CTAs: as many, but none empty.
__device__ __forceinline__ int ranges_of(int64_t T, int P) { return T < P ? max(static_cast<int>(T), 1) : P; }
// Range (of P) that holds flat unit f
__device__ __forceinline__ int range_of(int64_t f, int64_t T, int P) { return static_cast<int>(((f + 1) * P - 1) / T); }

// Every sequence's length and queries, the groups' span, the units before each sequence and this CTA's
// first unit.  `named`: 2 bits a row of the table (in shared memory), for rows that two sequences name.
__device__ void plan(const MassParams& p, Ctl* ctl, uint32_t* named, int64_t* fb, int64_t* fe, int64_t* total, int* ranges) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int words = (p.n_rows + 31) >> 5;
  const bool rivals = p.rows && p.n > 1;
  if (rivals) {
    for (int i = tid; i < 2 * words; i += kThreads) named[i] = 0;
    __syncthreads();
  }
  __shared__ unsigned long long tiles;
  if (tid == 0) tiles = 0;
  for (int i = tid; i < p.n; i += kThreads) {
    const int row = p.rows ? p.rows[i] : p.row0 + i;
    Item it;
    it.n = p.n_tokens ? p.n_tokens[i] : p.T;
    it.L = row >= 0 && row < p.n_rows ? p.len[row] : -1;
    if (it.n < 0 || it.n > p.T || (it.n > 0 && (it.L < it.n || it.L > static_cast<int64_t>(p.max_pages) << p.shift))) {
      it.n = 0;
      atomicOr(p.err, kErrRow);
    }
    if (rivals && it.n > 0 && (atomicOr(&named[row >> 5], 1u << (row & 31)) & (1u << (row & 31))))
      atomicOr(&named[words + (row >> 5)], 1u << (row & 31));
    ctl->item[i] = it;
  }
  __syncthreads();
  unsigned long long mine = 0;
  for (int i = tid; i < p.n; i += kThreads) {
    const int row = p.rows ? p.rows[i] : p.row0 + i;
    if (rivals && ctl->item[i].n > 0 && (named[words + (row >> 5)] >> (row & 31) & 1)) {
      ctl->item[i].n = 0;
      atomicOr(p.err, kErrRow);
    }
    if (ctl->item[i].n > 0) mine += groups_of(ctl->item[i].L, 1);
  }
  if (mine) atomicAdd(&tiles, mine);
  __syncthreads();
  const int span = p.span > 1 && static_cast<int64_t>(tiles) * p.G >= static_cast<int64_t>(p.span_from) * gridDim.x ? p.span : 1;
  if (tid == 0) ctl->span = span;
  for (int i = warp; i < p.n; i += kMassWarps) {
    const Item it = ctl->item[i];
    const int ng = it.n > 0 ? groups_of(it.L, span) : 0;
    int64_t u = 0;
    if (!p.cut) u = lane == 0 ? ng : 0;
    else
      for (int s = lane; s < ng; s += 32) u += Group(p, it, span, s).units(p);
#pragma unroll
    for (int o = 16; o; o >>= 1) u += __shfl_xor_sync(kFull, u, o);
    if (lane == 0) ctl->before[i + 1] = u * p.G;
  }
  __syncthreads();
  if (warp == 0) {
    int64_t at = 0;
    for (int i0 = 0; i0 < p.n; i0 += 32) {
      int64_t u = i0 + lane < p.n ? ctl->before[i0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(kFull, u, o);
        if (lane >= o) u += x;
      }
      if (i0 + lane < p.n) ctl->before[i0 + lane + 1] = at + u;
      at += __shfl_sync(kFull, u, 31);
    }
    if (lane == 0) ctl->before[0] = 0;
    __syncwarp();
    const int64_t T = ctl->before[p.n];
    const int R = ranges_of(T, gridDim.x);
    const int64_t f = range_begin(T, blockIdx.x, R);
    if (f < range_begin(T, blockIdx.x + 1, R)) {
      int a = 0, b = p.n;   // the last sequence with no more than f units before it
      while (b - a > 1) {
        const int mid = (a + b) >> 1;
        if (ctl->before[mid] <= f) a = mid;
        else b = mid;
      }
      while (ctl->before[a + 1] <= f) ++a;
      const int64_t per = (ctl->before[a + 1] - ctl->before[a]) / p.G;
      int64_t off = f - ctl->before[a];
      Start st;
      st.seq = a;
      st.g = static_cast<int>(off / per);
      off -= st.g * per;
      st.s = static_cast<int>(off);
      st.b = 0;
      if (p.cut) {
        const Item it = ctl->item[a];
        const int ng = groups_of(it.L, span);
        for (int s0 = 0;; s0 += 32) {
          const int u = s0 + lane < ng ? Group(p, it, span, s0 + lane).units(p) : 0;
          int64_t inc = u;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(kFull, inc, o);
            if (lane >= o) inc += x;
          }
          const uint32_t past = __ballot_sync(kFull, inc > off);
          if (past || s0 + 32 >= ng) {
            const int l = past ? __ffs(past) - 1 : 31;
            st.s = s0 + l;
            st.b = static_cast<int>(off - __shfl_sync(kFull, inc - u, l));
            break;
          }
          off -= __shfl_sync(kFull, inc, 31);
        }
      }
      if (lane == 0) ctl->start = st;
    }
  }
  __syncthreads();
  *total = ctl->before[p.n];
  *ranges = ranges_of(*total, gridDim.x);
  *fb = range_begin(*total, blockIdx.x, *ranges);
  *fe = range_begin(*total, blockIdx.x + 1, *ranges);
}

// ---------------------------------------------------------------- mass: waits

__device__ __forceinline__ uint64_t drain_limit(uint64_t wait_ns) { return wait_ns > kDrainWaitNs ? wait_ns : kDrainWaitNs; }

__device__ __forceinline__ void fail(Ctl* ctl, uint32_t* err) {
  ctl->abort = 1;
  atomicOr(err, kErrTimeout);
}

// True when every lane's barrier completed and, where that took time, no role had failed: the one
// place where a role learns of a failure, so that a warp's lanes leave together.
__device__ __forceinline__ bool warp_wait(const Ctl* ctl, uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
  if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
  const bool aborted = ctl->abort;
  const bool there = mbar_wait(bar, parity, limit_ns);
  return __all_sync(kFull, there && !aborted);
}

// A place in a ring of N barriers and the parity of its use.
template <int N>
struct Ring {
  int at = 0;
  uint32_t par = 0;
  __device__ __forceinline__ void next() {
    if (++at == N) at = 0, par ^= 1;
  }
};

// ---------------------------------------------------------------- mass: roles

// Keys: the tiles' pages into the ring.  Lane l holds the number of page base + l of the row.
__device__ void key_loop(const MassParams& p, Ctl* ctl, uint8_t* sK, int lane, int64_t units) {
  const uint64_t pol = policy_evict_first();
  const int P = 1 << p.shift, rows = min(P, 64), boxes = kMassTile / rows;
  Ring<kKeySlots> st;
  uint32_t used = 0, last_par = 0;   // last_par: bit s = parity of the last load into slot s
  bool ok = true;
  for (PieceIter c(p, ctl, units); ok && c.valid(); c.next(p, ctl)) {
    if (c.b0 == c.b1) continue;
    const int row = p.rows ? p.rows[c.seq] : p.row0 + c.seq;
    const int32_t* entries = p.table + static_cast<int64_t>(row) * p.max_pages;
    const int held = (c.it.L + P - 1) >> p.shift;
    const int base = c.grp.k0 >> p.shift;   // (a group has 512 keys: 32 pages at most)
    int id = p.n_pages;                     // outside the map: zeros
    if (base + lane < held && lane << p.shift < c.grp.tiles * kMassTile) {
      const int x = entries[base + lane];
      if (x >= 0 && x < p.n_pages) id = x;
      else atomicOr(p.err, kErrRow);
    }
    __syncwarp();
    for (int i = 0; i < c.grp.tiles; ++i) {
      ok = warp_wait(ctl, &ctl->k_empty[st.at], st.par ^ 1, p.wait_ns);
      if (!ok) break;
      const bool leader = elect_one();
      if (leader) mbar_arrive_expect_tx(&ctl->k_full[st.at], kTileBytes);
      for (int b = 0; b < boxes; ++b) {
        const int key = c.grp.k0 + i * kMassTile + b * rows;
        const int page = __shfl_sync(kFull, id, (key >> p.shift) - base);
        if (leader)
          for (int h = 0; h < 2; ++h) {
            uint8_t* dst = sK + st.at * kTileBytes + h * kHalfBytes + b * rows * 128;
            if (p.cut) tma_load_4d(dst, &p.tmk, &ctl->k_full[st.at], h * 64, key & (P - 1), c.g, page);
            else tma_load_4d_hint(dst, &p.tmk, &ctl->k_full[st.at], h * 64, key & (P - 1), c.g, page, pol);
          }
      }
      __syncwarp();
      used |= 1u << st.at;
      last_par = (last_par & ~(1u << st.at)) | (st.par << st.at);
      st.next();
    }
  }
  if (!ok) fail(ctl, p.err);
  // every issued copy completes before the CTA can exit
  for (int i = 0; i < kKeySlots; ++i)
    if (used >> i & 1) mbar_wait(&ctl->k_full[i], last_par >> i & 1, drain_limit(p.wait_ns));
  __syncwarp();
}

// (token, head) pairs of a block: columns c < count, token t0 + c / heads, head h0 + c % heads of the group.
struct Block {
  int t0, h0, count;
  __device__ __forceinline__ Block(const MassParams& p, int n, int b) {
    const int tb = b / p.chunks;
    t0 = tb * p.tpb;
    h0 = (b - tb * p.chunks) * kMassTile;   // (0 unless the heads of a group are more than a block has columns)
    count = min(p.tpb, n - t0) * min(p.heads, p.hg - h0);
  }
  __device__ __forceinline__ int columns() const { return (count + 15) & ~15; }
};

// Queries: blocks into the ring, rows of 128 bytes with the chunks of 16 swizzled as the tensor core reads
// them, zeros behind the last pair.
__device__ void query_loop(const MassParams& p, Ctl* ctl, uint8_t* sQ, int tid, int64_t units) {
  Ring<kQuerySlots> st;
  bool ok = true, there = false;   // there: the blocks of this row and KV head stay
  const int lane = tid & 31, chunk = tid & 15;
  for (PieceIter c(p, ctl, units); ok && c.valid(); c.next(p, ctl)) {
    if (p.cut || !there)
      for (int b = c.b0; ok && b < c.b1; ++b) {
        ok = warp_wait(ctl, &ctl->q_empty[st.at], st.par ^ 1, p.wait_ns);
        if (!ok) break;
        const Block blk(p, c.it.n, b);
        const int heads = min(p.heads, p.hg - blk.h0);
        const __nv_bfloat16* q = p.q + c.seq * p.q_seq + (static_cast<int64_t>(c.g) * p.hg + blk.h0) * p.q_head + chunk * 8;
        uint8_t* dst = sQ + st.at * kTileBytes + (chunk >> 3) * kHalfBytes;
        for (int r0 = tid >> 4; r0 < blk.columns(); r0 += 64) {
          uint4 x[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int r = r0 + 8 * u, t = r / heads;
            x[u] = r < blk.count ? *reinterpret_cast<const uint4*>(q + (blk.t0 + t) * p.q_token + (r - t * heads) * p.q_head)
                                 : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int r = r0 + 8 * u;
            if (r < blk.columns()) *reinterpret_cast<uint4*>(dst + r * 128 + (((chunk & 7) ^ (r & 7)) << 4)) = x[u];
          }
        }
        if (tid < blk.count) {
          const int t = blk.t0 + tid / heads, h = c.g * p.hg + blk.h0 + tid % heads;
          const int64_t at = static_cast<int64_t>(c.seq) * p.T + t;
          Pairs& pr = ctl->pairs[st.at];
          pr.lse[tid] = -1.4426950408889634f * p.lse[at * p.H + h];
          pr.pos[tid] = c.it.L - c.it.n + t;
          if (p.tree) pr.bits[tid] = p.mask[at];
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl->q_full[st.at]);
        st.next();
        there = true;
      }
    if (c.last_of_head(ctl)) there = false;
  }
  if (!ok) fail(ctl, p.err);
}

__device__ void mma_loop(const MassParams& p, Ctl* ctl, const uint8_t* sK, const uint8_t* sQ, uint32_t tmem, int64_t units) {
  const uint64_t dk0 = sdesc_k_sw128(smem_u32(sK)), dq0 = sdesc_k_sw128(smem_u32(sQ));
  Ring<kKeySlots> st;
  Ring<kQuerySlots> q;    // the next block to come
  uint32_t s_par = 0;     // bit a: parity of accumulator a's next use
  bool ok = true;
  int held = 0, first = 0;   // blocks of this row and KV head that stay, and the first one's slot
  for (PieceIter c(p, ctl, units); ok && c.valid(); c.next(p, ctl)) {
    const int nb = c.b1 - c.b0;
    const bool take = p.cut || held == 0;
    if (take) first = q.at;
    Ring<kKeySlots> at = st;
    for (int j = 0; ok && j < nb; ++j) {
      const int slot = (first + j) % kQuerySlots;
      if (take) {
        ok = warp_wait(ctl, &ctl->q_full[q.at], q.par, p.wait_ns);
        q.next();
      }
      const Block blk(p, c.it.n, c.b0 + j);
      const uint32_t idesc = idesc_bf16(kMassTile, blk.columns());
      const uint64_t dq = dq0 + static_cast<uint64_t>(slot * (kTileBytes >> 4));
      at = st;
      for (int i = 0; ok && i < c.grp.tiles; ++i) {
        if (j == 0) ok = warp_wait(ctl, &ctl->k_full[at.at], at.par, p.wait_ns);
        ok = ok && warp_wait(ctl, &ctl->s_empty[at.at], (s_par >> at.at & 1) ^ 1, p.wait_ns);
        if (!ok) break;
        tc_fence_after();
        const uint64_t dk = dk0 + static_cast<uint64_t>(at.at * (kTileBytes >> 4));
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < 8; ++kk) {
            const uint64_t off = (kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2;
            mma_bf16(tmem + at.at * kMassTile, dk + off, dq + off, idesc, kk > 0);
          }
          mma_commit(&ctl->s_full[at.at]);
          if (j == nb - 1) mma_commit(&ctl->k_empty[at.at]);
          if (p.cut && i == c.grp.tiles - 1) mma_commit(&ctl->q_empty[slot]);
        }
        __syncwarp();
        s_par ^= 1u << at.at;
        at.next();
      }
    }
    st = at;
    if (!p.cut) {
      if (take) held = nb;
      if (c.last_of_head(ctl)) {
        if (ok && elect_one())
          for (int j = 0; j < held; ++j) mma_commit(&ctl->q_empty[(first + j) % kQuerySlots]);
        __syncwarp();
        held = 0;
      }
    }
  }
  if (!ok) fail(ctl, p.err);
  // every MMA issued above must be complete before TMEM is released
  if (elect_one()) mma_commit(&ctl->drain);
  mbar_wait(&ctl->drain, 0, drain_limit(p.wait_ns));
  __syncwarp();
}

// Sum of 32 pairs' weights, all of them seen.
__device__ __forceinline__ float weigh32(uint32_t addr, const float* lse, float c2) {
  uint32_t z[32];
  tmem_ld32_async(addr, z);
  tmem_wait32(z);
  const float2 sc = make_float2(c2, c2);
  float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const float4 l = *reinterpret_cast<const float4*>(lse + i);
    const float2 a = ffma2(make_float2(__uint_as_float(z[i]), __uint_as_float(z[i + 1])), sc, make_float2(l.x, l.y));
    const float2 b = ffma2(make_float2(__uint_as_float(z[i + 2]), __uint_as_float(z[i + 3])), sc, make_float2(l.z, l.w));
    acc[0] = fadd2(acc[0], make_float2(ex2_approx(a.x), ex2_approx(a.y)));
    acc[1] = fadd2(acc[1], make_float2(ex2_approx(b.x), ex2_approx(b.y)));
  }
  const float2 s = fadd2(acc[0], acc[1]);
  return s.x + s.y;
}

// Of 16 pairs from column c on, those that see key j.
__device__ __forceinline__ float weigh16(const MassParams& p, uint32_t addr, const Pairs& pr, int c, int count, int j, int ctx, int L) {
  uint32_t z[16];
  tmem_ld16_async(addr + c, z);
  tmem_wait16(z);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    bool seen = c + i < count;   // (behind the last pair: whatever an earlier block left)
    if (seen) {
      if (p.tree) {
        seen = j < ctx || (j < L && (pr.bits[c + i] >> (j - ctx) & 1));
      } else {
        const int pos = pr.pos[c + i];
        seen = j <= pos && (j < p.n_sink || j > pos - p.window);
      }
    }
    const float w = seen ? ex2_approx(fmaf(__uint_as_float(z[i]), p.scale2, pr.lse[c + i])) : 0.f;
    sum += w;
  }
  return sum;
}

// Weighing warpgroup `own`: the tiles whose accumulator it is, a key a thread.
__device__ void weigh_loop(const MassParams& p, Ctl* ctl, uint32_t tmem, int own, int quad, int lane, int64_t units) {
  const int r = quad * 32 + lane;
  const uint32_t addr = tmem + (static_cast<uint32_t>(quad * 32) << 16) + own * kMassTile;
  Ring<kQuerySlots> q;
  int tile = 0;            // number (mod 4) of the next tile to come
  uint32_t par = 0;        // of the accumulator's next use
  bool ok = true;
  int held = 0, slot0 = 0; // blocks of this row and KV head that stay, and the first one's slot
  for (PieceIter c(p, ctl, units); ok && c.valid(); c.next(p, ctl)) {
    const int nb = c.b1 - c.b0;
    const bool take = p.cut || held == 0;
    if (take) slot0 = q.at;
    const int i = (own - (nb > 0 ? tile : 0)) & (kKeySlots - 1);   // which of the group's tiles is this one's
    const bool mine = i < c.grp.tiles;
    const int k0 = c.grp.k0 + i * kMassTile, j = k0 + r, ctx = c.it.L - c.it.n;
    const int row = p.rows ? p.rows[c.seq] : p.row0 + c.seq;
    float* mass = p.mass.m + row * p.mass.row_stride + c.g * p.mass.group_stride + j;
    const bool whole = c.whole();
    float sum = 0.f, had = 0.f;
    if (mine && whole && j < ctx) had = *mass;
    for (int b = 0; b < nb; ++b) {
      const int slot = (slot0 + b) % kQuerySlots;
      if (take) {
        ok = warp_wait(ctl, &ctl->q_full[q.at], q.par, p.wait_ns);
        q.next();
      }
      ok = ok && (!mine || warp_wait(ctl, &ctl->s_full[own], par, p.wait_ns));
      if (!ok) break;
      if (mine) {
        tc_fence_after();
        const Block blk(p, c.it.n, c.b0 + b);
        const Pairs& pr = ctl->pairs[slot];
        const int first = ctx + blk.t0, end = ctx + min(blk.t0 + p.tpb, c.it.n) - 1;   // positions of the block's tokens
        const bool all = p.tree ? k0 + kMassTile <= ctx
                                : k0 + kMassTile - 1 <= first && (k0 + kMassTile <= p.n_sink || k0 > end - p.window);
        int col = 0;
        if (all)
          for (; col + 32 <= blk.count; col += 32) sum += weigh32(addr + col, pr.lse + col, p.scale2);
#pragma unroll 1
        for (; col < blk.count; col += 16) sum += weigh16(p, addr, pr, col, blk.count, j, ctx, c.it.L);
        tc_fence_before();
        par ^= 1;
      }
      __syncwarp();
      if (lane == 0) {
        if (mine) mbar_arrive(&ctl->s_empty[own]);
        if (p.cut) mbar_arrive(&ctl->q_empty[slot]);
      }
    }
    if (!ok) break;
    if (!p.cut) {
      if (take) held = nb;
      if (c.last_of_head(ctl)) {
        if (lane == 0)
          for (int b = 0; b < held; ++b) mbar_arrive(&ctl->q_empty[(slot0 + b) % kQuerySlots]);
        held = 0;
      }
    }
    if (mine && whole) {
      if (j < c.it.L) *mass = fmaf(p.decay, had, sum);
    } else if (mine) {
      p.part[(2 * static_cast<int64_t>(blockIdx.x) + (c.b0 == c.grp.lo)) * (kMassSpan * kMassTile) + i * kMassTile + r] = sum;
    }
    if (nb > 0) tile = (tile + c.grp.tiles) & (kKeySlots - 1);
  }
  if (!ok) fail(ctl, p.err);
}

}  // namespace

__global__ void __launch_bounds__(kThreads, 1) k_mass(const __grid_constant__ MassParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem;                            // [slots][2 halves][128 keys][128 B]
  uint8_t* sQ = sK + kKeySlots * kTileBytes;     // [slots][2 halves][128 pairs][128 B]
  Ctl* ctl = reinterpret_cast<Ctl*>(sQ + kQuerySlots * kTileBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kKeySlots; ++i) {
      mbar_init(&ctl->k_full[i], 1);
      mbar_init(&ctl->k_empty[i], 1);
      mbar_init(&ctl->s_full[i], 1);
      mbar_init(&ctl->s_empty[i], 4);
    }
    for (int i = 0; i < kQuerySlots; ++i) {
      mbar_init(&ctl->q_full[i], 4);
      mbar_init(&ctl->q_empty[i], 1 + kMassWarps - kSoftWarp);   // the products and every weighing warp
    }
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&ctl->tmem_base, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch_dependents();
  griddep_wait();
  const uint32_t tmem = ctl->tmem_base;
  int64_t fb, fe, total;
  int ranges;
  plan(p, ctl, reinterpret_cast<uint32_t*>(sQ), &fb, &fe, &total, &ranges);
  const int64_t units = fe - fb;
  if (warp == 0) {
    key_loop(p, ctl, sK, lane, units);
  } else if (warp == 1) {
    mma_loop(p, ctl, sK, sQ, tmem, units);
  } else if (warp >= kSoftWarp) {
    weigh_loop(p, ctl, tmem, (warp - kSoftWarp) >> 2, warp & 3, lane, units);
  } else if (warp >= kQueryWarp) {
    query_loop(p, ctl, sQ, threadIdx.x - 32 * kQueryWarp, units);
  }
  if (threadIdx.x == 0 && p.cut) {   // what the sum of the parts has to know of this range's end
    MassSplit s;
    s.valid = 0;
    for (PieceIter c(p, ctl, units); c.valid(); c.next(p, ctl))
      if (c.b0 == c.grp.lo && c.b1 < c.grp.hi) {
        s.valid = 1;
        s.seq = c.seq;
        s.g = c.g;
        s.k0 = c.grp.k0;
        s.keys = min(c.grp.tiles * kMassTile, c.it.L - c.grp.k0);
        s.last = range_of(fe + (c.grp.hi - c.b1) - 1, total, ranges);
      }
    p.split[blockIdx.x] = s;
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Adds up the parts of the groups that ranges cut, in the order of the ranges: block c has the one that range c began.
__global__ void __launch_bounds__(kMassSpan * kMassTile) k_mass_sum(const __grid_constant__ MassParams p) {
  griddep_launch_dependents();
  griddep_wait();
  const MassSplit s = p.split[blockIdx.x];
  if (!s.valid || static_cast<int>(threadIdx.x) >= s.keys) return;
  const int row = p.rows ? p.rows[s.seq] : p.row0 + s.seq;
  const int n = p.n_tokens ? p.n_tokens[s.seq] : p.T;
  const int L = p.len[row], j = s.k0 + threadIdx.x;
  float* mass = p.mass.m + row * p.mass.row_stride + s.g * p.mass.group_stride + j;
  const float had = j < L - n ? *mass : 0.f;
  float sum = 0.f;
  for (int c = blockIdx.x; c <= s.last; ++c)
    sum += p.part[(2 * static_cast<int64_t>(c) + (c == static_cast<int>(blockIdx.x))) * (kMassSpan * kMassTile) + threadIdx.x];
  *mass = fmaf(p.decay, had, sum);
}

namespace {

constexpr size_t kSmemBytes = 1024 + static_cast<size_t>(kKeySlots + kQuerySlots) * kTileBytes + sizeof(Ctl);
static_assert(kSmemBytes <= 227 * 1024, "the rings and the control block fit an SM");
static_assert(kMaxTableRows / 4 <= kQuerySlots * kTileBytes, "the rows' bits fit the queries' ring");

}  // namespace

cudaError_t mass_configure() {
  return cudaFuncSetAttribute(k_mass, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes));
}

cudaError_t mass_launch(const MassParams& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.grid), kThreads, stream);
  cfg.dynamicSmemBytes = kSmemBytes;
  return cudaLaunchKernelEx(&cfg, k_mass, p);
}

cudaError_t mass_sum_launch(const MassParams& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.grid), kMassSpan * kMassTile, stream);
  return cudaLaunchKernelEx(&cfg, k_mass_sum, p);
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
