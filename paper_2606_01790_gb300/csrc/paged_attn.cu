// Attention of new tokens over a paged cache.  Query t of sequence s is the token
// at position i = L - n + t of its row (L tokens, n queries) and sees
//   tree:  the keys j < L - n, and the drafted token j = L - n + b where bit b of
//          mask[t] is set;
//   sink:  the keys j <= i with j < n_sink or j > i - window.
//   o[t,h]   = sum_j softmax_j(q[t,h] . K[g(h),j] / sqrt(d)) V[g(h),j]
//   lse[t,h] = log sum_j exp(q[t,h] . K[g(h),j] / sqrt(d))
// over the keys seen; a query that sees none has o = 0 and lse = -inf.
//
// Work split: an item is a block of up to 128 query rows of one sequence, consecutive
// (token, head of the group) pairs.  The flat (item, group, 64-key unit) space, of units
// that some row of the block sees, is cut into one contiguous range per CTA
// (persistent grid).  Lengths are read on the device, so every CTA first adds up the
// items' units.  A run of units of one (item, group) inside a range is a piece; a
// whole one is finished by its CTA, the parts of a cut one (at most the first and the
// last piece of a range) go to slots 2 c and 2 c + 1 of CTA c and k_paged_combine merges
// them.
//
// Per unit on tcgen05 (one thread per query row in the softmax):
//   S = Q K^T   M = 128 rows, N = 64 keys, bf16 -> fp32, A = Q in tensor memory;
//   P           p = exp2(S c - m), l += p in fp32; p = hi + lo, two bf16 (16 bits),
//               in the place of S in tensor memory;
//   O += P V    M = 128, N = d = 128, K = 64 keys, once for hi and once for lo.
// One bf16 part would round each weight by 2^-9, as much as the output's own
// rounding; the second part costs four more products a unit, which the stream of K
// and V covers where a block's rows are few.  (fp16 weights would need V in fp16, which
// holds neither its range nor its small values.)
//
// Even and odd units are two lines with a softmax warpgroup each, which keep a
// reference m, a sum l and an O of their own: nothing passes between them until a
// piece's end, where both read both O and write half of the columns.  With one
// warpgroup for all units the chain S -> registers -> exp2 -> P took 1,900 to 2,100 cycles
// a unit, more than the stream (1,490) and the products (850).  Three S / P places go
// round, so that S of a line's next unit is ready when its last P is written.
//
// Pages come by TMA, a box per page (or 64 of its rows); a page number that is none
// lies outside the map and reads as zeros.  Units that not every row of the block sees
// whole take a masked softmax, whose warpgroup also looks after V: the rows that no
// query sees are zeroed in shared memory (0 times what a free slot holds need not be
// 0).  A V element that is not finite and is seen by some rows of a block only must reach
// those alone, which the product cannot do: it is zeroed as well, and each row that sees
// it adds it at the end (patch_poison).
//
// Warp roles: 0 loads K, 3 loads V, 1 issues S and owns tensor memory, 2 issues P V,
// 4..7 and 8..11 softmax.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "paged_attn.cuh"
#include "ptx.cuh"

namespace starkv {

namespace {

constexpr int kThreads = 384;
constexpr int kStages = 4;                         // depth of the K ring and of the V ring
constexpr int kUnitBytes = kPagedUnitKeys * 256;   // 64 keys x 128 bf16: 16 KB (K or V)
constexpr int kHalfBytes = kPagedUnitKeys * 128;   // one 64-column half of a unit
constexpr int kTmemCols = 512;
constexpr int kSoftWarps = 8;                      // four a line
constexpr uint32_t kFull = 0xffffffffu;
constexpr float kMoveThreshold = 15.f;             // log2 units that a row may rise above its reference
constexpr uint64_t kDrainWaitNs = 2000000000ull;
constexpr uint64_t kAll = ~uint64_t(0);

// Tensor memory, in columns: O 2 x 128, S or P 3 x 64 (P: 32 hi, 32 lo), Q 64.
constexpr int kPlaces = 3;
constexpr uint32_t kColO = 0, kColS = 256, kColQ = 448;

__device__ __forceinline__ uint64_t drain_limit(uint64_t wait_ns) {
  return wait_ns > kDrainWaitNs ? wait_ns : kDrainWaitNs;
}

struct Item {
  int L, n;   // tokens of the row and queries; L = -1: the sequence does not fit, nothing is seen
};

struct Ctl {
  uint64_t k_full[kStages], k_empty[kStages];
  uint64_t v_full[kStages], v_empty[kStages];
  uint64_t s_full[kPlaces], p_full[kPlaces], p_empty[kPlaces];   // S is there; P is; the product that reads P is done
  uint64_t qt_full;                 // a piece's queries are in tensor memory
  uint64_t ml_full;                 // both lines' m and l of a piece are in `ml`
  uint64_t o_empty;                 // a piece's O has been read
  uint64_t drain;
  uint32_t tmem_base;
  volatile int abort;
  volatile int poison[8];           // [piece & 7]: piece + 1 if the piece met such elements
  int warp_sum[kThreads / 32];
  float2 ml[2][2][kPagedRows];      // [piece & 1][line]
  int before[kPagedItems + 1];      // units before an item (one KV group)
  Item item[kPagedItems];
};

// Unit u of a CTA uses place u % 3 and the stages u % kStages for the (u / 3)-th or
// (u / kStages)-th time, which gives the parities of their barriers.
__device__ __forceinline__ int place_of(uint32_t u) { return static_cast<int>(u % kPlaces); }
__device__ __forceinline__ uint32_t place_par(uint32_t u) { return u / kPlaces & 1; }

__device__ __forceinline__ void fail(Ctl* ctl, uint32_t* err) {
  ctl->abort = 1;
  atomicOr(err, kErrTimeout);
}

// A wait of a warp-wide role: true when every lane's barrier completed and no role
// had failed before it.  The one place where these roles learn of a failure, so
// that a warp's lanes leave together (`abort` is read ahead of the wait, where it
// costs nothing).
__device__ __forceinline__ bool warp_wait(const Ctl* ctl, uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
  const bool aborted = ctl->abort;
  return __all_sync(kFull, mbar_wait(bar, parity, limit_ns) && !aborted);
}

// Instruction descriptor of tcgen05.mma kind::f16 with bf16 A (K-major) and bf16 B
// (MN-major), fp32 accumulator, shape M x N.
__host__ __device__ constexpr uint32_t idesc_bf16_bmn(int M, int N) { return idesc_bf16(M, N) | (1u << 16); }

// ---------------------------------------------------------------- what is seen

// Bits b of [0, x)
__device__ __forceinline__ uint64_t below(int x) { return x <= 0 ? 0 : x >= 64 ? kAll : (uint64_t(1) << x) - 1; }

__device__ __forceinline__ uint64_t shifted(uint64_t m, int s) {
  return s >= 64 || s <= -64 ? 0 : s >= 0 ? m << s : m >> -s;
}

// Keys j < first, lo <= j < hi, and drafted tokens ctx + b with bit b of `bits`.
struct Seen {
  int first, lo, hi, ctx;
  uint64_t bits;
  // of the keys k0 .. k0 + 63
  __device__ __forceinline__ uint64_t operator()(int k0) const {
    return below(first - k0) | (below(hi - k0) & ~below(lo - k0)) | (bits ? shifted(bits, ctx - k0) : 0);
  }
};

// One query block: rows row0 .. row0 + nrows - 1 of a sequence's n * hg (token, head) pairs.
struct Block {
  int seq, row0, nrows;
  int tf, tl;          // its first and last token
  int L, n;
  int sinks, win0;     // units of the sinks before the window's first unit; that unit

  __device__ __forceinline__ Block(const PagedAttnParams& p, const Item& it, int item) : L(it.L), n(it.n) {
    seq = item / p.nblk;
    row0 = (item - seq * p.nblk) * kPagedRows;
    nrows = min(kPagedRows, n * p.hg - row0);
    tf = row0 / p.hg;
    tl = (row0 + max(nrows, 1) - 1) / p.hg;
    const int lo = p.tree ? 0 : max(0, first_pos() - p.window + 1), hi = end(p);
    win0 = lo >> 6;
    sinks = p.tree ? 0 : min((min(p.n_sink, hi) + 63) >> 6, win0);
  }
  __device__ __forceinline__ int first_pos() const { return L - n + tf; }
  __device__ __forceinline__ int last_pos() const { return L - n + tl; }
  // keys from here on are seen by none
  __device__ __forceinline__ int end(const PagedAttnParams& p) const { return L < 0 ? 0 : p.tree ? L : last_pos() + 1; }
  // units that some row sees (one where none is left: it gives the empty result); none without queries
  __device__ __forceinline__ int units(const PagedAttnParams& p) const {
    return nrows <= 0 ? 0 : max(1, sinks + ((end(p) + 63) >> 6) - win0);
  }
  __device__ __forceinline__ int key(int unit) const { return (unit < sinks ? unit : win0 + unit - sinks) << 6; }
  // by the query at position i with mask bits `bits`
  __device__ __forceinline__ Seen row(const PagedAttnParams& p, int i, uint64_t bits) const {
    if (L < 0) return Seen{0, 0, 0, 0, 0};
    if (p.tree) return Seen{0, 0, L - n, L - n, bits & below(n)};
    return Seen{min(p.n_sink, i + 1), max(0, i - p.window + 1), i + 1, 0, 0};
  }
  // by every row, without the drafted tokens (which no unit counts as seen by all)
  __device__ __forceinline__ Seen all(const PagedAttnParams& p) const {
    if (L < 0) return Seen{0, 0, 0, 0, 0};
    if (p.tree) return Seen{0, 0, L - n, 0, 0};
    return Seen{min(p.n_sink, first_pos() + 1), max(0, last_pos() - p.window + 1), first_pos() + 1, 0, 0};
  }
  // by some row; `bits`: the union of the block's masks
  __device__ __forceinline__ Seen any(const PagedAttnParams& p, uint64_t bits) const {
    if (L < 0) return Seen{0, 0, 0, 0, 0};
    if (p.tree) return Seen{0, 0, L - n, L - n, bits & below(n)};
    return Seen{min(p.n_sink, last_pos() + 1), max(0, first_pos() - p.window + 1), last_pos() + 1, 0, 0};
  }
};

// Every CTA: the items' lengths and the units before each.
__device__ void count_units(const PagedAttnParams& p, Ctl* ctl) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kPer = (kPagedItems + kThreads - 1) / kThreads;
  int u[kPer];
  int sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int item = tid * kPer + k;
    u[k] = 0;
    if (item >= p.items) continue;
    const int seq = item / p.nblk;
    const int row = p.rows ? p.rows[seq] : p.row0 + seq;
    Item it;
    it.n = p.n_tokens ? p.n_tokens[seq] : p.T;
    it.L = row >= 0 && row < p.n_rows ? p.len[row] : -1;
    if (it.n < 0 || it.n > p.T) {
      it.n = 0;
      atomicOr(p.err, kErrRow);
    } else if (it.L < it.n || it.L > static_cast<int64_t>(p.max_pages) << p.shift) {
      it.L = -1;
      if (it.n) atomicOr(p.err, kErrRow);
    }
    ctl->item[item] = it;
    u[k] = Block(p, it, item).units(p);
    sum += u[k];
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kFull, inc, o);
    if (lane >= o) inc += x;
  }
  if (lane == 31) ctl->warp_sum[warp] = inc;
  __syncthreads();
  int at = inc - sum;
  for (int w = 0; w < warp; ++w) at += ctl->warp_sum[w];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int item = tid * kPer + k;
    if (item <= p.items) ctl->before[item] = at;
    at += u[k];
  }
  __syncthreads();
}

__device__ __forceinline__ int64_t range_begin(int64_t T, int c, int P) { return T * c / P; }

// CTA whose range holds flat unit f
__device__ __forceinline__ int cta_of(int64_t f, int64_t T, int P) { return static_cast<int>(((f + 1) * P - 1) / T); }

// The pieces of a CTA's flat range [f0, f1), in order: a run of n units j0, j0 + 1,
// ... of the nu units of one (item, group).
struct PieceIter {
  int item, g, j0, n, nu;
  int64_t rem;   // units of the range from this piece on
  __device__ __forceinline__ PieceIter(const PagedAttnParams& p, const Ctl* ctl, int64_t f0, int64_t f1)
      : item(0), g(0), j0(0), n(0), nu(0), rem(f1 - f0) {
    if (rem <= 0) return;
    int hi = p.items;   // the last item with no more than f0 units before it (items without units are passed over)
    while (hi - item > 1) {
      const int mid = (item + hi) >> 1;
      if (static_cast<int64_t>(ctl->before[mid]) * p.G <= f0) item = mid;
      else hi = mid;
    }
    nu = ctl->before[item + 1] - ctl->before[item];
    const int64_t u = f0 - static_cast<int64_t>(ctl->before[item]) * p.G;
    g = static_cast<int>(u / nu);
    j0 = static_cast<int>(u - static_cast<int64_t>(g) * nu);
    n = static_cast<int>(min(rem, static_cast<int64_t>(nu - j0)));
  }
  __device__ __forceinline__ bool valid() const { return rem > 0; }
  __device__ __forceinline__ bool whole() const { return n == nu; }
  __device__ __forceinline__ void next(const PagedAttnParams& p, const Ctl* ctl) {
    rem -= n;
    j0 = 0;
    if (rem <= 0) return;
    if (++g == p.G) {
      g = 0;
      do {
        ++item;
        nu = ctl->before[item + 1] - ctl->before[item];
      } while (nu == 0);
    }
    n = static_cast<int>(min(rem, static_cast<int64_t>(nu)));
  }
};

// ---------------------------------------------------------------- loaders

// K or V loader: the units' pages into a ring.  Lane l holds the number of page
// base + l of the row, so that the table is read once in 32 pages.
__device__ void load_loop(const PagedAttnParams& p, Ctl* ctl, const CUtensorMap* map, uint8_t* ring, uint64_t* full,
                          uint64_t* empty, int lane, int64_t fb, int64_t fe) {
  const uint64_t pol = policy_evict_first();   // a single query block reads K and V once
  const bool once = p.nblk == 1;
  const int P = 1 << p.shift;
  const int boxes = P < kPagedUnitKeys ? kPagedUnitKeys >> p.shift : 1;
  const int box_bytes = min(P, kPagedUnitKeys) * 128;
  int stage = 0;
  uint32_t phase = 0, used = 0, last_ph = 0;   // last_ph: bit s = phase of the last load into stage s
  bool ok = true;
  for (PieceIter c(p, ctl, fb, fe); ok && c.valid(); c.next(p, ctl)) {
    const Item it = ctl->item[c.item];
    const Block blk(p, it, c.item);
    const int row = p.rows ? p.rows[blk.seq] : p.row0 + blk.seq;
    const int32_t* entries = p.table + static_cast<int64_t>(row) * p.max_pages;
    const int held = it.L < 0 ? 0 : (it.L + P - 1) >> p.shift;
    int base = 0, have = 0, id = 0;
    for (int j = c.j0; ok && j < c.j0 + c.n; ++j) {
      const int k0 = blk.key(j), page0 = k0 >> p.shift;
      if (page0 < base || page0 + boxes > base + have) {
        base = page0;
        have = 32;
        id = p.n_pages;   // outside the map: zeros
        if (base + lane < held) {
          const int x = entries[base + lane];
          if (x >= 0 && x < p.n_pages) id = x;
          else atomicOr(p.err, kErrRow);
        }
        __syncwarp();
      }
      ok = warp_wait(ctl, &empty[stage], phase ^ 1, p.wait_ns);
      if (!ok) break;
      const bool leader = elect_one();
      if (leader) mbar_arrive_expect_tx(&full[stage], kUnitBytes);
      for (int b = 0; b < boxes; ++b) {
        const int page = __shfl_sync(kFull, id, page0 + b - base);
        if (leader)
          for (int h = 0; h < 2; ++h) {
            uint8_t* dst = ring + stage * kUnitBytes + h * kHalfBytes + b * box_bytes;
            const int slot = P < kPagedUnitKeys ? 0 : k0 & (P - 1);
            if (once) tma_load_4d_hint(dst, map, &full[stage], h * 64, slot, c.g, page, pol);
            else tma_load_4d(dst, map, &full[stage], h * 64, slot, c.g, page);
          }
      }
      __syncwarp();
      used |= 1u << stage;
      last_ph = (last_ph & ~(1u << stage)) | (phase << stage);
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1;
      }
    }
  }
  if (!ok) fail(ctl, p.err);
  // every issued copy completes before the CTA can exit
  for (int i = 0; i < kStages; ++i)
    if (used >> i & 1) mbar_wait(&full[i], last_ph >> i & 1, drain_limit(p.wait_ns));
  __syncwarp();
}

// ---------------------------------------------------------------- MMA issuers

__device__ void mma_s_loop(const PagedAttnParams& p, Ctl* ctl, const uint8_t* sK, uint32_t tmem, int64_t fb, int64_t fe) {
  const uint32_t idesc = idesc_bf16(kPagedRows, kPagedUnitKeys);
  const uint64_t dk0 = sdesc_k_sw128(smem_u32(sK));
  int pc = 0;
  uint32_t ui = 0;
  bool ok = true;
  for (PieceIter c(p, ctl, fb, fe); ok && c.valid(); c.next(p, ctl)) {
    ok = warp_wait(ctl, &ctl->qt_full, pc & 1, p.wait_ns);
    ++pc;
    for (int i = 0; ok && i < c.n; ++i, ++ui) {
      const int stage = ui % kStages, pl = place_of(ui);
      ok = warp_wait(ctl, &ctl->k_full[stage], ui / kStages & 1, p.wait_ns) &&
           warp_wait(ctl, &ctl->p_empty[pl], place_par(ui) ^ 1, p.wait_ns);   // the place's previous P has been used
      if (!ok) break;
      tc_fence_after();
      const uint64_t dk = dk0 + static_cast<uint64_t>(stage * (kUnitBytes >> 4));
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          mma_f16_ts(tmem + kColS + 64 * pl, tmem + kColQ + kk * 8, dk + ((kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2), idesc, kk > 0);
        mma_commit(&ctl->s_full[pl]);
        mma_commit(&ctl->k_empty[stage]);
      }
      __syncwarp();
    }
  }
  if (!ok) fail(ctl, p.err);
  // every MMA issued above must be complete before TMEM is released
  if (elect_one()) mma_commit(&ctl->drain);
  mbar_wait(&ctl->drain, 0, drain_limit(p.wait_ns));
  __syncwarp();
}

__device__ void mma_pv_loop(const PagedAttnParams& p, Ctl* ctl, const uint8_t* sV, uint32_t tmem, int64_t fb, int64_t fe) {
  const uint32_t idesc = idesc_bf16_bmn(kPagedRows, kHeadDim);
  const uint64_t dv0 = sdesc_mn_sw128(smem_u32(sV), kHalfBytes, 1024);
  int pc = 0;
  uint32_t ui = 0;
  bool ok = true;
  for (PieceIter c(p, ctl, fb, fe); ok && c.valid(); c.next(p, ctl)) {
    ok = warp_wait(ctl, &ctl->o_empty, (pc & 1) ^ 1, p.wait_ns);   // both O of the previous piece have been read
    ++pc;
    for (int i = 0; ok && i < c.n; ++i, ++ui) {
      const int stage = ui % kStages, pl = place_of(ui);
      ok = warp_wait(ctl, &ctl->v_full[stage], ui / kStages & 1, p.wait_ns) &&
           warp_wait(ctl, &ctl->p_full[pl], place_par(ui), p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      const uint64_t dv = dv0 + static_cast<uint64_t>(stage * (kUnitBytes >> 4));
      if (elect_one()) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)   // 16 keys per step: 8 columns of P, 16 rows of V; a line's first product of a piece overwrites O
            mma_f16_ts(tmem + kColO + kHeadDim * (ui & 1), tmem + kColS + 64 * pl + 32 * part + kk * 8,
                       dv + static_cast<uint64_t>(kk * 128), idesc, (i > 1 || part > 0 || kk > 0) ? 1u : 0u);
        mma_commit(&ctl->p_empty[pl]);
        mma_commit(&ctl->v_empty[stage]);
      }
      __syncwarp();
    }
  }
  if (!ok) fail(ctl, p.err);
  if (elect_one()) mma_commit(&ctl->drain);
  mbar_wait(&ctl->drain, 0, drain_limit(p.wait_ns));
  __syncwarp();
}

// ---------------------------------------------------------------- softmax

// 32 keys of a unit, exp2 arguments and sums as packed pairs; p = hi + lo, hi the
// upper 16 bits of p.  Masked keys (bits of `vis` clear) have p = 0.
template <bool FULL>
__device__ __forceinline__ void exp_split(const uint32_t (&z0)[16], const uint32_t (&z1)[16], uint32_t vis, float2 sc2, float2 nm2,
                                          float2 (&acc)[4], uint32_t (&hi)[16], uint32_t (&lo)[16]) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const uint32_t a = i < 16 ? z0[i & 15] : z1[i & 15], b = i < 16 ? z0[(i + 1) & 15] : z1[(i + 1) & 15];
    const float2 e = ffma2(make_float2(__uint_as_float(a), __uint_as_float(b)), sc2, nm2);
    const float p0 = FULL || (vis >> i & 1) ? ex2_approx(e.x) : 0.f;
    const float p1 = FULL || (vis >> (i + 1) & 1) ? ex2_approx(e.y) : 0.f;
    acc[(i >> 1) & 3] = fadd2(acc[(i >> 1) & 3], make_float2(p0, p1));
    const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
    hi[i >> 1] = __byte_perm(u0, u1, 0x7632);
    const float2 rest = fadd2(make_float2(p0, p1), make_float2(-__uint_as_float(u0 & 0xFFFF0000u), -__uint_as_float(u1 & 0xFFFF0000u)));
    const __nv_bfloat162 r = __floats2bfloat162_rn(rest.x, rest.y);
    lo[i >> 1] = *reinterpret_cast<const uint32_t*>(&r);
  }
}

template <bool FULL>
__device__ __forceinline__ float unit_max(const uint32_t (&z)[4][16], uint64_t vis) {
  float pm[8];   // independent partial maxima
#pragma unroll
  for (int k = 0; k < 8; ++k) pm[k] = -INFINITY;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t bits = static_cast<uint32_t>(vis >> (16 * q));
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (FULL || (bits >> i & 1)) pm[i & 7] = fmaxf(pm[i & 7], __uint_as_float(z[q][i]));
  }
  return fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), fmaxf(fmaxf(pm[4], pm[5]), fmaxf(pm[6], pm[7])));
}

// Rescales this warp's O rows by alpha (1 in lanes whose reference stays).
__device__ __forceinline__ void rescale_o(uint32_t o_addr, float alpha) {
#pragma unroll 1
  for (int ch = 0; ch < kHeadDim / 16; ++ch) {
    uint32_t o[16];
    tmem_ld16_async(o_addr + ch * 16, o);
    tmem_wait16(o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
    tmem_st16(o_addr + ch * 16, o);
  }
}

// One unit of a softmax warp with rows: S into registers, P in its place.  A row's
// reference m starts at its first maximum (its O is 0 until then) and moves only when a
// later maximum lies more than 15 above it; the move rescales its O row once the product
// of the line's previous unit is done.  Returns false when a wait ran out.
template <bool FULL>
__device__ __forceinline__ bool softmax_unit(const PagedAttnParams& p, Ctl* ctl, uint64_t vis, uint32_t s_addr, uint32_t o_addr,
                                             uint32_t ui, float& m, float& l) {
  const float c2 = p.scale2;
  uint32_t z[4][16];
#pragma unroll
  for (int q = 0; q < 4; ++q) tmem_ld16_async(s_addr + q * 16, z[q]);
#pragma unroll
  for (int q = 0; q < 4; ++q) tmem_wait16(z[q]);
  const float mx = unit_max<FULL>(z, vis) * c2;
  const bool first = m == -INFINITY;
  const bool move = !first && mx > m + kMoveThreshold;
  if (__any_sync(kFull, move)) {   // rare
    const float alpha = move ? ex2_approx(m - mx) : 1.f;
    const uint32_t up = ui - 2;
    if (!warp_wait(ctl, &ctl->p_empty[place_of(up)], place_par(up), p.wait_ns)) return false;
    tc_fence_after();
    rescale_o(o_addr, alpha);
    l *= alpha;
  }
  if (first || move) m = mx;
  const float ref = m == -INFINITY ? 0.f : m;
  const float2 sc2 = make_float2(c2, c2), nm2 = make_float2(-ref, -ref);
  float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t hi[16], lo[16];
    exp_split<FULL>(z[2 * k], z[2 * k + 1], static_cast<uint32_t>(vis >> (32 * k)), sc2, nm2, acc, hi, lo);
    tmem_st16(s_addr + 16 * k, hi);
    tmem_st16(s_addr + 32 + 16 * k, lo);
  }
  const float2 a = fadd2(fadd2(acc[0], acc[1]), fadd2(acc[2], acc[3]));
  l += a.x + a.y;
  return true;
}

__device__ __forceinline__ bool not_finite(uint32_t bf16_bits) { return (bf16_bits & 0x7F80u) == 0x7F80u; }

// Adds to 16 columns of a row's O what its product left out: the elements of V that
// are not finite, at the keys it sees in the piece's masked units.  (Their weight is
// taken as positive: one that has underflowed to 0 gives the infinity and not a NaN.)
__device__ __noinline__ void patch_poison(const PagedAttnParams& p, const Block& blk, const Seen& see, int g, int j0, int n, int col,
                                          float (&o)[16]) {
  const Seen all = blk.all(p);
  const int row = p.rows ? p.rows[blk.seq] : p.row0 + blk.seq;
  const int32_t* entries = p.table + static_cast<int64_t>(row) * p.max_pages;
  for (int j = j0; j < j0 + n; ++j) {
    const int k0 = blk.key(j);
    if (all(k0) == kAll) continue;
    for (uint64_t bits = see(k0); bits; bits &= bits - 1) {
      const int key = k0 + __ffsll(static_cast<long long>(bits)) - 1;
      const int page = entries[key >> p.shift];
      if (page < 0 || page >= p.n_pages) continue;
      const __nv_bfloat16* v = p.v + page * p.page_stride +
                               ((static_cast<int64_t>(g) << p.shift) + (key & ((1 << p.shift) - 1))) * kHeadDim + col;
      for (int i = 0; i < 16; ++i) {
        const uint32_t b = *reinterpret_cast<const uint16_t*>(v + i);
        if (not_finite(b)) o[i] += __uint_as_float(b << 16);
      }
    }
  }
}

// V of a unit that not every row sees whole (by the 128 threads of its line): rows that
// no query sees (bits of `seen` clear) and elements that are not finite become zeros.
// Returns whether this thread met one of the latter.
__device__ __forceinline__ bool clean_v(uint4* v4, uint64_t seen, int thread) {
  bool met = false;
#pragma unroll 1
  for (int x = thread; x < kUnitBytes / 16; x += 128) {
    if (!(seen >> (x >> 3 & 63) & 1)) {   // 8 chunks of 16 bytes a key and half
      v4[x] = make_uint4(0u, 0u, 0u, 0u);
      continue;
    }
    const uint4 w = v4[x];
    uint32_t e[4] = {w.x, w.y, w.z, w.w};
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (not_finite(e[k])) e[k] &= 0xFFFF0000u, bad = true;
      if (not_finite(e[k] >> 16)) e[k] &= 0xFFFFu, bad = true;
    }
    if (bad) {
      v4[x] = make_uint4(e[0], e[1], e[2], e[3]);
      met = true;
    }
  }
  fence_proxy_async_smem();
  return met;
}

// Softmax warps of a line (0: even units, 1: odd): one thread per query row (TMEM lane
// quad * 32 + lane).
__device__ void softmax_loop(const PagedAttnParams& p, Ctl* ctl, uint8_t* sV, uint32_t tmem, uint32_t line, int quad, int lane,
                             int64_t fb, int64_t fe) {
  const int r = quad * 32 + lane;
  const uint32_t lane_base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
  const uint32_t o_addr = lane_base + kColO + kHeadDim * line;
  uint32_t u0 = 0;   // number of the piece's first unit
  // line 0: the queries of a piece (no product reads the previous piece's any more)
  auto take_queries = [&](const PieceIter& c) {
    const Block blk(p, ctl->item[c.item], c.item);
    if (quad * 32 < blk.nrows) {
      const bool live = r < blk.nrows;
      const int t = (blk.row0 + r) / p.hg, h = c.g * p.hg + (blk.row0 + r) % p.hg;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + blk.seq * p.q_seq + t * p.q_token + h * p.q_head);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 x = live ? src[4 * k + i] : make_uint4(0u, 0u, 0u, 0u);
          w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
        }
        __syncwarp();   // (`live` differs between lanes)
        tmem_st16(lane_base + kColQ + 16 * k, w);
      }
      tmem_wait_st();
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl->qt_full);
  };
  bool ok = true;
  int pc = 0;
  PieceIter c(p, ctl, fb, fe);
  if (line == 0 && c.valid()) take_queries(c);
  for (; ok && c.valid(); ++pc) {
    const Block blk(p, ctl->item[c.item], c.item);
    const bool wactive = quad * 32 < blk.nrows;
    const bool live = r < blk.nrows;
    const int t = (blk.row0 + r) / p.hg, h = c.g * p.hg + (blk.row0 + r) % p.hg;
    const Seen all = blk.all(p);
    const uint64_t* masks = p.mask + static_cast<int64_t>(blk.seq) * p.T;
    Seen see = blk.row(p, blk.L - blk.n + t, p.tree && live ? masks[t] : 0);
    if (!live) see = Seen{0, 0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    for (uint32_t ui = u0 + ((u0 ^ line) & 1); ui < u0 + c.n; ui += 2) {
      const int pl = place_of(ui);
      const uint32_t s_addr = lane_base + kColS + 64 * pl;
      ok = warp_wait(ctl, &ctl->s_full[pl], place_par(ui), p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      const int k0 = blk.key(c.j0 + static_cast<int>(ui - u0));
      if (all(k0) == kAll) {
        if (wactive) ok = softmax_unit<true>(p, ctl, kAll, s_addr, o_addr, ui, m, l);
      } else {
        if (wactive) ok = softmax_unit<false>(p, ctl, see(k0), s_addr, o_addr, ui, m, l);
        if (!ok) break;
        uint64_t bits = 0;
        if (p.tree) {   // the union of the block's masks (at most 64 tokens)
          for (int x = blk.tf + lane; x <= blk.tl && x < blk.n; x += 32) bits |= masks[x];
          bits = static_cast<uint64_t>(__reduce_or_sync(kFull, static_cast<uint32_t>(bits >> 32))) << 32 |
                 __reduce_or_sync(kFull, static_cast<uint32_t>(bits));
        }
        const int stage = ui % kStages;
        ok = warp_wait(ctl, &ctl->v_full[stage], ui / kStages & 1, p.wait_ns);
        if (!ok) break;
        if (clean_v(reinterpret_cast<uint4*>(sV + stage * kUnitBytes), blk.any(p, bits)(k0), r)) ctl->poison[pc & 7] = pc + 1;
      }
      if (!ok) break;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl->p_full[pl]);
    }
    if (!ok) break;
    const uint32_t lu = u0 + c.n - 1;
    PieceIter nx = c;
    nx.next(p, ctl);
    if (line == 0 && nx.valid()) {   // S of the next piece runs under this piece's end
      ok = warp_wait(ctl, &ctl->s_full[place_of(lu)], place_par(lu), p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      take_queries(nx);
    }
    // both lines' references and sums, and both O
    ctl->ml[pc & 1][line][r] = make_float2(m, l);
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl->ml_full);
    ok = warp_wait(ctl, &ctl->ml_full, pc & 1, p.wait_ns) && warp_wait(ctl, &ctl->p_empty[place_of(lu)], place_par(lu), p.wait_ns);
    if (!ok) break;
    tc_fence_after();
    if (wactive) {
      const bool whole = c.whole();
      const bool two = c.n > 1;   // (a line without units has no O)
      const float2 other = ctl->ml[pc & 1][line ^ 1][r];
      const float M = fmaxf(m, other.x), ref = M == -INFINITY ? 0.f : M;
      const float w_own = exp2f(m - ref), w_other = exp2f(other.x - ref);
      const float L = w_own * l + w_other * other.y;
      const float norm = !whole ? 1.f : L == 0.f ? 0.f : 1.f / L;
      const float w0 = (line ? w_other : w_own) * norm, w1 = (line ? w_own : w_other) * norm;
      const uint32_t first = lane_base + kColO + kHeadDim * (two ? 0 : u0 & 1);
      const float wf = two || !(u0 & 1) ? w0 : w1;
      const bool poison = ctl->poison[pc & 7] == pc + 1;
      const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (c.j0 == 0);
      __nv_bfloat16* out = p.o + blk.seq * p.o_seq + t * p.o_token + h * p.o_head;
      float* part = p.part_o + (slot * kPagedRows + r) * kHeadDim;
#pragma unroll 1
      for (int ch = 4 * line; ch < 4 * static_cast<int>(line) + 4; ++ch) {
        uint32_t a[16], b[16];
        tmem_ld16_async(first + ch * 16, a);
        if (two) tmem_ld16_async(lane_base + kColO + kHeadDim + ch * 16, b);
        tmem_wait16(a);
        float o[16];
        if (two) {
          tmem_wait16(b);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(a[i]) * wf + __uint_as_float(b[i]) * w1;
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(a[i]) * wf;
        }
        if (live) {
          if (poison) {
            float x[16];   // (a copy: the address of o would keep it out of registers)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = o[i];
            patch_poison(p, blk, see, c.g, c.j0, c.n, ch * 16, x);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = x[i];
          }
          if (whole) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const __nv_bfloat162 x = __floats2bfloat162_rn(o[2 * i], o[2 * i + 1]);
              w[i] = *reinterpret_cast<const uint32_t*>(&x);
            }
            reinterpret_cast<uint4*>(out + ch * 16)[0] = make_uint4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<uint4*>(out + ch * 16)[1] = make_uint4(w[4], w[5], w[6], w[7]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              reinterpret_cast<float4*>(part + ch * 16)[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          }
        }
        __syncwarp();
      }
      if (live && line == 0) {
        if (!whole) p.part_ml[slot * kPagedRows + r] = make_float2(M, L);
        else if (p.lse)
          p.lse[(static_cast<int64_t>(blk.seq) * p.T + t) * p.H + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
      }
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl->o_empty);
    u0 += c.n;
    c = nx;
  }
  if (!ok) fail(ctl, p.err);
}

}  // namespace

__global__ void __launch_bounds__(kThreads, 1) k_paged_attn(const __grid_constant__ PagedAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem;                           // [kStages][2 halves][64 keys][128 B]
  uint8_t* sV = sK + kStages * kUnitBytes;      // the same
  Ctl* ctl = reinterpret_cast<Ctl*>(sV + kStages * kUnitBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&ctl->k_full[i], 1);
      mbar_init(&ctl->k_empty[i], 1);
      mbar_init(&ctl->v_full[i], 1);
      mbar_init(&ctl->v_empty[i], 1);
    }
    for (int i = 0; i < kPlaces; ++i) {
      mbar_init(&ctl->s_full[i], 1);
      mbar_init(&ctl->p_full[i], kSoftWarps / 2);
      mbar_init(&ctl->p_empty[i], 1);
    }
    mbar_init(&ctl->qt_full, kSoftWarps / 2);
    mbar_init(&ctl->ml_full, kSoftWarps);
    mbar_init(&ctl->o_empty, kSoftWarps);
    mbar_init(&ctl->drain, 2);   // one commit per MMA issuer
    ctl->abort = 0;
    for (int i = 0; i < 8; ++i) ctl->poison[i] = 0;
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
  count_units(p, ctl);
  const int64_t T = static_cast<int64_t>(ctl->before[p.items]) * p.G;
  const int64_t fb = range_begin(T, blockIdx.x, gridDim.x);
  const int64_t fe = range_begin(T, blockIdx.x + 1, gridDim.x);

  if (warp == 0) {
    load_loop(p, ctl, &p.tmk, sK, ctl->k_full, ctl->k_empty, lane, fb, fe);
  } else if (warp == 3) {
    load_loop(p, ctl, &p.tmv, sV, ctl->v_full, ctl->v_empty, lane, fb, fe);
  } else if (warp == 1) {
    mma_s_loop(p, ctl, sK, tmem, fb, fe);
  } else if (warp == 2) {
    mma_pv_loop(p, ctl, sV, tmem, fb, fe);
  } else {
    softmax_loop(p, ctl, sV, tmem, (warp - 4) >> 2, warp & 3, lane, fb, fe);
  }
  if (threadIdx.x == 0) {   // what the merge has to know of this range's end
    PagedSplit s;
    s.total = T;
    s.valid = 0;
    if (fe > fb) {   // the piece that the range's last unit is in, if it begins here and goes on
      const PieceIter e(p, ctl, fe - 1, fe);
      const int64_t f0 = static_cast<int64_t>(ctl->before[e.item]) * p.G + static_cast<int64_t>(e.g) * e.nu;
      if (f0 >= fb && f0 + e.nu > fe) {
        s.valid = 1;
        s.item = e.item;
        s.g = e.g;
        s.c1 = cta_of(f0 + e.nu - 1, T, gridDim.x);
      }
    }
    p.split[blockIdx.x] = s;
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Merges the parts of the (item, group)s that ranges cut: M = max m, L = sum 2^(m - M)
// l, O = sum 2^(m - M) O_part / L, lse = (M + log2 L) ln 2.  Block (c, y): the one that
// CTA c began, query rows 8 y and on, a warp per row; the loads of eight parts are in
// flight before the first is used (one after the other, 40 parts took 75 us).
constexpr int kBatch = 8;

__global__ void __launch_bounds__(256) k_paged_combine(const __grid_constant__ PagedAttnParams p) {
  griddep_launch_dependents();
  griddep_wait();
  const int c0 = blockIdx.x;
  const PagedSplit s = p.split[c0];
  if (!s.valid) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int seq = s.item / p.nblk, row0 = (s.item - seq * p.nblk) * kPagedRows;
  const int n = p.n_tokens ? p.n_tokens[seq] : p.T;
  const int r = blockIdx.y * 8 + warp;
  if (r >= min(kPagedRows, n * p.hg - row0)) return;
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int cb = c0; cb <= s.c1; cb += kBatch) {
    float2 ml[kBatch];
    float4 o[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int c = cb + k;
      ml[k] = make_float2(-INFINITY, 0.f);
      o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c > s.c1 || range_begin(s.total, c, p.grid) == range_begin(s.total, c + 1, p.grid)) continue;   // (a CTA without units)
      const int64_t at = (2 * static_cast<int64_t>(c) + (c == c0)) * kPagedRows + r;
      ml[k] = p.part_ml[at];
      o[k] = reinterpret_cast<const float4*>(p.part_o + at * kHeadDim)[lane];
    }
    float top = M;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = fmaxf(top, ml[k].x);
    const float ref = top == -INFINITY ? 0.f : top, keep = exp2f(M - ref);
    M = top;
    L *= keep;
    acc = make_float4(acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float w = exp2f(ml[k].x - ref);
      L += w * ml[k].y;
      acc = make_float4(acc.x + w * o[k].x, acc.y + w * o[k].y, acc.z + w * o[k].z, acc.w + w * o[k].w);
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int t = (row0 + r) / p.hg, h = s.g * p.hg + (row0 + r) % p.hg;
  const __nv_bfloat162 x[2] = {__floats2bfloat162_rn(acc.x * inv, acc.y * inv), __floats2bfloat162_rn(acc.z * inv, acc.w * inv)};
  *reinterpret_cast<uint2*>(p.o + seq * p.o_seq + t * p.o_token + h * p.o_head + lane * 4) = *reinterpret_cast<const uint2*>(x);
  if (p.lse && lane == 0)
    p.lse[(static_cast<int64_t>(seq) * p.T + t) * p.H + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

namespace {

constexpr size_t kSmemBytes = 1024 + 2 * static_cast<size_t>(kStages) * kUnitBytes + sizeof(Ctl);
static_assert(kSmemBytes <= 227 * 1024, "the rings and the control block fit an SM");

cudaLaunchConfig_t config(cudaLaunchAttribute* attr, dim3 grid, int threads, size_t smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // set-up under the previous kernel's tail
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.stream = stream;
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  return cfg;
}

}  // namespace

cudaError_t paged_attn_configure() {
  return cudaFuncSetAttribute(k_paged_attn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemBytes));
}

cudaError_t paged_attn_launch(const PagedAttnParams& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.grid), kThreads, kSmemBytes, stream);
  return cudaLaunchKernelEx(&cfg, k_paged_attn, p);
}

cudaError_t paged_combine_launch(const PagedAttnParams& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.grid, (std::min(kPagedRows, p.T * p.hg) + 7) / 8), 256, 0, stream);
  return cudaLaunchKernelEx(&cfg, k_paged_combine, p);
}

}  // namespace starkv
