// Attention mass of cached tokens, and the choice of those that stay by it.
//
// Mass: token j of a row, KV head g, after a call whose queries (the row's last n tokens)
// have normalisers lse:
//   mass_j = (j < L - n ? decay mass_j : 0) + sum_t sum_{h in g} [t sees j] exp(q_th . k_j / sqrt(d) - lse_th).
//
// Keys lie on the lanes of tensor memory and (token, head) pairs in its columns, so that a key's sum is a thread's own, no
// sum crosses lanes, and a key that holds NaN or garbage touches nothing but its own.  A tile of 128 keys (A) meets blocks of up
// to 128 pairs (B), nine K = 16 steps: eight of q . k, and one of three ones against -lse sqrt(d) in three bf16 parts (24 bits),
// after which a weight is exp2 of the accumulator times one constant: no normaliser has to be fetched for each
// element (from shared memory they took as much of its path as the accumulators: a chunk, see below, 112 us for 99).
//
// Work split.  A group is one tile or four (512 keys) of one row and KV head.  Where a call has one or two blocks of queries
// they stay in shared memory while a row's keys pass once; groups go whole to contiguous ranges, one a CTA (persistent
// grid), and are written by their CTA.  Where it has more, a group's keys stay and the blocks that see them pass; (group, block)
// units are cut into ranges, and the parts of a group that is cut (at most the first and the last of a range) are added up by
// k_mass_sum in the order of the ranges: no atomics, the same sums every time.
//
// What bounds it.  Few queries: the stream of K (64 rows of one token over 14k ragged keys, 8 KV heads: 1.2 GB in 176 to 184 us,
// the copy rate).  13 to 26 drafted tokens of 32 rows: 57 us for a stream of 45, beside the weighing (its exponentials, of which
// an SM takes 32 a clock, 17).  Many: the products' operands (8 KB a step, 90 to 97 cycles at what shared memory delivers, where
// the tensor core takes 64), and the weighing between them, since a tile has one accumulator, which its next products wait
// for.  A chunk of 2,704 tokens under a window of 4,096, 81 GFLOP: 97 us, tensor pipe 54 % busy (at 99 us: without the weighing 67,
// with everything in it but the exponentials 93).  Not kept: exponentials in part as polynomials on the FMA pipe (an eighth of them
// 104, a quarter 109); one key loader (246 for 205 us in the first case) and one issuer of products (205 for 183); groups of a tile
// each (183 for 176); two weighing warpgroups (63 for 59 in the second case, 112 for 99 in the chunk, 175 for 176 in the first);
// a look through the ring for the queries' next slot before their last block is handed over (230 for 218 in an earlier state of
// the chunk, since asking a barrier may wait); weights unrolled over a block (212 for 162).
//
// Warp roles: 0 and 1 load keys, 2 and 3 issue products, 4 to 7 copy queries, the others weigh.
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

constexpr int kKeySlots = 4, kQuerySlots = 2;     // rings; a tile of keys has an accumulator and a weighing warpgroup of its own
constexpr int kMmaWarp = 2, kQueryWarp = 4, kSoftWarp = 8;   // (0 and 1: keys; 2 issuers; 4 query warps; the weighing warps)
constexpr int kWarps = kSoftWarp + 4 * kKeySlots, kThreads = 32 * kWarps;
constexpr int kQueryThreads = 32 * (kSoftWarp - kQueryWarp);
static_assert(kQueryThreads / 16 == kMassQueryStep && kQueryThreads >= kMassTile, "16 threads take a row of 256 bytes");
constexpr int kTileBytes = kMassTile * 256;       // 128 keys x 128 bf16, or as many (token, head) pairs: 32 KB
constexpr int kHalfBytes = kTileBytes / 2;
constexpr int kExtraBytes = kMassTile * 32;       // 128 rows of 16 more elements: the step of the products that takes lse off
constexpr int kOneBytes = 256;
constexpr float kRootDim = 11.313708498984761f;   // sqrt(d)
constexpr int kTmemCols = 512;
constexpr int kTileShift = 7, kSpanShift = 2;
static_assert(kMassTile == 1 << kTileShift && kMassSpan == 1 << kSpanShift, "");
constexpr uint64_t kDrainWaitNs = 2000000000ull;

struct Item {
  int L, n;     // tokens of the row and queries; n = 0: nothing to do
  int row;
  int blocks;   // of its queries
};

// x / n by its reciprocal ceil(2^32 / n) (0 for n = 1), for x n < 2^32
__device__ __forceinline__ int quotient(int x, uint32_t inv) {
  return inv ? static_cast<int>(__umulhi(static_cast<uint32_t>(x), inv)) : x;
}

// An item in 64 bits: a length of 25, a count of 18, a row of 16 (n > 0 only where they fit the call).
__device__ __forceinline__ uint64_t packed(int L, int n, int row) {
  return static_cast<uint64_t>(L) | static_cast<uint64_t>(n) << 25 | static_cast<uint64_t>(row) << 43;
}
__device__ __forceinline__ int packed_n(uint64_t x) { return static_cast<int>(x >> 25 & 0x3ffff); }
__device__ __forceinline__ int packed_L(uint64_t x) { return static_cast<int>(x & 0x1ffffff); }
__device__ __forceinline__ int packed_row(uint64_t x) { return static_cast<int>(x >> 43); }
__device__ __forceinline__ Item item_of(const MassParams& p, uint64_t x) {
  Item it;
  it.L = packed_L(x);
  it.n = packed_n(x);
  it.row = packed_row(x);
  it.blocks = quotient(it.n + p.tpb - 1, p.inv_tpb) * p.chunks;
  return it;
}

// Units of a group whose blocks stay (one or two), by what it takes.  32 rows of 13 to 26 drafted tokens: 6 and 11 56.6 us,
// 1 and 2 57.0, 4 and 7 57.9, 2 and 3 62.5, 3 and 7 60.5 (of one case: between the first two it decides nothing).
__device__ __forceinline__ int weight_of(int blocks) { return 5 * blocks + 1; }

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
  int span;             // log2 of the keys of a group
  int ranges;
  int held;             // 1: a call was refused before this CTA looked (on another stream CTAs may differ), its range is empty
  int64_t begin, end;   // this CTA's range
  Start start;
  uint64_t bits[kQuerySlots][kMassTile];   // tree: drafted tokens that the pairs of a block see
  int64_t before[kMaxCallRows + 1];        // units before a sequence
  uint64_t item[kMaxCallRows];             // packed
};

// The tiles of one group of a row and the query blocks that see some of it.
struct Group {
  int k0, tiles, lo, hi;   // first key; tiles of 128; blocks lo .. hi - 1

  Group() = default;
  // where blocks may be cut: those that see some of it
  __device__ __forceinline__ Group(const MassParams& p, const Item& it, int span, int s) {
    k0 = s << span;
    const int end = min(it.L, k0 + (1 << span)), ctx = it.L - it.n;
    tiles = (end - k0 + kMassTile - 1) / kMassTile;
    int t0 = 0, t1 = it.n;
    if (!p.tree) {
      t0 = max(0, k0 - ctx);
      if (k0 >= p.n_sink) t1 = min(it.n, end - 1 + p.window - ctx);
    }
    lo = quotient(t0, p.inv_tpb) * p.chunks;
    hi = t1 <= t0 ? lo : quotient(t1 + p.tpb - 1, p.inv_tpb) * p.chunks;
  }
  // where they are not: all or none (keys from `seen` on are in some query's window)
  __device__ __forceinline__ Group(int n_sink, const Item& it, int span, int s, int seen) {
    k0 = s << span;
    const int end = min(it.L, k0 + (1 << span));
    tiles = (end - k0 + kMassTile - 1) / kMassTile;
    lo = 0;
    hi = k0 < n_sink || end > seen ? it.blocks : 0;
  }
  // a group that nothing sees is a unit all the same: its mass may fade
  __device__ __forceinline__ int units() const { return max(1, hi - lo); }
};

__device__ __forceinline__ int groups_of(int L, int span) { return (L + (1 << span) - 1) >> span; }

// Runs of blocks of one group, in the order of a CTA's range.  (Every role steps through them, and a step is
// a chain of dependent instructions: no divisions, and what a row does not change is kept.)
struct PieceIter {
  int seq, g, s;
  int b0, b1;        // blocks b0 .. b1 - 1
  int span, groups;  // log2 of the keys of a group; groups of the row
  int seen;          // first key in a window
  int64_t rem;       // units of the range from here on
  Group grp;
  Item it;
  __device__ __forceinline__ PieceIter(const MassParams& p, const Ctl* ctl)
      : seq(ctl->start.seq), g(ctl->start.g), s(ctl->start.s), span(ctl->span), rem(ctl->end - ctl->begin) {
    if (rem <= 0) return;
    row(p, ctl);
    take(p, ctl->start.b);
  }
  __device__ __forceinline__ void row(const MassParams& p, const Ctl* ctl) {
    it = item_of(p, ctl->item[seq]);
    groups = groups_of(it.L, span);
    seen = p.tree ? 0 : it.L - it.n - p.window + 1;
  }
  __device__ __forceinline__ bool valid() const { return rem > 0; }
  __device__ __forceinline__ bool whole() const { return b0 == grp.lo && b1 == grp.hi; }
  __device__ __forceinline__ void take(const MassParams& p, int from) {
    if (p.cut) {
      grp = Group(p, it, span, s);
      b0 = grp.lo + from;
      b1 = static_cast<int>(min(static_cast<int64_t>(grp.hi), b0 + rem));
    } else {
      grp = Group(p.n_sink, it, span, s, seen);
      b0 = 0;
      b1 = grp.hi;
    }
  }
  // the last group of this row and KV head that the range has
  __device__ __forceinline__ bool last_of_head() const { return rem <= weight_of(it.blocks) || s + 1 == groups; }
  __device__ __forceinline__ void next(const MassParams& p, const Ctl* ctl) {
    rem -= p.cut ? max(1, b1 - b0) : weight_of(it.blocks);
    if (rem <= 0) return;
    if (++s == groups) head(p, ctl);
    take(p, 0);
  }
  // p.cut is 0: on to the next row or KV head
  __device__ __forceinline__ void skip_head(const MassParams& p, const Ctl* ctl) {
    rem -= static_cast<int64_t>(groups - s) * weight_of(it.blocks);
    if (rem <= 0) return;
    head(p, ctl);
    take(p, 0);
  }
  __device__ __forceinline__ void head(const MassParams& p, const Ctl* ctl) {
    s = 0;
    if (++g == p.G) {
      g = 0;
      do ++seq;
      while (ctl->before[seq + 1] == ctl->before[seq]);
      row(p, ctl);
    }
  }
};

__device__ __forceinline__ int64_t range_begin(int64_t T, int c, int P) { return c < P ? T * c / P : T; }
// Ranges of a launch of T units on P CTAs: as many, but none empty.
__device__ __forceinline__ int ranges_of(int64_t T, int P) { return T < P ? max(static_cast<int>(T), 1) : P; }
// Range (of P) that holds flat unit f
__device__ __forceinline__ int range_of(int64_t f, int64_t T, int P) { return static_cast<int>(((f + 1) * P - 1) / T); }

// Every sequence's length and queries, the groups' span, the units before each sequence and this CTA's
// range.  `named`: 2 bits a row of the table (in shared memory), for rows that two sequences name.
// (Runs once, and cold code costs its size: one pass a thread over the sequences, one warp for the rest.)
__device__ void plan(const MassParams& p, Ctl* ctl, uint32_t* named) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int words = (p.n_rows + 31) >> 5;
  const bool rivals = p.rows && p.n > 1;
  const uint32_t latched = tid == 0 ? *p.err : 0;   // (behind a refused call nothing is added)
  if (rivals) {
    for (int i = tid; i < 2 * words; i += kThreads) named[i] = 0;
    __syncthreads();
  }
  int64_t tiles = 0;
  for (int i = tid; i < p.n; i += kThreads) {
    Item it;
    it.row = p.rows ? p.rows[i] : i;
    it.n = p.n_tokens ? p.n_tokens[i] : p.T;
    it.L = it.row >= 0 && it.row < p.n_rows ? p.len[it.row] : -1;
    if (it.n < 0 || it.n > p.T || (it.n > 0 && (it.L < it.n || it.L > static_cast<int64_t>(p.max_pages) << p.shift))) {
      it.n = 0;
      atomicOr(p.err, kErrRow);
    }
    if (rivals && it.n > 0 && (atomicOr(&named[it.row >> 5], 1u << (it.row & 31)) & (1u << (it.row & 31))))
      atomicOr(&named[words + (it.row >> 5)], 1u << (it.row & 31));
    if (it.n > 0) tiles += groups_of(it.L, kTileShift);
    ctl->item[i] = it.n > 0 ? packed(it.L, it.n, it.row) : 0;
  }
  if (tiles) atomicAdd(reinterpret_cast<unsigned long long*>(&ctl->end), static_cast<unsigned long long>(tiles));
  __syncthreads();
  const int span = kTileShift + (ctl->end * p.G >= p.span_from ? kSpanShift : 0);
  if (!p.cut) {
    for (int i = tid; i < p.n; i += kThreads) {
      const Item it = item_of(p, ctl->item[i]);
      if (rivals && it.n > 0 && (named[words + (it.row >> 5)] >> (it.row & 31) & 1)) {
        ctl->item[i] = 0;
        atomicOr(p.err, kErrRow);
        ctl->before[i + 1] = 0;
      } else {
        ctl->before[i + 1] = it.n > 0 ? static_cast<int64_t>(groups_of(it.L, span)) * weight_of(it.blocks) : 0;
      }
    }
  } else {
    for (int i = warp; i < p.n; i += kWarps) {
      const Item it = item_of(p, ctl->item[i]);
      const bool twice = rivals && it.n > 0 && (named[words + (it.row >> 5)] >> (it.row & 31) & 1);
      const int ng = it.n > 0 && !twice ? groups_of(it.L, span) : 0;
      // (below 2^26: 2^15 groups of four tiles at most, of one tile only where all units are few, and 2,032 blocks, of 1,016 tokens
      // with 129 heads a group; T H / G is no more than 2^17)
      int u = 0;
      for (int s = lane; s < ng; s += 32) u += Group(p, it, span, s).units();
      u = __reduce_add_sync(kFull, u);
      if (lane == 0) {
        ctl->before[i + 1] = u;
        if (twice) {
          ctl->item[i] = 0;
          atomicOr(p.err, kErrRow);
        }
      }
    }
  }
  __syncthreads();
  if (warp == 0) {
    int64_t at = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < p.n; i0 += 32) {
      int64_t u = i0 + lane < p.n ? ctl->before[i0 + lane + 1] * p.G : 0;
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
    const int R = ranges_of(at, gridDim.x);
    const int64_t f0 = range_begin(at, blockIdx.x + (lane & 1), R);   // (lanes 0 and 1: the range's ends)
    const int64_t fe = __shfl_sync(kFull, f0, 1);
    int64_t fb = __shfl_sync(kFull, f0, 0);
    Start st{0, 0, 0, 0};
    if (fb < fe) {
      int a = 0, b = p.n;   // the last sequence with no more than fb units before it
      while (b - a > 1) {
        const int mid = (a + b) >> 1;
        if (ctl->before[mid] <= fb) a = mid;
        else b = mid;
      }
      st.seq = a;
      const Item it = item_of(p, ctl->item[a]);
      const int ng = groups_of(it.L, span);
      int64_t off = fb - ctl->before[a];
      const int64_t heads = ctl->before[a + 1] - ctl->before[a];   // G times the units of one
      while ((st.g + 1) * heads <= off * p.G) ++st.g;
      off -= st.g * (heads / p.G);
      if (!p.cut) {   // the first group that begins in the range
        const int each = weight_of(it.blocks), part = static_cast<int>(off % each);
        st.s = static_cast<int>(off / each) + (part > 0);
        fb += part ? each - part : 0;
        if (st.s == ng) {
          st.s = 0;
          if (++st.g == p.G) {
            st.g = 0;
            do ++st.seq;
            while (st.seq < p.n && ctl->before[st.seq + 1] == ctl->before[st.seq]);
          }
        }
      } else {
        for (int left = static_cast<int>(off), s0 = 0;; s0 += 32) {
          const int u = s0 + lane < ng ? Group(p, it, span, s0 + lane).units() : 0;
          int inc = u;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(kFull, inc, o);
            if (lane >= o) inc += x;
          }
          const uint32_t past = __ballot_sync(kFull, inc > left);
          if (past || s0 + 32 >= ng) {
            const int l = past ? __ffs(past) - 1 : 31;
            st.s = s0 + l;
            st.b = left - __shfl_sync(kFull, inc - u, l);
            break;
          }
          left -= __shfl_sync(kFull, inc, 31);
        }
      }
    }
    const bool held = __shfl_sync(kFull, latched, 0) & kErrHeld;
    if (held) fb = fe;
    if (lane == 0) {
      ctl->held = held;
      ctl->start = st;
      ctl->span = span;
      ctl->ranges = R;
      ctl->begin = fb;
      ctl->end = fe;
    }
  }
  __syncthreads();
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
  const bool there = mbar_try_wait(bar, parity) || mbar_wait(bar, parity, limit_ns);   // (most waits end before a clock is read)
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

// Keys: the tiles' pages into the ring, half of the channels a warp (one warp alone took 2,100 cycles a tile of four
// pages, where the copy rate leaves 1,500).
__device__ void key_loop(const MassParams& p, Ctl* ctl, uint8_t* sK, int half, int lane) {
  const uint64_t pol = policy_evict_first();
  const int P = 1 << p.shift, rows = min(P, 64), boxes = kMassTile / rows;
  Ring<kKeySlots> st;
  uint32_t used = 0, last_par = 0;   // last_par: bit s = parity of the last load into slot s
  bool ok = true;
  int base = 0, held = 0;            // lane l: pages base + l and base + 32 + l of the row, on their way before they are due
  int id = 0, id_next = 0;
  const int32_t* entries = nullptr;
  int seq = -1;
  auto number = [&](int at) {        // outside the map: zeros
    int x = p.n_pages;
    if (at < held) {
      x = entries[at];
      if (x < 0 || x >= p.n_pages) {
        x = p.n_pages;
        atomicOr(p.err, kErrRow);
      }
    }
    return x;
  };
  for (PieceIter c(p, ctl); ok && c.valid(); c.next(p, ctl)) {
    if (c.b0 == c.b1) continue;
    const int page0 = c.grp.k0 >> p.shift;   // (a group has 512 keys: 32 pages at most)
    const int page1 = (c.grp.k0 + c.grp.tiles * kMassTile - 1) >> p.shift;
    if (c.seq != seq || page0 < base || page1 >= base + 64) {
      seq = c.seq;
      entries = p.table + static_cast<int64_t>(c.it.row) * p.max_pages;
      held = (c.it.L + P - 1) >> p.shift;
      base = page0;
      id = number(base + lane);
      id_next = number(base + 32 + lane);
    } else if (page0 >= base + 32) {
      base += 32;
      id = id_next;
      id_next = number(base + 32 + lane);
    }
    __syncwarp();
    for (int i = 0; i < c.grp.tiles; ++i) {
      ok = warp_wait(ctl, &ctl->k_empty[st.at], st.par ^ 1, p.wait_ns);
      if (!ok) break;
      if (elect_one()) mbar_arrive_expect_tx(&ctl->k_full[st.at], kHalfBytes);
      // a box a lane (one after the other by one lane, each with its page number fetched, took 245 cycles a box)
      const int key = c.grp.k0 + i * kMassTile + lane * rows, at = (key >> p.shift) - base;
      const int near = __shfl_sync(kFull, id, at & 31), far = __shfl_sync(kFull, id_next, at & 31);
      if (lane < boxes) {
        uint8_t* dst = sK + st.at * kTileBytes + half * kHalfBytes + lane * rows * 128;
        const int page = at < 32 ? near : far;
        if (p.cut) tma_load_4d(dst, &p.tmk, &ctl->k_full[st.at], half * 64, key & (P - 1), c.g, page);
        else tma_load_4d_hint(dst, &p.tmk, &ctl->k_full[st.at], half * 64, key & (P - 1), c.g, page, pol);
      }
      __syncwarp();
      used |= 1u << st.at;
      last_par = (last_par & ~(1u << st.at)) | (st.par << st.at);
      st.next();
    }
  }
  if (!ok) fail(ctl, p.err);
  // Every issued copy completes before the CTA can exit.  (Where the other key warp gave up first, its share of a slot never
  // comes and the barrier does not complete: once the limit has passed all copies have had that time.)
  bool in_time = true;
  for (int i = 0; i < kKeySlots; ++i)
    if (in_time && (used >> i & 1)) in_time = mbar_wait(&ctl->k_full[i], last_par >> i & 1, drain_limit(p.wait_ns));
  __syncwarp();
}

// (token, head) pairs of a block: columns c < count, token t0 + c / heads, head h0 + c % heads of the group.
struct Block {
  int t0, h0, count;
  __device__ __forceinline__ Block(const MassParams& p, int n, int b) {
    const int tb = quotient(b, p.inv_chunks);
    t0 = tb * p.tpb;
    h0 = (b - tb * p.chunks) * kMassTile;   // (0 unless the heads of a group are more than a block has columns)
    count = min(p.tpb, n - t0) * min(p.heads, p.hg - h0);
  }
  __device__ __forceinline__ int columns() const { return (count + 15) & ~15; }
};

// Queries: blocks into the ring, rows of 128 bytes with the chunks of 16 swizzled as the tensor core reads
// them, zeros behind the last pair.
__device__ void query_loop(const MassParams& p, Ctl* ctl, uint8_t* sQ, uint8_t* sL, int tid) {
  Ring<kQuerySlots> st;
  bool ok = true, there = false;   // there: the blocks of this row and KV head stay
  const int lane = tid & 31, chunk = tid & 15;
  // (a slot whose blocks stay is free when the CTA is through with a row and KV head: microseconds a group)
  const uint64_t wait_ns = p.wait_ns + (p.cut ? 0 : static_cast<uint64_t>(ctl->end - ctl->begin) * 5000);
  for (PieceIter c(p, ctl); ok && c.valid(); there ? c.skip_head(p, ctl) : c.next(p, ctl)) {
    there = false;
    for (int b = c.b0; ok && b < c.b1; ++b) {
      ok = warp_wait(ctl, &ctl->q_empty[st.at], st.par ^ 1, wait_ns);
      if (!ok) break;
      const Block blk(p, c.it.n, b);
      const int columns = blk.columns();
      float lse = 0.f;
      uint64_t bits = 0;
      if (tid < blk.count) {   // (a pair a thread; on their way before the copies)
        const int at_t = quotient(tid, p.inv_heads);
        const int64_t at = static_cast<int64_t>(c.seq) * p.T + blk.t0 + at_t;
        lse = p.lse[at * p.H + c.g * p.hg + blk.h0 + tid - at_t * p.heads];
        if (p.tree) bits = p.mask[at];
      }
      int r = tid >> 4, t = quotient(r, p.inv_heads), h = r - t * p.heads;
      const __nv_bfloat16* q = p.q + c.seq * p.q_seq + (static_cast<int64_t>(c.g) * p.hg + blk.h0 + h) * p.q_head +
                               (blk.t0 + t) * p.q_token + chunk * 8;
      uint32_t dst = smem_u32(sQ) + st.at * kTileBytes + (chunk >> 3) * kHalfBytes + r * 128 + (((chunk & 7) ^ (r & 7)) << 4);
#pragma unroll 4
      for (; r < columns; r += kMassQueryStep) {   // (eight rows on, the swizzle is the same)
        cp_async16(dst, r < blk.count ? q : p.q, r < blk.count);
        dst += kMassQueryStep * 128;
        q += p.step;
        h += p.step_h;
        if (h >= p.heads) {
          h -= p.heads;
          q += p.wrap;
        }
      }
      if (tid < columns) {
        // -lse in units of the products, three bf16 parts (24 bits; one where it is not finite)
        const float x = -lse * kRootDim;
        const __nv_bfloat16 hi = __float2bfloat16_rn(x);
        const float rest = fabsf(x) < INFINITY ? x - __bfloat162float(hi) : 0.f;
        const __nv_bfloat16 mid = __float2bfloat16_rn(rest), lo = __float2bfloat16_rn(rest - __bfloat162float(mid));
        uint4* row = reinterpret_cast<uint4*>(sL + st.at * kExtraBytes + (tid >> 3) * 256 + (tid & 7) * 16);
        row[0] = make_uint4(__bfloat16_as_ushort(hi) | static_cast<uint32_t>(__bfloat16_as_ushort(mid)) << 16, __bfloat16_as_ushort(lo), 0u, 0u);
        row[8] = make_uint4(0u, 0u, 0u, 0u);
        if (p.tree) ctl->bits[st.at][tid] = bits;
      }
      cp_async_wait();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl->q_full[st.at]);
      st.next();
      there = !p.cut;
    }
  }
  if (!ok) fail(ctl, p.err);
}

// Products: issuer 0 or 1 has every other tile.  (One for all left the tensor pipe idle for 400 of 1,000 cycles a tile and
// block, between the end of one's instructions and the start of the next one's.)
__device__ void mma_loop(const MassParams& p, Ctl* ctl, const uint8_t* sK, const uint8_t* sQ, const uint8_t* sOne, const uint8_t* sL,
                         uint32_t tmem, int issuer) {
  const uint64_t dk0 = sdesc_k_sw128(smem_u32(sK)), dq0 = sdesc_k_sw128(smem_u32(sQ));
  const uint64_t one = sdesc_k_none(smem_u32(sOne), 128, 0), dl0 = sdesc_k_none(smem_u32(sL), 128, 256);
  Ring<kKeySlots> st;
  Ring<kQuerySlots> q;    // the next block to come
  uint32_t s_par = 0;     // bit a: parity of accumulator a's next use
  bool ok = true;
  int held = 0, first = 0;   // blocks of this row and KV head that stay, and the first one's slot
  for (PieceIter c(p, ctl); ok && c.valid(); c.next(p, ctl)) {
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
      for (int i = 0; ok && i < c.grp.tiles; ++i, at.next()) {
        if ((at.at & 1) != issuer) continue;
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
          mma_bf16(tmem + at.at * kMassTile, one, dl0 + static_cast<uint64_t>(slot * (kExtraBytes >> 4)), idesc, 1);
          mma_commit(&ctl->s_full[at.at]);
          if (j == nb - 1) mma_commit(&ctl->k_empty[at.at]);
        }
        __syncwarp();
        s_par ^= 1u << at.at;
      }
      if (p.cut) {   // (with no tile of its own as well: both issuers are counted)
        if (ok && elect_one()) mma_commit(&ctl->q_empty[slot]);
        __syncwarp();
      }
    }
    st = at;
    if (!p.cut) {
      if (take) held = nb;
      if (c.last_of_head()) {
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

// 16 accumulator columns, as tmem_ld16_async and tmem_wait16, but without their order against other memory: what
// is read between them is read-only here, and may be read ahead.
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void wait16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;\n"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}

// Sum of 16 pairs' weights, all of them seen; TAIL: of those in front of `count` (behind them an earlier block
// may have left anything).
template <bool TAIL>
__device__ __forceinline__ float2 weigh16(const uint32_t (&z)[16], float2 sc, int count, float2 acc) {
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    const float2 a = fmul2(make_float2(__uint_as_float(z[i]), __uint_as_float(z[i + 1])), sc);
    const float2 b = fmul2(make_float2(__uint_as_float(z[i + 2]), __uint_as_float(z[i + 3])), sc);
    float2 x = make_float2(ex2_approx(a.x), ex2_approx(a.y)), y = make_float2(ex2_approx(b.x), ex2_approx(b.y));
    if (TAIL) {
      x = make_float2(i < count ? x.x : 0.f, i + 1 < count ? x.y : 0.f);
      y = make_float2(i + 2 < count ? y.x : 0.f, i + 3 < count ? y.y : 0.f);
    }
    acc = fadd2(acc, fadd2(x, y));
  }
  return acc;
}

// A block that the warp's keys are seen by: 16 columns at a time, the next ones on their way.  (A short loop: unrolled
// over the block, whose code is then longer than the innermost instruction caches, it took half as long again.)
__device__ __forceinline__ float weigh_block(uint32_t addr, float c2, int count) {
  const float2 sc = make_float2(c2, c2);
  uint32_t z0[16], z1[16];
  float2 acc = make_float2(0.f, 0.f);
  ld16(addr, z0);
#pragma unroll 1
  for (; count >= 32; count -= 32) {
    wait16(z0);
    ld16(addr + 16, z1);
    acc = weigh16<false>(z0, sc, 0, acc);
    wait16(z1);
    if (count > 32) ld16(addr + 32, z0);
    acc = weigh16<false>(z1, sc, 0, acc);
    addr += 32;
  }
#pragma unroll 1
  for (; count > 0; count -= 16) {
    wait16(z0);
    acc = weigh16<true>(z0, sc, count, acc);
    addr += 16;
    if (count > 16) ld16(addr, z0);
  }
  return acc.x + acc.y;
}

// A block under a window that is not: the tokens that see a key follow one another, so that their pairs are the columns
// lo .. hi - 1 (of this thread's key).
__device__ __forceinline__ float weigh_columns(uint32_t addr, float c2, int lo, int hi, int count) {
  float sum = 0.f;
#pragma unroll 1
  for (; count > 0; count -= 16) {
    uint32_t z[16];
    ld16(addr, z);
    wait16(z);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float w = ex2_approx(__uint_as_float(z[i]) * c2);
      sum += i >= lo && i < hi ? w : 0.f;
    }
    addr += 16;
    lo -= 16;
    hi -= 16;
  }
  return sum;
}

// A block of a tree that is not: of the pairs in front of `count` those whose token has bit j - ctx, or all for a cached key.
__device__ __forceinline__ float weigh_bits(uint32_t addr, const uint64_t* bits, float c2, int count, int j, int ctx, int L) {
  float sum = 0.f;
  const int drafted = max(j - ctx, 0), shift = drafted & 31;
  const uint32_t any = j < ctx ? ~0u : 0u;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(bits) + (drafted >> 5 & 1);
  if (j >= L) count = 0;
  const int most = __reduce_max_sync(kFull, count);
#pragma unroll 1
  for (int c = 0; c < most; c += 16) {
    uint32_t z[16];
    ld16(addr + c, z);
    wait16(z);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float w = ex2_approx(__uint_as_float(z[i]) * c2);
      sum += ((words[2 * (c + i)] | any) >> shift & 1) && c + i < count ? w : 0.f;
    }
  }
  return sum;
}

// Whether token j of a row lies in a page that is one.  (Keys of another are loaded as zeros, and their tokens' mass is left alone.)
__device__ __forceinline__ bool in_a_page(const MassParams& p, int row, int j) {
  return static_cast<uint32_t>(p.table[static_cast<int64_t>(row) * p.max_pages + (j >> p.shift)]) < static_cast<uint32_t>(p.n_pages);
}

// Weighing warpgroup `own`: every fourth tile, a key a thread.
__device__ void weigh_loop(const MassParams& p, Ctl* ctl, uint32_t tmem, int own, int quad, int lane) {
  const int r = quad * 32 + lane;
  const uint32_t at = tmem + (static_cast<uint32_t>(quad * 32) << 16) + own * kMassTile;   // this warp's part of the accumulator
  Ring<kQuerySlots> q;
  uint32_t tile = 0;       // number of the next tile to come
  uint32_t par = 0;        // parity of the accumulator's next use
  bool ok = true;
  int held = 0, slot0 = 0; // blocks of this row and KV head that stay, and the first one's slot
  for (PieceIter c(p, ctl); ok && c.valid(); c.next(p, ctl)) {
    const int nb = c.b1 - c.b0;
    const bool take = p.cut || held == 0;
    if (take) slot0 = q.at;
    const int i = (own - tile) & (kKeySlots - 1);   // the group's tile that is this warpgroup's, if it has as many
    const bool mine = i < c.grp.tiles;
    const int ctx = c.it.L - c.it.n, k0 = c.grp.k0 + i * kMassTile + 32 * quad, k1 = k0 + 31, j = k0 + lane;
    float* mass = p.mass.m + c.it.row * p.mass.row_stride + c.g * p.mass.group_stride + j;
    const bool whole = c.whole();
    float sum = 0.f, had = 0.f;
    bool paged = true;
    if (mine && whole && j < c.it.L) {
      paged = in_a_page(p, c.it.row, j);
      if (j < ctx) had = *mass;
    }
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
        // by the warp's 32 keys: seen by all of the block, by none, or by some
        const Block blk(p, c.it.n, c.b0 + b);
        const int first = ctx + blk.t0, end = ctx + min(blk.t0 + p.tpb, c.it.n) - 1;   // positions of the block's tokens
        bool all, none = k0 >= c.it.L;
        if (p.tree) {
          all = k1 < ctx;
        } else {
          all = k1 <= first && (k1 < p.n_sink || k0 > end - p.window);
          none = none || k0 > end || (k0 >= p.n_sink && k1 <= first - p.window);
        }
        if (all) {
          sum += weigh_block(at, p.scale2, blk.count);
        } else if (p.tree) {
          if (!none) sum += weigh_bits(at, ctl->bits[slot], p.scale2, blk.count, j, ctx, c.it.L);
        } else if (!none) {
          const int nt = end - first + 1;
          const int ta = min(max(j - first, 0), nt), tb = j < p.n_sink ? nt : min(max(j + p.window - first, 0), nt);
          const int per = nt > 1 ? p.heads : blk.count;   // columns of a token
          sum += weigh_columns(at, p.scale2, ta * per, tb * per, blk.count);
        }
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
      if (c.last_of_head()) {
        if (lane == 0)
          for (int b = 0; b < held; ++b) mbar_arrive(&ctl->q_empty[(slot0 + b) % kQuerySlots]);
        held = 0;
      }
    }
    if (mine && !whole)
      p.part[(2 * static_cast<int64_t>(blockIdx.x) + (c.b0 == c.grp.lo)) * (kMassSpan * kMassTile) + i * kMassTile + r] = sum;
    else if (mine && j < c.it.L) {
      if (paged) *mass = fmaf(p.decay, had, sum);
      else atomicOr(p.err, kErrRow);
    }
    if (nb > 0) tile += c.grp.tiles;
  }
  if (!ok) fail(ctl, p.err);
}

}  // namespace

__global__ void __launch_bounds__(kThreads, 1) k_mass(const __grid_constant__ MassParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem;                            // [slots][2 halves][128 keys][128 B]
  uint8_t* sQ = sK + kKeySlots * kTileBytes;     // [slots][2 halves][128 pairs][128 B]
  uint8_t* sOne = sQ + kQuerySlots * kTileBytes; // [8][16]: 1, 1, 1, 0 ..., for every eight keys of a tile
  uint8_t* sL = sOne + kOneBytes;                // [slots][128 pairs][16]: the parts of -lse, 0 ...
  Ctl* ctl = reinterpret_cast<Ctl*>(sL + kQuerySlots * kExtraBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kKeySlots; ++i) {
      mbar_init(&ctl->k_full[i], 2);
      mbar_init(&ctl->k_empty[i], 1);
      mbar_init(&ctl->s_full[i], 1);
      mbar_init(&ctl->s_empty[i], 4);
    }
    for (int i = 0; i < kQuerySlots; ++i) {
      mbar_init(&ctl->q_full[i], kSoftWarp - kQueryWarp);
      mbar_init(&ctl->q_empty[i], 2 + kWarps - kSoftWarp);   // both issuers and every weighing warp
    }
    mbar_init(&ctl->drain, 2);
    ctl->abort = 0;
    ctl->end = 0;
    fence_mbar_init();
  }
  if (threadIdx.x < 8) {
    uint4* row = reinterpret_cast<uint4*>(sOne + threadIdx.x * 16);
    row[0] = make_uint4(0x3F803F80u, 0x3F80u, 0u, 0u);
    row[8] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&ctl->tmem_base, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch_dependents();
  griddep_wait();
  const uint32_t tmem = ctl->tmem_base;
  plan(p, ctl, reinterpret_cast<uint32_t*>(sQ));
  if (warp < kMmaWarp) {
    key_loop(p, ctl, sK, warp, lane);
  } else if (warp < kQueryWarp) {
    mma_loop(p, ctl, sK, sQ, sOne, sL, tmem, warp - kMmaWarp);
  } else if (warp >= kSoftWarp) {
    weigh_loop(p, ctl, tmem, (warp - kSoftWarp) >> 2, warp & 3, lane);
  } else if (warp >= kQueryWarp) {
    query_loop(p, ctl, sQ, sL, threadIdx.x - 32 * kQueryWarp);
  }
  if (threadIdx.x == 0 && p.cut) {   // what the sum of the parts has to know of this range's end
    MassSplit s;
    s.valid = 0;
    for (PieceIter c(p, ctl); c.valid(); c.next(p, ctl))
      if (c.b0 == c.grp.lo && c.b1 < c.grp.hi) {
        s.valid = 1;
        s.seq = c.seq;
        s.g = c.g;
        s.k0 = c.grp.k0;
        s.keys = min(c.grp.tiles * kMassTile, c.it.L - c.grp.k0);
        s.last = range_of(ctl->end + (c.grp.hi - c.b1) - 1, ctl->before[p.n], ctl->ranges);
      }
    s.failed = ctl->held;
    p.split[blockIdx.x] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0 && p.cut && ctl->abort) p.split[blockIdx.x].failed = 1;
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Adds up the parts of the groups that ranges cut, in the order of the ranges: block c has the one that range c began.
// Where one of these ranges was given up, the group's tokens keep their mass (a part that was not written holds anything).
__global__ void __launch_bounds__(kMassSpan * kMassTile) k_mass_sum(const __grid_constant__ MassParams p) {
  griddep_launch_dependents();
  griddep_wait();
  const MassSplit s = p.split[blockIdx.x];
  if (!s.valid || static_cast<int>(threadIdx.x) >= s.keys) return;
  const int row = p.rows ? p.rows[s.seq] : s.seq;
  const int n = p.n_tokens ? p.n_tokens[s.seq] : p.T;
  const int L = p.len[row], j = s.k0 + threadIdx.x;
  if (!in_a_page(p, row, j)) return;   // (reported when its keys were loaded)
  float* mass = p.mass.m + row * p.mass.row_stride + s.g * p.mass.group_stride + j;
  const float had = j < L - n ? *mass : 0.f;
  float sum = 0.f;
  int failed = 0;
  for (int c = blockIdx.x; c <= s.last; ++c) {
    sum += p.part[(2 * static_cast<int64_t>(c) + (c == static_cast<int>(blockIdx.x))) * (kMassSpan * kMassTile) + threadIdx.x];
    failed |= p.split[c].failed;
  }
  if (!failed) *mass = fmaf(p.decay, had, sum);
}

namespace {

constexpr size_t kSmemBytes =
    1024 + static_cast<size_t>(kKeySlots + kQuerySlots) * kTileBytes + kOneBytes + kQuerySlots * kExtraBytes + sizeof(Ctl);
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

constexpr int kSelThreads = 512;   // (1,024: one block an SM, 41 us for 35 in the 224 blocks of eight rows in 28 layers; 21 for 22 in
                                   // the 112 of one row)
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelKeys = 49152;    // keys that shared memory holds
constexpr int kSelLoads = 8;       // masses of a thread and KV head on their way at once (one: 48 us for 41 there)
constexpr int kSelMoves = 4;       // masses of a thread on their way at once
constexpr int kSelBins = 2048;
constexpr int kSelClose = 512;     // close tokens that are ranked by comparing each with each
static_assert(kSelThreads >= kSelClose && kSelThreads >= 256 && kSelBins % kSelThreads == 0, "a thread a close token and a digit");

// Ascending order as unsigned numbers; a NaN (a mass that is none) comes with infinity, so that its token
// stays, and -0 is 0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) x = INFINITY;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(double x) {
  if (x != x) x = INFINITY;
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

struct SelSmem {
  int hist[256];
  int warp_sum[kSelWarps];
  uint64_t digit;
  int need, bin;
  uint32_t least, most, size, negative;
  int bins[kSelBins];
  uint64_t close[kSelClose];
  int close_at[kSelClose];
  uint8_t stays[kSelClose];
  uint32_t key[1];   // as many as the launch asks for
};

// Sum over the block of a count per thread, in front of this thread's; the total to everybody.
__device__ int sum_before(int x, int* warp_sum, int* total) {
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
  for (int w = 0; w < kSelWarps; ++w) {
    if (w < warp) before += warp_sum[w];
    all += warp_sum[w];
  }
  __syncthreads();
  *total = all;
  return before;
}

// The k-th greatest of key(0) .. key(n - 1), eight bits at a time; *of_it: how many of those that have it are among the
// k greatest.  (Keys share their first bits: a warp adds up those that meet before it goes to shared memory.)
template <typename Key, typename F>
__device__ Key kth_greatest(SelSmem& s, int n, int k, F key, int* of_it) {
  const int tid = threadIdx.x, lane = tid & 31;
  constexpr int kTop = static_cast<int>(sizeof(Key)) * 8 - 8;
  Key prefix = 0;
#pragma unroll 1
  for (int bit = kTop; bit >= 0; bit -= 8) {
    if (tid < 256) s.hist[tid] = 0;
    __syncthreads();
    for (int j0 = 0; j0 < n; j0 += kSelThreads) {
      const Key x = j0 + tid < n ? key(j0 + tid) : 0;
      const bool counts = j0 + tid < n && (bit == kTop || (x ^ prefix) >> (bit + 8) == 0);
      if (!__any_sync(kFull, counts)) continue;
      const int digit = counts ? static_cast<int>(x >> bit & 255) : -1;
      const uint32_t same = __match_any_sync(kFull, digit);
      if (counts && lane == __ffs(same) - 1) atomicAdd(&s.hist[digit], __popc(same));
    }
    __syncthreads();
    if (tid < 32) {   // lane l: the digits 255 - 8 l downwards
      int sum = 0, c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += c[i] = s.hist[255 - 8 * lane - i];
      int inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, inc, o);
        if (lane >= o) inc += y;
      }
      int left = k - (inc - sum);
      if (left > 0 && left <= sum) {
        int i = 0;
        while (i < 7 && c[i] < left) left -= c[i++];
        s.digit = 255 - 8 * lane - i;
        s.need = left;
      }
    }
    __syncthreads();
    prefix |= static_cast<Key>(s.digit) << bit;
    k = s.need;
  }
  *of_it = k;
  return prefix;
}

}  // namespace

// Block (set, layer, sequence): the budget tokens j < L - w of greatest mass (PER_HEAD: of one KV head, else of
// all of them added up), equal ones the lowest first, in ascending order; then the mass of the kept ones and of the window
// moves to their new places.
//
// Sums are formed in 32 bits first.  Of G masses that are not negative one is off by at most (G - 1) 2^-24 of itself (of the
// largest sum of sizes else): tokens further than that from the budget-th greatest are in or out, and the few between are
// added up in 64 bits.  (In 64 bits throughout, and again for every digit, eight rows of 12,000 tokens in 28 layers took 560 us.)
template <bool PER_HEAD>
__global__ void __launch_bounds__(kSelThreads)
    k_mass_select(const __grid_constant__ PagesView pg, const __grid_constant__ SeqBatch b, const int32_t* rows, int row0, int w,
                  const PagePlan* plan, const __grid_constant__ MassView mv) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  SelSmem& s = *reinterpret_cast<SelSmem*>(smem_raw);
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
  const float* heads = mass + g0 * mv.group_stride;
  auto sum_of = [&](int j, float* size) {
    float x = heads[j], a = fabsf(x);
    for (int g = g0 + 1; g < g1; ++g) {
      const float y = mass[g * mv.group_stride + j];
      x += y;
      a += fabsf(y);
    }
    *size = a;
    return x;
  };
  const bool here = Lp <= kSelKeys;
  auto key_of = [&](int j) {
    float a;
    return here ? s.key[j] : order_key(sum_of(j, &a));
  };
  if (B > 0 && B < Lp) {
    if (tid == 0) s.size = s.negative = s.most = 0, s.least = ~0u;
    for (int i = tid; i < kSelBins; i += kSelThreads) s.bins[i] = 0;
    __syncthreads();
    uint32_t size = 0, least = ~0u, most = 0;
    bool negative = false;
    for (int j0 = tid; j0 < Lp; j0 += kSelLoads * kSelThreads) {
      float x[kSelLoads], a[kSelLoads];
#pragma unroll
      for (int u = 0; u < kSelLoads; ++u) {
        x[u] = heads[min(j0 + u * kSelThreads, Lp - 1)];   // (behind the last token: the last one again)
        a[u] = fabsf(x[u]);
      }
      if (!PER_HEAD)
#pragma unroll 1
        for (int g = 1; g < pg.G; ++g) {
          float y[kSelLoads];
#pragma unroll
          for (int u = 0; u < kSelLoads; ++u) y[u] = mass[g * mv.group_stride + min(j0 + u * kSelThreads, Lp - 1)];
#pragma unroll
          for (int u = 0; u < kSelLoads; ++u) x[u] += y[u], a[u] += fabsf(y[u]);
        }
#pragma unroll
      for (int u = 0; u < kSelLoads; ++u) {
        const uint32_t k = order_key(x[u]);
        if (here && j0 + u * kSelThreads < Lp) s.key[j0 + u * kSelThreads] = k;
        least = min(least, k);
        most = max(most, k);
        if (!PER_HEAD) {
          size = max(size, __float_as_uint(a[u]));   // (a NaN is above infinity)
          negative = negative || a[u] != x[u];       // (also where a sum is not a number)
        }
      }
    }
    least = __reduce_min_sync(kFull, least);
    most = __reduce_max_sync(kFull, most);
    if (!PER_HEAD) {
      size = __reduce_max_sync(kFull, size);
      negative = __any_sync(kFull, negative);
    }
    if ((tid & 31) == 0) {
      atomicMin(&s.least, least);
      atomicMax(&s.most, most);
      if (!PER_HEAD) atomicMax(&s.size, size);
      if (negative) s.negative = 1;
    }
    __syncthreads();
    least = s.least;
    most = s.most;
    // the bin of keys (of equal width between the least and the greatest) that the budget-th greatest is in
    const int shift = max(0, 32 - __clz(most - least) - 11);   // (kSelBins = 2^11)
    for (int j = tid; j < Lp; j += kSelThreads) atomicAdd(&s.bins[(key_of(j) - least) >> shift], 1);
    __syncthreads();
    {
      constexpr int kOwn = kSelBins / kSelThreads;   // bins of a thread, from the greatest down
      int count[kOwn], sum = 0, total;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) sum += count[i] = s.bins[kSelBins - 1 - tid * kOwn - i];
      int left = B - sum_before(sum, s.warp_sum, &total);
      if (left > 0 && left <= sum) {
        int i = 0;
#pragma unroll
        for (int u = 0; u < kOwn - 1; ++u)
          if (i == u && count[u] < left) left -= count[u], ++i;
        s.bin = kSelBins - 1 - tid * kOwn - i;
      }
      __syncthreads();
    }
    const uint32_t first = least + (static_cast<uint32_t>(s.bin) << shift);
    uint32_t bottom = first, top = min(most, first + ((1u << shift) - 1));   // keys that the budget-th greatest lies between
    const int run = ((Lp + kSelThreads - 1) / kSelThreads) | 1;   // tokens of a thread (odd: no two of a warp in one bank)
    const int from = min(tid * run, Lp), to = min(from + run, Lp);
    // A second round, with the budget-th greatest itself, where the bin holds more tokens than are compared one by one.
#pragma unroll 1
    for (bool again = false;; again = true) {
      int need;   // of the tokens that have the key
      if (again) top = bottom = kth_greatest<uint32_t>(s, Lp, B, key_of, &need);
      uint32_t above = top, below = bottom;   // greater keys are in, lower ones out
      if (!PER_HEAD) {
        const float t = key_value(top), e = pg.G * 2.5f * 0x1p-24f;   // (twice the error, and roundings)
        const float off = s.negative || !(fabsf(t) < INFINITY) ? __uint_as_float(s.size) * e : t * e;
        above = order_key(t + off + 1e-44f);
        below = order_key(key_value(bottom) - off - 1e-44f);
        if (!(off < INFINITY)) above = ~0u, below = 0;   // all of them are between
      }
      int sure = 0, close = 0, n_sure, n_close;
      for (int j = from; j < to; ++j) {
        const uint32_t k = key_of(j);
        sure += k > above;
        close += k <= above && k >= below;
      }
      int at_sure = sum_before(sure, s.warp_sum, &n_sure), at_close = sum_before(close, s.warp_sum, &n_close);
      const int left = B - n_sure;
      if (left == n_close || (PER_HEAD && top == bottom)) {   // of the close ones the lowest
        for (int j = from; j < to; ++j) {
          const uint32_t k = key_of(j);
          const bool near = k <= above && k >= below;
          if (k > above || (near && at_close < left)) idx[at_sure + min(at_close, left)] = j;
          at_sure += k > above;
          at_close += near;
        }
        break;
      }
      auto exact = [&](int j) -> uint64_t {
        if (PER_HEAD) return key_of(j);
        double x = heads[j];
        for (int g = g0 + 1; g < g1; ++g) x += static_cast<double>(mass[g * mv.group_stride + j]);
        return order_key(x);
      };
      if (n_close <= kSelClose) {   // each compared with each
        int c = at_close;
        for (int j = from; j < to; ++j) {
          const uint32_t k = key_of(j);
          if (k <= above && k >= below) s.close_at[c++] = j;
        }
        __syncthreads();
        if (tid < n_close) s.close[tid] = exact(s.close_at[tid]);
        __syncthreads();
        int stays = 0, total;
        if (tid < n_close) {
          const uint64_t k = s.close[tid];
          int better = 0;
          for (int i = 0; i < n_close; ++i) better += s.close[i] > k || (s.close[i] == k && i < tid);
          stays = better < left;
          s.stays[tid] = stays;
        }
        __syncthreads();
        c = at_close;
        int taken = sure;
        for (int j = from; j < to; ++j) {
          const uint32_t k = key_of(j);
          if (k <= above && k >= below) taken += s.stays[c++];
        }
        int out = sum_before(taken, s.warp_sum, &total);
        c = at_close;
        for (int j = from; j < to; ++j) {
          const uint32_t k = key_of(j);
          if (k > above || (k <= above && k >= below && s.stays[c++])) idx[out++] = j;
        }
        break;
      }
      if (!again) continue;
      // too many of them: digits of the sums in 64 bits
      int equal, total;
      const uint64_t border = kth_greatest<uint64_t>(s, Lp, left, [&](int j) {
        const uint32_t k = key_of(j);
        return k <= above && k >= below ? exact(j) : 0;
      }, &equal);
      int same = 0, taken = 0;
      for (int j = from; j < to; ++j) {
        const uint32_t k = key_of(j);
        if (k <= above && k >= below) same += exact(j) == border;
      }
      const int at_same = sum_before(same, s.warp_sum, &total);
      auto stays = [&](int j, int* e) {
        const uint32_t k = key_of(j);
        if (k > above || k < below) return k > above;
        const uint64_t x = exact(j);
        return x > border || (x == border && (*e)++ < equal);
      };
      for (int j = from, e = at_same; j < to; ++j) taken += stays(j, &e);
      int out = sum_before(taken, s.warp_sum, &total);
      for (int j = from, e = at_same; j < to; ++j)
        if (stays(j, &e)) idx[out++] = j;
      break;
    }
  } else {
    for (int j = tid; j < B; j += kSelThreads) idx[j] = j;
  }
  __syncthreads();   // the indices are written
  // A token's new place is never behind its old one: what a round writes has been read.
  for (int r0 = 0; r0 < B + w; r0 += kSelMoves * kSelThreads) {
    int src[kSelMoves];
#pragma unroll
    for (int u = 0; u < kSelMoves; ++u) {
      const int r = r0 + u * kSelThreads + tid;
      src[u] = r < B ? idx[r] : r < B + w ? Lp + (r - B) : -1;
    }
    for (int g = g0; g < g1; ++g) {
      float* m = mass + g * mv.group_stride;
      float x[kSelMoves];
#pragma unroll
      for (int u = 0; u < kSelMoves; ++u) x[u] = src[u] >= 0 ? m[src[u]] : 0.f;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kSelMoves; ++u)
        if (src[u] >= 0) m[r0 + u * kSelThreads + tid] = x[u];
    }
    __syncthreads();
  }
}

cudaError_t mass_select_configure() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  const int most = sizeof(SelSmem) + kSelKeys * 4;
  const cudaError_t e = cudaFuncSetAttribute(k_mass_select<true>, attr, most);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(k_mass_select<false>, attr, most);
}

cudaError_t mass_select_launch(const PagesView& pg, const SeqBatch& b, const int32_t* rows, int row0, int w, int per_head,
                               const PagePlan* plan, const MassView& mass, cudaStream_t stream) {
  int keys = 0;
  for (int i = 0; i < b.nseq; ++i)
    if (b.s[i].Lp <= kSelKeys) keys = std::max(keys, b.s[i].Lp);
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(per_head ? pg.G : 1, b.nlayers, b.nseq), kSelThreads, stream);
  cfg.dynamicSmemBytes = sizeof(SelSmem) + keys * 4;
  return cudaLaunchKernelEx(&cfg, per_head ? k_mass_select<true> : k_mass_select<false>, pg, b, rows, row0, w, plan, mass);
}

}  // namespace starkv
