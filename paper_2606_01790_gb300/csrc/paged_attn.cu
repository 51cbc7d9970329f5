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
// One bf16 part would round each weight by up to 2^-8, as much as the output's own
// rounding; the second part costs four more products a unit, which the stream of K
// and V covers where a block's rows are few.  (fp16 weights would need V in fp16, which
// holds neither its range nor its small values.)
//
// Even and odd units go to two softmax warpgroups.  A unit's way from its first product
// to the end of its last (S 300 cycles, P V 540, arithmetic and the barriers between)
// takes about 4,000 cycles, so five units are under way, each in a place of its own in
// tensor memory.  Both warpgroups weigh against one reference m per row, which passes
// from unit to unit in order through shared memory (warp to warp); it moves only when a
// unit's maximum lies more than 8 above it, which rescales the row's O.
//
// Query blocks of one drafted tree read the same keys.  Where most sequences have as
// many blocks, a gang of CTAs, one per block, goes through a range of keys at the same
// time, so that the second reader finds them in L2; the flat order, whose readers come
// apart, reads them from memory again.
//
// Pages come by TMA, a box per page (or 64 of its rows); a page number that is none
// lies outside the map and reads as zeros.  Units that not every row of the block sees
// whole take a masked softmax.  A weight of 0 does not keep out a V that is not finite: the
// slots behind the last token, which may hold anything, are zeroed in shared memory, and a
// piece with masked units whose O has elements that are not finite takes those rows
// again, key by key (recompute_rows): what a row does not see then has no part in it, and
// what it sees has its due.  In a piece without masked units such a column is settled by its
// V alone (settle_columns).  (Looking through V of every masked unit beforehand took 1,500
// cycles a unit.)
//
// What bounds it.  Few query rows: the stream of K and V (64 rows of one token, 4.2k keys
// each in sight, 1.07 GB in 166 to 169 us: 94 % of the copy rate).  Many: shared memory and the
// tensor pipe, which a unit keeps busy for 840 of its 1,000 cycles (K once, V twice, the
// loads: 80 KB at some 91 B a cycle); four 56k caches with 64 drafted tokens 240 to 250 us (222
// with the same inputs again and again), tensor pipe 76 % busy, a chunk of 2,704 tokens under a
// window of 4,096 181 to 184 us (172), of which a sixth at the ends of pieces.  Measured when
// these two took 222 and 168 with the same inputs, and not kept: one softmax warpgroup for
// all units (344 and 278 us), two with an O each and three places (232 and 185), one issuer for
// S and P V (291 and 275), waits that spin (276 and 218), five or six stages (2 to 4 % slower),
// rows of O written by bulk copies (5 % slower), range ends moved to the ends of (item, group)s
// (3 % faster for the chunk, 1 % slower for decoding).  The looks for values that are not finite
// take 2 % of the chunk and 0.5 % of decoding; inside the softmax of a unit they took 8 %.
//
// Warp roles: 0 loads K, 3 loads V, 1 issues S and owns tensor memory, 2 issues P V,
// 4..7 and 8..11 softmax.
#include <algorithm>

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
constexpr int kStageO = 32 * 64 * 4;                // a softmax warp's half of O: 32 rows x 64 columns
constexpr int kSoftWarps = 8;                      // four a line (even or odd units)
constexpr uint32_t kFull = 0xffffffffu;
constexpr float kSumLimit = 16384.f;               // largest sum of a unit's 64 weights against a row's reference ...
constexpr float kMoveThreshold = 8.f;              // ... a larger one holds a weight above 2^8
constexpr uint64_t kDrainWaitNs = 2000000000ull;
constexpr float kLeast = 1e-45f;                  // (2^-149)
constexpr uint64_t kAll = ~uint64_t(0);

// Tensor memory, in columns: O 128, S or P 5 x 64 (P: 32 hi, 32 lo), Q 64.
constexpr int kPlaces = 5;
constexpr uint32_t kColO = 0, kColS = 128, kColQ = 448;

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
  uint64_t ref[2][4];               // [line][warp]: the references after its unit are in `m`
  uint64_t qt_full;                 // a piece's queries are in tensor memory
  uint64_t ml_full;                 // both lines' m and l of a piece are in `ml`
  uint64_t o_empty;                 // a piece's O has been read
  uint64_t drain;
  uint32_t tmem_base;
  volatile int abort;
  volatile int beat;                // grows while rows are taken key by key
  int warp_sum[kThreads / 32];
  int items;                        // of the launch: sequences in gangs, else query blocks
  int gang;                         // CTAs of a gang (1: none)
  int64_t sum[2];                   // units, and units times blocks
  volatile float m[1 + kPagedRows]; // [1 + row]: the rows' references, as they pass from unit to unit
  float2 ml[2][2][kPagedRows];      // [piece & 1][line]
  volatile int masked[2][2];        // [piece & 1][line]: a unit of the piece was masked
  int before[kPagedItems + 1];      // units before an item (one KV group)
  Item item[kPagedItems];
};

// Where a unit stands in a ring of N barriers: its place and the parity of its use.
template <int N>
struct Ring {
  int at = 0;
  uint32_t par = 0;
  __device__ __forceinline__ void next() {
    if (++at == N) at = 0, par ^= 1;
  }
};

__device__ __forceinline__ void fail(Ctl* ctl, uint32_t* err) {
  ctl->abort = 1;
  atomicOr(err, kErrTimeout);
}

// A wait of a warp-wide role: true when every lane's barrier completed and, where that
// took time, no role had failed.  The one place where these roles learn of a failure, so
// that a warp's lanes leave together: a barrier that a failed role should have
// completed does not complete.  The limit counts from the last sign of life of rows that are
// taken key by key (recompute_rows and the like): these may take long, but come to an end.
__device__ __forceinline__ bool warp_wait(const Ctl* ctl, uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
  if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
  const bool aborted = ctl->abort;
  bool there = mbar_try_wait(bar, parity);   // (most waits end before a clock is read)
  int beat = ctl->beat;
  for (uint64_t t0 = global_timer_ns(); !there;) {
    there = mbar_try_wait_sleep(bar, parity, 20000u);
    if (there || global_timer_ns() - t0 <= limit_ns) continue;
    if (ctl->beat == beat) break;
    beat = ctl->beat;
    t0 = global_timer_ns();
  }
  return __all_sync(kFull, there && !aborted);
}

// Two of them, at the price of one where both are complete.  They may be looked at in
// either order: each has to be a barrier whose previous phase this warp knows to be
// complete already (a parity cannot tell a phase from the one two before it).
__device__ __forceinline__ bool warp_wait2(const Ctl* ctl, uint64_t* a, uint32_t pa, uint64_t* b, uint32_t pb, uint64_t limit_ns) {
  const bool ra = mbar_try_wait(a, pa), rb = mbar_try_wait(b, pb);
  if (__all_sync(kFull, ra && rb)) return true;
  return warp_wait(ctl, a, pa, limit_ns) && warp_wait(ctl, b, pb, limit_ns);
}

// Instruction descriptor of tcgen05.mma kind::f16 with bf16 A (K-major) and bf16 B
// (MN-major), fp32 accumulator, shape M x N.
__host__ __device__ constexpr uint32_t idesc_bf16_bmn(int M, int N) { return idesc_bf16(M, N) | (1u << 16); }

// x / n by its reciprocal ceil(2^32 / n) (0 for n = 1), for x n < 2^32
__device__ __forceinline__ int quotient(int x, uint32_t inv) {
  return inv ? static_cast<int>(__umulhi(static_cast<uint32_t>(x), inv)) : x;
}

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
  // all of the keys k0 .. k0 + 63 (apart from drafted tokens)
  __device__ __forceinline__ bool whole(int k0) const { return k0 + 64 <= first || (k0 >= lo && k0 + 64 <= hi); }
  __device__ __forceinline__ bool none() const { return first <= 0 && hi <= lo && !bits; }
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

  __device__ __forceinline__ Block(const PagedAttnParams& p, const Item& it, int seq_, int b) : seq(seq_), L(it.L), n(it.n) {
    row0 = b * kPagedRows;
    nrows = min(kPagedRows, n * p.hg - row0);
    tf = quotient(row0, p.inv_hg);
    tl = quotient(row0 + max(nrows, 1) - 1, p.inv_hg);
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
};

// Where a launch finds a sequence's pages, queries and outputs.  Attention over chosen pages
// takes every query of the call as a sequence of one, with the pages chosen for it.
__device__ __forceinline__ const int32_t* entries_of(const PagedAttnParams& p, int seq, int) {
  const int row = p.rows ? p.rows[seq] : p.row0 + seq;
  return p.table + static_cast<int64_t>(row) * p.max_pages;
}
__device__ __forceinline__ const int32_t* entries_of(const SparseAttnParams& p, int seq, int g) {
  return p.list + (static_cast<int64_t>(seq) * p.G + g) * p.n_list;
}

__device__ __forceinline__ int64_t q_at(const PagedAttnParams& p, int seq, int t, int h) {
  return seq * p.q_seq + t * p.q_token + h * p.q_head;
}
__device__ __forceinline__ int64_t o_at(const PagedAttnParams& p, int seq, int t, int h) {
  return seq * p.o_seq + t * p.o_token + h * p.o_head;
}
__device__ __forceinline__ int64_t q_at(const SparseAttnParams& p, int item, int, int h) {
  const int v = p.item0 + item, seq = v / p.tokens;
  return seq * p.q_seq + (v - seq * p.tokens) * p.q_token + h * p.q_head;
}
__device__ __forceinline__ int64_t o_at(const SparseAttnParams& p, int item, int, int h) {
  const int v = p.item0 + item, seq = v / p.tokens;
  return seq * p.o_seq + (v - seq * p.tokens) * p.o_token + h * p.o_head;
}

// A query of a call over chosen pages: a sequence of the tokens that these hold up to its own.
__device__ Item read_item(const SparseAttnParams& p, int item) {
  const int2 x = p.found[item];
  return Item{x.x, x.y};
}

// A sequence's length and queries (read by every CTA: the call may be replayed).
__device__ Item read_item(const PagedAttnParams& p, int seq) {
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
  return it;
}

// Whether the launch goes in gangs, and the units before each item.
template <class Params>
__device__ void count_units(const Params& p, Ctl* ctl) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (p.tree && p.nblk > 1) {
    // A gang of B (the most blocks of a sequence) leaves CTAs idle at sequences with fewer.
    // The flat order leaves none idle but takes about 1.2 times as long a unit, since it reads
    // each block's keys on its own.  Busy for all of the time, gangs took 124 us where the flat order
    // took 143 (32 trees of 36 over 6,000), for 0.76 of it 140 and 131 (ragged, 64), for 0.71 151
    // and 145 (ragged, 26).  CTAs too few for a gang more are idle too: with 80 blocks of four
    // rows of 20,000 gangs (one, 80 of 152 CTAs) took 635, the flat order 379; with 40 (three) 228 and 203.
    int64_t units = 0, work = 0;
    int most = 1;
    for (int seq = tid; seq < p.n; seq += kThreads) {
      const Item it = read_item(p, seq);
      const int nb = (it.n * p.hg + kPagedRows - 1) / kPagedRows, u = Block(p, it, seq, 0).units(p);
      units += u;
      work += static_cast<int64_t>(u) * nb;
      most = max(most, nb);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      units += __shfl_xor_sync(kFull, units, o);
      work += __shfl_xor_sync(kFull, work, o);
      most = max(most, __shfl_xor_sync(kFull, most, o));
    }
    if (lane == 0) {
      atomicAdd(reinterpret_cast<unsigned long long*>(&ctl->sum[0]), static_cast<unsigned long long>(units));
      atomicAdd(reinterpret_cast<unsigned long long*>(&ctl->sum[1]), static_cast<unsigned long long>(work));
      atomicMax(&ctl->gang, most);
    }
    __syncthreads();
    if (tid == 0) {
      const int B = ctl->gang, used = gridDim.x / B * B;   // CTAs in gangs: none if B is more than all
      if (B == 1 || 6 * ctl->sum[1] * used < 5 * ctl->sum[0] * B * static_cast<int64_t>(gridDim.x)) ctl->gang = 1;
    }
    __syncthreads();
  }
  const bool gangs = ctl->gang > 1;
  const int items = gangs ? p.n : p.n * p.nblk;
  constexpr int kPer = (kPagedItems + kThreads - 1) / kThreads;
  int u[kPer];
  int sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int item = tid * kPer + k;
    u[k] = 0;
    if (item >= items) continue;
    const int seq = gangs ? item : quotient(item, p.inv_nblk);
    const Item it = read_item(p, seq);
    ctl->item[item] = it;
    u[k] = Block(p, it, seq, gangs ? 0 : item - seq * p.nblk).units(p);
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
    if (item <= items) ctl->before[item] = at;
    at += u[k];
  }
  if (tid == 0) ctl->items = items;
  __syncthreads();
}

__device__ __forceinline__ int64_t range_begin(int64_t T, int c, int P) { return T * c / P; }

// Ranges of a launch of T units on P CTAs (or gangs): as many, but none empty.  (Fewer and
// longer ones for small launches: a tree of 8 tokens over 2,744, 172 units, 16.9 us with a
// unit a CTA, 18.5 with four; one token over 577, 36 units, 11.4 and 13.8.)
__device__ __forceinline__ int ranges_of(int64_t T, int P) { return T < P ? max(static_cast<int>(T), 1) : P; }

// Range (of P) that holds flat unit f
__device__ __forceinline__ int range_of(int64_t f, int64_t T, int P) { return static_cast<int>(((f + 1) * P - 1) / T); }

// The pieces of a flat range [f0, f1), in order: a run of n units j0, j0 + 1, ... of
// the nu units of one (item, group).  A gang's CTA number `member` has the query block
// `member` of every sequence, and passes over the sequences that have no such block.
struct PieceIter {
  int item, g, j0, n, nu;
  int member;    // -1: no gangs
  int64_t rem;   // units of the range from this piece on
  __device__ __forceinline__ PieceIter(const PagedAttnParams& p, const Ctl* ctl, int member_, int64_t f0, int64_t f1)
      : item(0), g(0), j0(0), n(0), nu(0), member(member_), rem(f1 - f0) {
    if (rem <= 0) return;
    int hi = ctl->items;   // the last item with no more than f0 units before it (items without units are passed over)
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
    if (skipped(p, ctl)) next(p, ctl);
  }
  __device__ __forceinline__ bool valid() const { return rem > 0; }
  __device__ __forceinline__ bool whole() const { return n == nu; }
  __device__ __forceinline__ bool skipped(const PagedAttnParams& p, const Ctl* ctl) const {
    return member > 0 && member * kPagedRows >= ctl->item[item].n * p.hg;
  }
  __device__ __forceinline__ Block block(const PagedAttnParams& p, const Ctl* ctl) const {
    const int seq = member >= 0 ? item : quotient(item, p.inv_nblk);
    return Block(p, ctl->item[item], seq, member >= 0 ? member : item - seq * p.nblk);
  }
  __device__ __forceinline__ void next(const PagedAttnParams& p, const Ctl* ctl) {
    do {
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
    } while (skipped(p, ctl));
  }
};

// A CTA's share: its place in a gang, and its range.
struct Share {
  int member;            // -1: no gangs
  int range, ranges;
  int64_t total, fb, fe;
  __device__ __forceinline__ Share(const PagedAttnParams& p, const Ctl* ctl) {
    const int B = ctl->gang;
    member = B > 1 ? static_cast<int>(blockIdx.x % B) : -1;
    range = blockIdx.x / B;
    total = static_cast<int64_t>(ctl->before[ctl->items]) * p.G;
    ranges = ranges_of(total, gridDim.x / B);
    fb = fe = 0;
    if (range < ranges) {   // (the last CTAs may be too few for a gang, the units too few for all)
      fb = range_begin(total, range, ranges);
      fe = range_begin(total, range + 1, ranges);
    }
  }
};

// ---------------------------------------------------------------- loaders

// K or V loader: the units' pages into a ring.  Lane l holds the number of page
// base + l of the row, so that the table is read once in 32 pages.
template <class Params>
__device__ void load_loop(const Params& p, Ctl* ctl, const CUtensorMap* map, uint8_t* ring, uint64_t* full,
                          uint64_t* empty, int lane, const Share& sh) {
  const uint64_t pol = policy_evict_first();   // a single query block reads K and V once
  const bool once = p.nblk == 1;
  const int P = 1 << p.shift;
  const int boxes = P < kPagedUnitKeys ? kPagedUnitKeys >> p.shift : 1;
  const int box_bytes = min(P, kPagedUnitKeys) * 128;
  int stage = 0;
  uint32_t phase = 0, used = 0, last_ph = 0;   // last_ph: bit s = phase of the last load into stage s
  bool ok = true;
  for (PieceIter c(p, ctl, sh.member, sh.fb, sh.fe); ok && c.valid(); c.next(p, ctl)) {
    const Block blk = c.block(p, ctl);
    const int32_t* entries = entries_of(p, blk.seq, c.g);
    const int held = blk.L < 0 ? 0 : (blk.L + P - 1) >> p.shift;
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

__device__ void mma_s_loop(const PagedAttnParams& p, Ctl* ctl, const uint8_t* sK, uint32_t tmem, const Share& sh) {
  const uint32_t idesc = idesc_bf16(kPagedRows, kPagedUnitKeys);
  const uint64_t dk0 = sdesc_k_sw128(smem_u32(sK));
  Ring<kStages> st;
  Ring<kPlaces> pl;
  int pc = 0;
  bool ok = true;
  for (PieceIter c(p, ctl, sh.member, sh.fb, sh.fe); ok && c.valid(); c.next(p, ctl)) {
    ok = warp_wait(ctl, &ctl->qt_full, pc & 1, p.wait_ns);
    ++pc;
    for (int i = 0; ok && i < c.n; ++i) {
      // (the place's previous P has been used)
      ok = warp_wait2(ctl, &ctl->k_full[st.at], st.par, &ctl->p_empty[pl.at], pl.par ^ 1, p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      const uint64_t dk = dk0 + static_cast<uint64_t>(st.at * (kUnitBytes >> 4));
      const uint32_t s = tmem + kColS + 64 * pl.at;
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          mma_f16_ts(s, tmem + kColQ + kk * 8, dk + ((kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2), idesc, kk > 0);
        mma_commit(&ctl->s_full[pl.at]);
        mma_commit(&ctl->k_empty[st.at]);
      }
      __syncwarp();
      st.next();
      pl.next();
    }
  }
  if (!ok) fail(ctl, p.err);
  // every MMA issued above must be complete before TMEM is released
  if (elect_one()) mma_commit(&ctl->drain);
  mbar_wait(&ctl->drain, 0, drain_limit(p.wait_ns));
  __syncwarp();
}

__device__ void mma_pv_loop(const PagedAttnParams& p, Ctl* ctl, const uint8_t* sV, uint32_t tmem, const Share& sh) {
  const uint32_t idesc = idesc_bf16_bmn(kPagedRows, kHeadDim);
  const uint64_t dv0 = sdesc_mn_sw128(smem_u32(sV), kHalfBytes, 1024);
  Ring<kStages> st;
  Ring<kPlaces> pl;
  int pc = 0;
  bool ok = true;
  for (PieceIter c(p, ctl, sh.member, sh.fb, sh.fe); ok && c.valid(); c.next(p, ctl)) {
    ok = warp_wait(ctl, &ctl->o_empty, (pc & 1) ^ 1, p.wait_ns);   // O of the previous piece has been read
    ++pc;
    for (int i = 0; ok && i < c.n; ++i) {
      ok = warp_wait2(ctl, &ctl->v_full[st.at], st.par, &ctl->p_full[pl.at], pl.par, p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      const uint64_t dv = dv0 + static_cast<uint64_t>(st.at * (kUnitBytes >> 4));
      const uint32_t s = tmem + kColS + 64 * pl.at;
      if (elect_one()) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)   // 16 keys per step: 8 columns of P, 16 rows of V; the piece's first product overwrites O
            mma_f16_ts(tmem + kColO, s + 32 * part + kk * 8, dv + static_cast<uint64_t>(kk * 128), idesc,
                       (i > 0 || part > 0 || kk > 0) ? 1u : 0u);
        mma_commit(&ctl->p_empty[pl.at]);
        mma_commit(&ctl->v_empty[st.at]);
      }
      __syncwarp();
      st.next();
      pl.next();
    }
  }
  if (!ok) fail(ctl, p.err);
  if (elect_one()) mma_commit(&ctl->drain);
  mbar_wait(&ctl->drain, 0, drain_limit(p.wait_ns));
  __syncwarp();
}

// ---------------------------------------------------------------- softmax

// 32 keys of a unit, exp2 arguments and sums as packed pairs; p = hi + lo, hi the
// upper 16 bits of p.
__device__ __forceinline__ void exp_split(const uint32_t (&z)[32], float2 sc2, float2 nm2, float2 (&acc)[4], uint32_t (&hi)[16],
                                          uint32_t (&lo)[16]) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const float2 e = ffma2(make_float2(__uint_as_float(z[i]), __uint_as_float(z[i + 1])), sc2, nm2);
    const float p0 = ex2_approx(e.x), p1 = ex2_approx(e.y);
    acc[(i >> 1) & 3] = fadd2(acc[(i >> 1) & 3], make_float2(p0, p1));
    const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
    hi[i >> 1] = __byte_perm(u0, u1, 0x7632);
    const float2 rest = fadd2(make_float2(p0, p1), make_float2(-__uint_as_float(u0 & 0xFFFF0000u), -__uint_as_float(u1 & 0xFFFF0000u)));
    const __nv_bfloat162 r = __floats2bfloat162_rn(rest.x, rest.y);
    lo[i >> 1] = *reinterpret_cast<const uint32_t*>(&r);
  }
}

// What runs once or twice a piece is kept in short loops over 16 columns: code that is
// not in the instruction cache costs about ten cycles an instruction, and unrolled over a
// unit a masked softmax took 2,600 and a second pass 5,300 cycles.

// Largest raw logit of a unit.
__device__ __forceinline__ float unit_max(uint32_t s_addr) {
  float mx = -INFINITY;
#pragma unroll 1
  for (int c = 0; c < kPagedUnitKeys; c += 16) {
    uint32_t z[16];
    tmem_ld16_async(s_addr + c, z);
    tmem_wait16(z);
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, __uint_as_float(z[i]));
  }
  return mx;
}

// S = -inf at the keys that this thread's row does not see (bits of `vis` clear).
__device__ __forceinline__ void mask_s(uint32_t s_addr, uint64_t vis) {
#pragma unroll 1
  for (int c = 0; c < kPagedUnitKeys; c += 16) {
    uint32_t z[16];
    tmem_ld16_async(s_addr + c, z);
    tmem_wait16(z);
    const uint32_t bits = static_cast<uint32_t>(vis >> c);
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = bits >> i & 1 ? z[i] : 0xFF800000u;
    tmem_st16(s_addr + c, z);
  }
  tmem_wait_st();
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

// P of a unit against `ref`; returns the sum.
__device__ __forceinline__ float weights(const uint32_t (&z)[2][32], float c2, float ref, uint32_t (&hi)[2][16], uint32_t (&lo)[2][16]) {
  const float2 sc2 = make_float2(c2, c2), nm2 = make_float2(-ref, -ref);
  float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
  for (int k = 0; k < 2; ++k) exp_split(z[k], sc2, nm2, acc, hi[k], lo[k]);
  const float2 a = fadd2(fadd2(acc[0], acc[1]), fadd2(acc[2], acc[3]));
  return a.x + a.y;
}

__device__ __forceinline__ void load_s(uint32_t s_addr, uint32_t (&z)[2][32]) {
  tmem_ld32_async(s_addr, z[0]);
  tmem_ld32_async(s_addr + 32, z[1]);
  tmem_wait32(z[0]);
  tmem_wait32(z[1]);
}

// One unit of a softmax warp with rows: S into registers, P in its place.
//
// The weights are taken against the reference m that the line knows, without looking for
// the unit's maximum.  Before they are used, the reference that holds after the unit
// before (the other line's warp of these rows passes it on) has to be that one, and no
// row's sum may be large: otherwise (the piece's first unit, a rising maximum) they are
// taken again, against a reference that the unit's maximum moves where it lies more
// than 8 above it; the row of O is rescaled once the previous unit's product is done.  (A
// reference far above a unit's logits does no harm: the weights keep their relative
// precision, and those below 2^-126 of the largest seen so far are nothing.)  l counts
// against m.  `unit`: its number in the piece.  Returns false when a wait ran out.
__device__ __forceinline__ bool softmax_unit(const PagedAttnParams& p, Ctl* ctl, uint64_t* ref_in, uint32_t ref_par, uint64_t* ref_out,
                                             uint64_t* prev_empty, uint32_t prev_par, volatile float* slot, int lane, bool live, int unit,
                                             bool masked, uint64_t vis, uint32_t s_addr, uint32_t o_addr, float& m, float& l) {
  const float c2 = p.scale2;
  if (masked) mask_s(s_addr, vis);
  uint32_t hi[2][16], lo[2][16];
  float sum, was = live ? -INFINITY : 0.f;   // (rows that are none weigh against 0 and never ask for more)
  bool again = unit == 0;                    // (nothing to weigh against)
  if (unit == 1) {                           // the line's first: nothing known yet
    if (!warp_wait(ctl, ref_in, ref_par, p.wait_ns)) return false;
    m = *slot;
  }
#pragma unroll 1
  while (true) {
    if (again) {
      const float mx = unit_max(s_addr) * c2;
      const bool first = was == -INFINITY, move = live && !first && mx > was + kMoveThreshold;
      if (__any_sync(kFull, move)) {
        if (!warp_wait(ctl, prev_empty, prev_par, p.wait_ns)) return false;
        tc_fence_after();
        rescale_o(o_addr, move ? ex2_approx(was - mx) : 1.f);
        tmem_wait_st();
      }
      const float now = first || move ? mx : was;
      l = now == m || m == -INFINITY ? l : l * ex2_approx(m - now);   // (l is 0 while m is -inf)
      m = now;
      *slot = now;
      __syncwarp();
    }
    uint32_t z[2][32];
    load_s(s_addr, z);
    sum = weights(z, c2, m == -INFINITY ? 0.f : m, hi, lo);
    if (again) break;
    // The slot is read only once the barrier has been seen complete: its address depends
    // on the answer (in front of row 0 lies a slot that is nobody's), since a load that
    // merely stands behind the question may be served before it.
    const bool in = mbar_try_wait(ref_in, ref_par);
    was = slot[static_cast<int>(in) - 1];
    if (!__any_sync(kFull, !in || was != m || was == -INFINITY || !(sum <= kSumLimit))) break;
    if (!warp_wait(ctl, ref_in, ref_par, p.wait_ns)) return false;
    was = *slot;
    if (!__any_sync(kFull, was != m || was == -INFINITY || !(sum <= kSumLimit))) break;
    again = true;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    tmem_st16(s_addr + 16 * k, hi[k]);
    tmem_st16(s_addr + 32 + 16 * k, lo[k]);
  }
  if (lane == 0) mbar_arrive(ref_out);
  l += sum;
  return true;
}

// 16-byte chunk c (of 16) of row i of a warp's staged half of O: rows of 64 floats, the
// chunks in an order that depends on the row, so that neither lanes on rows nor lanes on
// columns meet in a bank.
__device__ __forceinline__ float4* staged(float* stage, int i, int c) {
  return reinterpret_cast<float4*>(stage) + i * 16 + (c ^ (i & 15));
}

__device__ __forceinline__ float4 bf16x4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xFFFF0000u));
}

__device__ __forceinline__ bool is_inf(float x) { return fabsf(x) == INFINITY; }
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }

// w x for a weight w >= 0 that stands for one above 0, however small
__device__ __forceinline__ float weighted(float w, float x) { return is_inf(x) ? x : w * x; }

// A piece that every row sees whole, where O has elements that are not finite: every weight is above 0,
// so that a column with a V of infinity comes to infinity, with both or a NaN to NaN, whatever the weights
// (products of their parts say otherwise where a part is 0: 0 * infinity).  Columns col .. col + 63 of the
// staged rows `which`, by the whole warp, each lane two columns over all keys.
template <class Params>
__device__ __noinline__ void settle_columns(const Params& p, Ctl* ctl, const Block& blk, int g, int j0, int n, int col, uint32_t which,
                                            float* stage) {
  const int lane = threadIdx.x & 31;
  const int32_t* entries = entries_of(p, blk.seq, g);
  float2 sum = make_float2(0.f, 0.f);   // of the column's infinities and NaNs: 0 where it has none
  for (int j = j0; j < j0 + n; ++j) {
    const int k0 = blk.key(j);
    if (lane == 0) atomicAdd(const_cast<int*>(&ctl->beat), 1);
#pragma unroll 1
    for (int k1 = k0; k1 < k0 + kPagedUnitKeys; k1 += 16) {
      const int page = entries[k1 >> p.shift];   // (a page has 16 slots or more)
      if (page < 0 || page >= p.n_pages) continue;
      const __nv_bfloat16* v =
          p.v + page * p.page_stride + ((static_cast<int64_t>(g) << p.shift) + (k1 & ((1 << p.shift) - 1))) * kHeadDim + col + 2 * lane;
      uint32_t w[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) w[u] = *reinterpret_cast<const uint32_t*>(v + u * kHeadDim);
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const float x = __uint_as_float(w[u] << 16), y = __uint_as_float(w[u] & 0xFFFF0000u);
        sum.x += is_finite(x) ? 0.f : x;
        sum.y += is_finite(y) ? 0.f : y;
      }
    }
  }
  for (; which; which &= which - 1) {
    float2* o = &reinterpret_cast<float2*>(staged(stage, __ffs(which) - 1, lane >> 1))[lane & 1];
    if (sum.x != 0.f) o->x = sum.x;
    if (sum.y != 0.f) o->y = sum.y;
  }
}

// Columns col .. col + 63 of the staged rows `which` (bits) of a warp's 32, from row r0 of
// the block on, over the piece's keys: by the whole warp, one row and one key at a
// time, skipping the keys that the row does not see.  Against the reference `top` of the
// row (lane i: row i), times `norm` (the same).  Some microseconds a row and 64 keys, so that
// every unit is a sign of life for the roles that wait.
template <class Params>
__device__ __noinline__ void recompute_rows(const Params& p, Ctl* ctl, const Block& blk, int g, int j0, int n, int r0, int col, uint32_t which,
                                            float top, float norm, float* stage) {
  const int lane = threadIdx.x & 31;
  const int32_t* entries = entries_of(p, blk.seq, g);
  for (; which; which &= which - 1) {
    const int i = __ffs(which) - 1;
    const int t = quotient(blk.row0 + r0 + i, p.inv_hg), h = g * p.hg + blk.row0 + r0 + i - t * p.hg;
    const Seen see = blk.row(p, blk.L - blk.n + t, p.tree ? p.mask[static_cast<int64_t>(blk.seq) * p.T + t] : 0);
    const float4 q = bf16x4(p.q + q_at(p, blk.seq, t, h) + 4 * lane);
    const float ref = __shfl_sync(kFull, top, i), scale = __shfl_sync(kFull, norm, i);
    float2 acc = make_float2(0.f, 0.f);
    for (int j = j0; j < j0 + n; ++j) {
      const int k0 = blk.key(j);
      if (lane == 0) atomicAdd(const_cast<int*>(&ctl->beat), 1);
      for (uint64_t bits = see(k0); bits;) {
        float4 k[8];   // eight keys' loads at once: their latency is most of this path's time
        float2 v[8];
        bool any[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          any[u] = bits != 0;
          const int key = k0 + __ffsll(static_cast<long long>(bits)) - 1;
          bits &= bits - 1;
          k[u] = make_float4(0.f, 0.f, 0.f, 0.f);   // (a page number that is none: zeros)
          v[u] = make_float2(0.f, 0.f);
          const int page = any[u] ? entries[key >> p.shift] : -1;
          if (page >= 0 && page < p.n_pages) {
            const int64_t at = page * p.page_stride + ((static_cast<int64_t>(g) << p.shift) + (key & ((1 << p.shift) - 1))) * kHeadDim;
            k[u] = bf16x4(p.k + at + 4 * lane);
            const uint32_t w = *reinterpret_cast<const uint32_t*>(p.v + at + col + 2 * lane);
            v[u] = make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
          }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          float z = q.x * k[u].x + q.y * k[u].y + q.z * k[u].z + q.w * k[u].w;
#pragma unroll
          for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(kFull, z, o);
          const float e = exp2f(z * p.scale2 - ref);
          const float some = z > -INFINITY ? fmaxf(e, kLeast) : e;   // (a weight is 0 in fp32 only)
          if (any[u]) acc = make_float2(acc.x + (is_inf(v[u].x) ? some : e) * v[u].x, acc.y + (is_inf(v[u].y) ? some : e) * v[u].y);
        }
      }
    }
    reinterpret_cast<float2*>(staged(stage, i, lane >> 1))[lane & 1] = make_float2(acc.x * scale, acc.y * scale);
  }
}

// Rows `which` of a warp's 32 (from row r0 of the block on), whose largest logit is +inf: those with a logit
// that is NaN among the piece's keys, as bits.  (Their sums are NaN either way: inf - inf.)
template <class Params>
__device__ __noinline__ uint32_t rows_with_nan(const Params& p, Ctl* ctl, const Block& blk, int g, int j0, int n, int r0, uint32_t which) {
  const int lane = threadIdx.x & 31;
  const int32_t* entries = entries_of(p, blk.seq, g);
  uint32_t found = 0;
  for (; which; which &= which - 1) {
    const int i = __ffs(which) - 1;
    const int t = quotient(blk.row0 + r0 + i, p.inv_hg), h = g * p.hg + blk.row0 + r0 + i - t * p.hg;
    const Seen see = blk.row(p, blk.L - blk.n + t, p.tree ? p.mask[static_cast<int64_t>(blk.seq) * p.T + t] : 0);
    const float4 q = bf16x4(p.q + q_at(p, blk.seq, t, h) + 4 * lane);
    for (int j = j0; j < j0 + n; ++j) {
      const int k0 = blk.key(j);
      if (lane == 0) atomicAdd(const_cast<int*>(&ctl->beat), 1);
      for (uint64_t bits = see(k0); bits;) {
        float4 k[8];   // eight keys' loads at once
        bool any[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          any[u] = bits != 0;
          const int key = k0 + __ffsll(static_cast<long long>(bits)) - 1;
          const int page = any[u] ? entries[key >> p.shift] : -1;
          bits &= bits - 1;
          k[u] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (page >= 0 && page < p.n_pages)
            k[u] = bf16x4(p.k + page * p.page_stride + ((static_cast<int64_t>(g) << p.shift) + (key & ((1 << p.shift) - 1))) * kHeadDim + 4 * lane);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          float z = q.x * k[u].x + q.y * k[u].y + q.z * k[u].z + q.w * k[u].w;
#pragma unroll
          for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(kFull, z, o);
          if (any[u] && z != z) found |= 1u << i;
        }
      }
    }
  }
  return found;
}

// Softmax warps of a line (0: even units, 1: odd): one thread per query row (TMEM lane
// quad * 32 + lane).
template <class Params>
__device__ void softmax_loop(const Params& p, Ctl* ctl, uint8_t* sV, float* stage_o, uint32_t tmem, int line, int quad, int lane,
                             const Share& sh) {
  const int r = quad * 32 + lane;
  const uint32_t lane_base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
  const uint32_t o_addr = lane_base + kColO;
  uint32_t u0 = 0;   // number of the piece's first unit
  // line 0: the queries of a piece (no product reads the previous piece's any more)
  auto take_queries = [&](const PieceIter& c) {
    const Block blk = c.block(p, ctl);
    if (quad * 32 < blk.nrows) {
      const bool live = r < blk.nrows;
      const int t = quotient(blk.row0 + r, p.inv_hg), h = c.g * p.hg + blk.row0 + r - t * p.hg;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + q_at(p, blk.seq, t, h));
      uint4 w[16];   // every load before the first use
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = live ? src[i] : make_uint4(0u, 0u, 0u, 0u);
      __syncwarp();   // (`live` differs between lanes)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t x[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * i] = w[4 * k + i].x, x[4 * i + 1] = w[4 * k + i].y, x[4 * i + 2] = w[4 * k + i].z, x[4 * i + 3] = w[4 * k + i].w;
        tmem_st16(lane_base + kColQ + 16 * k, x);
      }
      tmem_wait_st();
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl->qt_full);
  };
  bool ok = true;
  int pc = 0;
  PieceIter c(p, ctl, sh.member, sh.fb, sh.fe);
  if (line == 0 && c.valid()) take_queries(c);
  for (; ok && c.valid(); ++pc) {
    bool any_masked = false;
    const Block blk = c.block(p, ctl);
    const bool wactive = quad * 32 < blk.nrows;
    const bool live = r < blk.nrows;
    const int t = quotient(blk.row0 + r, p.inv_hg), h = c.g * p.hg + blk.row0 + r - t * p.hg;
    const Seen all = blk.all(p);
    const uint64_t* masks = p.mask + static_cast<int64_t>(blk.seq) * p.T;
    Seen see = blk.row(p, blk.L - blk.n + t, p.tree && live ? masks[t] : 0);
    if (!live) see = Seen{0, 0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    for (int i = (u0 ^ static_cast<uint32_t>(line)) & 1; i < c.n; i += 2) {
      const uint32_t ui = u0 + i, pl = ui % kPlaces, up = ui - 1;
      const uint32_t s_addr = lane_base + kColS + 64 * pl;
      ok = warp_wait(ctl, &ctl->s_full[pl], ui / kPlaces & 1, p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      const int k0 = blk.key(c.j0 + i);
      const bool masked = !all.whole(k0);
      if (wactive) {
        ok = softmax_unit(p, ctl, &ctl->ref[line ^ 1][quad], up >> 1 & 1, &ctl->ref[line][quad], &ctl->p_empty[up % kPlaces],
                          up / kPlaces & 1, &ctl->m[1 + r], lane, live, i, masked, masked ? see(k0) : kAll, s_addr, o_addr, m, l);
      } else if (lane == 0) {   // a warp without rows only keeps the counts
        mbar_arrive(&ctl->ref[line][quad]);
      }
      if (masked) {
        any_masked = true;
        if (ok && k0 + kPagedUnitKeys > blk.L) {
          // The slots behind the last token.  V of this unit is asked for only once the stage's
          // previous V has been used: S runs further ahead than the ring of V is deep, and a
          // parity says nothing of a load while the one before it is still under way
          const uint32_t before = ui - kStages;
          if (ui >= kStages) ok = warp_wait(ctl, &ctl->p_empty[before % kPlaces], before / kPlaces & 1, p.wait_ns);
          const int stage = ui % kStages;
          ok = ok && warp_wait(ctl, &ctl->v_full[stage], ui / kStages & 1, p.wait_ns);
          if (!ok) break;
          uint4* v4 = reinterpret_cast<uint4*>(sV + stage * kUnitBytes);
          for (int x = (max(blk.L, k0) - k0) * 8 + r; x < kUnitBytes / 32; x += 128)   // 8 chunks of 16 bytes a key, in each half
            v4[x] = v4[x + kUnitBytes / 32] = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
        }
      }
      if (!ok) break;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl->p_full[pl]);
    }
    if (!ok) break;
    const uint32_t lu = u0 + c.n - 1, lpl = lu % kPlaces, lpar = lu / kPlaces & 1;
    // both lines' references and sums, and O
    ctl->ml[pc & 1][line][r] = make_float2(m, l);
    __syncwarp();
    if (lane == 0) {
      ctl->masked[pc & 1][line] = any_masked;   // (the same from each of the line's warps)
      mbar_arrive(&ctl->ml_full);
    }
    PieceIter nx = c;
    nx.next(p, ctl);
    if (line == 0 && nx.valid()) {   // S of the next piece runs under this piece's end
      ok = warp_wait(ctl, &ctl->s_full[lpl], lpar, p.wait_ns);
      if (!ok) break;
      tc_fence_after();
      take_queries(nx);
    }
    // (one after the other: until both lines are through, the last unit's place may not have
    // come round, and its parity would speak of the use before)
    ok = warp_wait(ctl, &ctl->ml_full, pc & 1, p.wait_ns) && warp_wait(ctl, &ctl->p_empty[lpl], lpar, p.wait_ns);
    if (!ok) break;
    tc_fence_after();
    if (wactive) {
      const bool whole = c.whole();
      const float2 other = ctl->ml[pc & 1][line ^ 1][r];
      const float M = fmaxf(m, other.x), ref = M == -INFINITY ? 0.f : M;   // (the last reference is the largest)
      float L = exp2f(m - ref) * l + exp2f(other.x - ref) * other.y;
      const float norm = !whole ? 1.f : L != 0.f ? 1.f / L : see.none() ? 0.f : NAN;   // (0 / 0 where every logit is -inf)
      const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (c.j0 == 0);
      // this line's half of the columns by way of shared memory, for rows that are written whole
      uint32_t a[2][32];
      load_s(o_addr + 64 * line, a);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t* x = &a[i >> 3][4 * (i & 7)];
        *staged(stage_o, lane, i) = make_float4(__uint_as_float(x[0]) * norm, __uint_as_float(x[1]) * norm, __uint_as_float(x[2]) * norm,
                                                __uint_as_float(x[3]) * norm);
      }
      float sum[4] = {0.f, 0.f, 0.f, 0.f};   // 0, or NaN where O is not finite
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        sum[i & 1] = fmaf(__uint_as_float(a[0][i]), 0.f, sum[i & 1]);
        sum[2 + (i & 1)] = fmaf(__uint_as_float(a[1][i]), 0.f, sum[2 + (i & 1)]);
      }
      const bool odd = live && (sum[0] + sum[1]) + (sum[2] + sum[3]) != 0.f;
      if (__any_sync(kFull, odd)) {
        __syncwarp();   // (rows that other lanes staged are written again)
        // (a logit that is NaN or +inf has all of its row's columns NaN, as they are to be, and L too)
        const uint32_t infinite = __ballot_sync(kFull, odd && M == INFINITY && line == 0);   // (the line that writes L)
        if (infinite) {
          const uint32_t nan = rows_with_nan(p, ctl, blk, c.g, c.j0, c.n, quad * 32, infinite);
          if (M == INFINITY) L = nan >> lane & 1 ? NAN : 1.f;   // lse is +inf where no logit is NaN
        }
        const uint32_t which = __ballot_sync(kFull, odd && L == L && M < INFINITY);
        if (which && (ctl->masked[pc & 1][0] | ctl->masked[pc & 1][1]))
          recompute_rows(p, ctl, blk, c.g, c.j0, c.n, quad * 32, 64 * line, which, ref, norm, stage_o);
        else if (which)
          settle_columns(p, ctl, blk, c.g, c.j0, c.n, 64 * line, which, stage_o);
      }
      __syncwarp();
      const int rows = min(32, blk.nrows - quad * 32);
      if (whole) {
        const int64_t at = o_at(p, blk.seq, t, h) + 64 * line;   // this lane's row
#pragma unroll 4
        for (int i = lane >> 3; i < 32; i += 4) {   // eight lanes a row, eight columns each
          const int64_t to = __shfl_sync(kFull, at, i);
          if (i >= rows) continue;
          const float4 a = *staged(stage_o, i, 2 * (lane & 7)), b = *staged(stage_o, i, 2 * (lane & 7) + 1);
          const __nv_bfloat162 x[4] = {__floats2bfloat162_rn(a.x, a.y), __floats2bfloat162_rn(a.z, a.w), __floats2bfloat162_rn(b.x, b.y),
                                       __floats2bfloat162_rn(b.z, b.w)};
          *reinterpret_cast<uint4*>(p.o + to + 8 * (lane & 7)) = *reinterpret_cast<const uint4*>(x);
        }
      } else {
        float* part = p.part_o + (slot * kPagedRows + quad * 32) * kHeadDim + 64 * line + 4 * (lane & 15);
#pragma unroll 4
        for (int i = lane >> 4; i < rows; i += 2) *reinterpret_cast<float4*>(part + i * kHeadDim) = *staged(stage_o, i, lane & 15);
      }
      if (live && line == 0) {
        if (!whole) p.part_ml[slot * kPagedRows + r] = make_float2(M, L);
        else if (p.lse)
          p.lse[(static_cast<int64_t>(blk.seq) * p.T + t) * p.H + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
      }
    }
    tc_fence_before();
    __syncwarp();   // (also: the staged rows have been read)
    if (lane == 0) mbar_arrive(&ctl->o_empty);
    u0 += c.n;
    c = nx;
  }
  if (!ok) fail(ctl, p.err);
}

}  // namespace

template <class Params>
__global__ void __launch_bounds__(kThreads, 1) k_paged_attn(const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem;                           // [kStages][2 halves][64 keys][128 B]
  uint8_t* sV = sK + kStages * kUnitBytes;      // the same
  float* sO = reinterpret_cast<float*>(sV + kStages * kUnitBytes);   // [8 softmax warps][32 rows][64 columns]
  Ctl* ctl = reinterpret_cast<Ctl*>(reinterpret_cast<uint8_t*>(sO) + kStageO * kSoftWarps);
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
    for (int i = 0; i < 8; ++i) mbar_init(&ctl->ref[i >> 2][i & 3], 1);
    mbar_init(&ctl->qt_full, kSoftWarps / 2);
    mbar_init(&ctl->ml_full, kSoftWarps);
    mbar_init(&ctl->o_empty, kSoftWarps);
    mbar_init(&ctl->drain, 2);   // one commit per MMA issuer
    ctl->abort = ctl->beat = 0;
    ctl->gang = 1;
    ctl->sum[0] = ctl->sum[1] = 0;
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
  const Share sh(p, ctl);

  if (warp == 0) {
    load_loop(p, ctl, &p.tmk, sK, ctl->k_full, ctl->k_empty, lane, sh);
  } else if (warp == 3) {
    load_loop(p, ctl, &p.tmv, sV, ctl->v_full, ctl->v_empty, lane, sh);
  } else if (warp == 1) {
    mma_s_loop(p, ctl, sK, tmem, sh);
  } else if (warp == 2) {
    mma_pv_loop(p, ctl, sV, tmem, sh);
  } else {
    softmax_loop(p, ctl, sV, sO + (warp - 4) * (kStageO / 4), tmem, (warp - 4) >> 2, warp & 3, lane, sh);
  }
  if (threadIdx.x == 0) {   // what the merge has to know of this range's end
    PagedSplit s;
    s.total = sh.total;
    s.valid = 0;
    s.gang = ctl->gang;
    if (sh.fe > sh.fb) {   // the piece that the range's last unit is in, if it begins here and goes on
      const PieceIter e(p, ctl, sh.member, sh.fe - 1, sh.fe);
      if (e.valid()) {
        const int64_t f0 = static_cast<int64_t>(ctl->before[e.item]) * p.G + static_cast<int64_t>(e.g) * e.nu;
        if (f0 >= sh.fb && f0 + e.nu > sh.fe) {
          const Block blk = e.block(p, ctl);
          s.valid = 1;
          s.seq = blk.seq;
          s.row0 = blk.row0;
          s.nrows = blk.nrows;
          s.g = e.g;
          s.last = range_of(f0 + e.nu - 1, sh.total, sh.ranges);
        }
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
// l, O = sum 2^(m - M) O_part / L, lse = (M + log2 L) ln 2.  Block (c, y): the one that range
// c began, 8 / WARPS query rows from there on; the WARPS warps of a row take every
// WARPS-th part, four at a time (their loads are in flight before the first is used), and
// the first adds up what they found.  (paged_combine_launch chooses WARPS.)
constexpr int kBatch = 4;

// 2^(m - ref) for m <= ref, also where both are infinite
__device__ __forceinline__ float decay(float m, float ref) { return m == ref ? 1.f : exp2f(m - ref); }

__device__ __forceinline__ float4 scaled(float w, const float4& o) {
  return make_float4(weighted(w, o.x), weighted(w, o.y), weighted(w, o.z), weighted(w, o.w));
}
__device__ __forceinline__ float4 sum_of(const float4& a, const float4& b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

template <int WARPS, class Params>
__global__ void __launch_bounds__(256) k_paged_combine(const __grid_constant__ Params p) {
  __shared__ float2 s_ml[8];
  __shared__ float4 s_o[8][32];
  griddep_launch_dependents();
  griddep_wait();
  const PagedSplit s = p.split[blockIdx.x];
  if (!s.valid) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = blockIdx.x / s.gang, member = blockIdx.x % s.gang;
  const int r = blockIdx.y * (8 / WARPS) + warp / WARPS;
  const bool live = r < s.nrows;
  if (WARPS == 1 && !live) return;
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int cb = first + warp % WARPS; live && cb <= s.last; cb += kBatch * WARPS) {
    float2 ml[kBatch];
    float4 o[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int c = cb + k * WARPS;
      ml[k] = make_float2(-INFINITY, 0.f);
      o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c > s.last) continue;
      const int64_t at = (2 * (static_cast<int64_t>(c) * s.gang + member) + (c == first)) * kPagedRows + r;
      ml[k] = p.part_ml[at];
      o[k] = reinterpret_cast<const float4*>(p.part_o + at * kHeadDim)[lane];
    }
    float top = M;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = fmaxf(top, ml[k].x);
    const float ref = top == -INFINITY ? 0.f : top, keep = decay(M, ref);
    M = top;
    L *= keep;
    acc = scaled(keep, acc);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float w = decay(ml[k].x, ref);
      L += w * ml[k].y;
      acc = sum_of(acc, scaled(w, o[k]));
    }
  }
  if (WARPS > 1) {
    s_ml[warp] = make_float2(M, L);
    s_o[warp][lane] = acc;
    __syncthreads();
    if (!live || warp % WARPS != 0) return;
    float top = M;
#pragma unroll
    for (int k = 1; k < WARPS; ++k) top = fmaxf(top, s_ml[warp + k].x);
    const float ref = top == -INFINITY ? 0.f : top, keep = decay(M, ref);
    M = top;
    L *= keep;
    acc = scaled(keep, acc);
#pragma unroll
    for (int k = 1; k < WARPS; ++k) {
      const float w = decay(s_ml[warp + k].x, ref);
      L += w * s_ml[warp + k].y;
      acc = sum_of(acc, scaled(w, s_o[warp + k][lane]));
    }
  }
  const int t = quotient(s.row0 + r, p.inv_hg), h = s.g * p.hg + s.row0 + r - t * p.hg;
  float inv = 1.f / L;
  if (L == 0.f) {   // no key seen, or every logit -inf
    const Block blk(p, read_item(p, s.seq), s.seq, s.row0 / kPagedRows);
    inv = blk.row(p, blk.L - blk.n + t, p.tree ? p.mask[static_cast<int64_t>(s.seq) * p.T + t] : 0).none() ? 0.f : NAN;
  }
  const __nv_bfloat162 x[2] = {__floats2bfloat162_rn(acc.x * inv, acc.y * inv), __floats2bfloat162_rn(acc.z * inv, acc.w * inv)};
  *reinterpret_cast<uint2*>(p.o + o_at(p, s.seq, t, h) + lane * 4) = *reinterpret_cast<const uint2*>(x);
  if (p.lse && lane == 0)
    p.lse[(static_cast<int64_t>(s.seq) * p.T + t) * p.H + h] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

namespace {

constexpr size_t kSmemBytes = 1024 + 2 * static_cast<size_t>(kStages) * kUnitBytes + kStageO * kSoftWarps + sizeof(Ctl);
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
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  const cudaError_t e = cudaFuncSetAttribute(k_paged_attn<PagedAttnParams>, attr, static_cast<int>(kSmemBytes));
  return e != cudaSuccess ? e : cudaFuncSetAttribute(k_paged_attn<SparseAttnParams>, attr, static_cast<int>(kSmemBytes));
}

namespace {

template <class Params>
cudaError_t attn_launch(const Params& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = config(attr, dim3(p.grid), kThreads, kSmemBytes, stream);
  return cudaLaunchKernelEx(&cfg, k_paged_attn<Params>, p);
}

template <class Params>
cudaError_t combine_launch(const Params& p, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  // one warp a row, but four where few rows meet more than 16 parts: one tree of 8 tokens (56
  // rows, 38 parts) 16.9 us so, 19.8 with one; of 18 (126 rows) 23.3 with four, 21.5 with one; four
  // trees of 8 (10 parts) 20.1 and 18.7; one of 60 (four blocks, 10 parts) 30.3 and 24.9
  const int rows = std::min(kPagedRows, p.T * p.hg);
  const bool many = p.n * p.nblk * p.G * 16 >= p.grid || rows > 64;
  const int per = many ? 8 : 2;
  cudaLaunchConfig_t cfg = config(attr, dim3(p.grid, (rows + per - 1) / per), 256, 0, stream);
  return cudaLaunchKernelEx(&cfg, many ? k_paged_combine<1, Params> : k_paged_combine<4, Params>, p);
}

}  // namespace

cudaError_t paged_attn_launch(const PagedAttnParams& p, cudaStream_t stream) { return attn_launch(p, stream); }
cudaError_t paged_attn_launch(const SparseAttnParams& p, cudaStream_t stream) { return attn_launch(p, stream); }
cudaError_t paged_combine_launch(const PagedAttnParams& p, cudaStream_t stream) { return combine_launch(p, stream); }
cudaError_t paged_combine_launch(const SparseAttnParams& p, cudaStream_t stream) { return combine_launch(p, stream); }

}  // namespace starkv
