// The paged cache: page tables, reference counts and the copies they call for.
//
// A token's keys and values of every layer and KV head lie under one page
// number; row r of the table lists the pages of a sequence in order and refs[p]
// counts the rows that hold page p (0: free).  Sharing a page is counting it once
// more, so that a branch costs a table row; what a row may write it holds alone
// (the last page is copied before tokens are added to a shared one).
//
// k_book: one cluster of eight 1024-thread CTAs.  Every CTA reads the call's rows
// (at most one per thread), checks them and adds up their needs, so that all come
// to the same verdict; its eighth of the counts becomes one bit per page.  After
// the only exchange, the number of free pages per CTA (written into the peers' shared
// memory once all of them are known to run), the a-th free page
// (lowest number first) belongs to the a-th need: results do not depend on the
// order in which threads run.  The call is carried out as a whole or not at all: the
// pages that its rows hold are looked at, an eighth of them per CTA, before anything
// changes, and a CTA that finds a wrong one says so in the same exchange.  A refused
// call sets kErrHeld, which holds back every call after it that changes a pool: a store
// queued behind an extend that found no page would write over the row's last tokens.
//
// What bounds it is a chain of memory waits (row, length, table, count), two sums over
// the block and the cluster barrier (0.7 us): 4 us a call of 64 rows for fork and free,
// launches one after another (0.8 of it for looking at the held pages first).  extend and
// compact read every count, through eight SMs: extend with its copies 4.9 us in a pool of
// 4,096 pages, 12 in 300,000, 30 in 2^20.
//
// The copies move 256-byte rows (d = 128 bf16) as k_compact does: a warp task is
// 32 rows, whose places its lanes resolve; 16-byte accesses, eight per lane in
// flight, past L1.  Bound by HBM: 28 layers of a 2,736-token row gathered, stored or
// loaded (314 MB read and written) in 50 us, 6.3 TB/s, 93 % of the copy rate; the filled slots
// of 64 shared pages (290 MB) in 45; rows of 256 bytes kept per KV head, in no order, 6.2 TB/s.
#include "common.cuh"
#include "pages.cuh"
#include "ptx.cuh"

namespace starkv {

namespace {

constexpr int kBookThreads = 1024;
constexpr int kBookCtas = 8;
constexpr int kSliceWords = kMaxPages / 32 / kBookCtas;   // free-page words of a CTA, at most
constexpr uint32_t kFull = 0xffffffffu;

struct BookSmem {
  int off[kMaxCallRows + 1];    // new pages before row i
  int held[kMaxCallRows + 1];   // pages held before row i
  int row[kMaxCallRows];
  int from[kMaxCallRows];       // fork: the row it branches from
  int pos[kMaxCallRows];        // table position of the row's first new page
  int len[kMaxCallRows];        // tokens before the call (fork: of the row branched from)
  uint32_t bits[kSliceWords];   // free pages of this CTA's part
  int before[kSliceWords];      // free pages before a word, in this CTA's part
  uint32_t seen[kMaxTableRows / 32];   // rows named so far
  int2 warp_sum[32];
  int count[kBookCtas];         // free pages of each CTA's part; -1: a page there that no row can hold; -2 (CTA 0): held back
  int bad;
  uint32_t hold;   // CTA 0: held back
};

// Exclusive sums over the block of two numbers at once (x, y: their sums fit 31 bits);
// every thread gets the totals.
__device__ int2 block_scan(int2 v, int2* warp_sum, int2* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int2 inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kFull, inc.x, o), y = __shfl_up_sync(kFull, inc.y, o);
    if (lane >= o) inc.x += x, inc.y += y;
  }
  if (lane == 31) warp_sum[warp] = inc;
  __syncthreads();
  // (every warp adds up the warps' sums for itself)
  int2 s = warp_sum[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kFull, s.x, o), y = __shfl_up_sync(kFull, s.y, o);
    if (lane >= o) s.x += x, s.y += y;
  }
  total->x = __shfl_sync(kFull, s.x, 31);
  total->y = __shfl_sync(kFull, s.y, 31);
  const int bx = __shfl_sync(kFull, s.x, max(warp - 1, 0)), by = __shfl_sync(kFull, s.y, max(warp - 1, 0));
  __syncthreads();   // warp_sum is free again
  return make_int2((warp ? bx : 0) + inc.x - v.x, (warp ? by : 0) + inc.y - v.y);
}

// Last i in [0, n) with off[i] <= a (rows that need nothing are passed over).
__device__ __forceinline__ int row_of(const int* off, int n, int a) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= a) lo = mid;
    else hi = mid;
  }
  return lo;
}

// (Not the read-only path: a kernel here starts while the ones before it still write the pool, and copies
// within it.)
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}

__device__ __forceinline__ void st_stream(uint4* p, const uint4& v) {
  asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
               : "memory");
}

}  // namespace

struct NoLens {};

template <int OP, typename Lens>
__global__ void __cluster_dims__(kBookCtas, 1, 1) __launch_bounds__(kBookThreads, 1)
    k_book(const __grid_constant__ BookParams p, const __grid_constant__ Lens lens) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  BookSmem& s = *reinterpret_cast<BookSmem*>(smem_raw);
  constexpr bool kTakes = OP == kBookExtend || OP == kBookForkDeep || OP == kBookCompact;
  constexpr bool kForks = OP == kBookFork || OP == kBookForkDeep;
  const PagesView& pg = p.pg;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x;
  const int P = 1 << pg.shift;
  const int64_t room = static_cast<int64_t>(pg.max_pages) << pg.shift;
  for (int i = tid; i < kMaxTableRows / 32; i += kBookThreads) s.seen[i] = 0;
  if (tid == 0) s.bad = 0;
  cluster_arrive();   // waited for before the first write into a peer's shared memory
  __syncthreads();
  griddep_launch_dependents();
  griddep_wait();

  // the counts of this CTA's part of the pages; a warp's first 32 on their way already
  const int words = (pg.n_pages + 31) >> 5;
  const int per = (words + kBookCtas - 1) / kBookCtas;
  const int w0 = min(rank * per, words), nw = min(per, words - w0);
  int count0 = 1;
  if (kTakes && warp < nw && ((w0 + warp) << 5) + lane < pg.n_pages) count0 = pg.refs[((w0 + warp) << 5) + lane];

  // An earlier call was refused and nobody has asked yet: what was queued behind it counts on it, and is not carried
  // out either.  One CTA asks for all (a call of another pool may be refused meanwhile).
  const uint32_t latched = rank == 0 && tid == 0 ? *p.err : 0;

  // ---- the call's rows
  const int i = tid;
  int need = 0, held = 0, L = 0, after = 0, fill = 0;
  bool copies = false;
  if (i < p.n) {
    bool bad = false;
    const int row = p.rows ? p.rows[i] : i;
    int from = row;
    if (row < 0 || row >= pg.n_rows) bad = true;
    else if (atomicOr(&s.seen[row >> 5], 1u << (row & 31)) & (1u << (row & 31))) bad = true;   // named twice
    if (kForks) {
      from = p.src[i];
      bad = bad || from < 0 || from >= pg.n_rows;
    }
    if (!bad) {
      L = pg.len[from];
      bad = L < 0 || L > room;
      if (kForks) bad = bad || pg.len[row] != 0;   // a branch starts in an empty row
      if constexpr (OP == kBookCompact) bad = bad || L != lens.L[i];
    }
    if (!bad) {
      held = (L + P - 1) >> pg.shift;
      fill = L & (P - 1);
      int pos = 0;
      after = kForks ? L : 0;
      if (OP == kBookExtend) {
        const int nn = p.n_new[i];
        if (nn < 0 || static_cast<int64_t>(L) + nn > room) bad = true;
        else {
          after = L + nn;
          if (fill && nn) {
            const int last = pg.table[static_cast<int64_t>(row) * pg.max_pages + held - 1];
            const int holders = last >= 0 && last < pg.n_pages ? pg.refs[last] : 0;
            bad = holders < 1;      // no page, or one that nobody holds
            copies = holders > 1;   // somebody else holds it too
          }
          need = ((after + P - 1) >> pg.shift) - held + copies;
          pos = held - copies;
        }
      }
      if (OP == kBookForkDeep) need = held;
      if constexpr (OP == kBookCompact) {
        after = lens.kept[i];
        need = (after + P - 1) >> pg.shift;
        bad = need > pg.max_pages;
      }
      s.pos[i] = pos;
    }
    s.row[i] = row;
    s.from[i] = from;
    s.len[i] = L;
    if (bad) {
      s.bad = 1;
      need = held = 0;
    }
  }
  if (tid == 0) s.hold = latched & kErrHeld;
  int2 totals;
  const int2 off = block_scan(make_int2(need, held), s.warp_sum, &totals);
  const int total = totals.x, held_total = totals.y;
  if (i < p.n) {
    s.off[i] = off.x;
    s.held[i] = off.y;
  }
  __syncthreads();
  const bool bad = s.bad != 0;

  // ---- the pages that the rows hold, an eighth of them per CTA: each has to be one that is held.
  // (Looked at before anything changes; a thread's first page is kept for afterwards.)
  constexpr bool kWalks = OP != kBookExtend;
  const int a0 = rank * kBookThreads + tid;
  int row0 = 0, page0 = 0;
  bool odd = false;
  if (kWalks && !bad)
    for (int a = a0; a < held_total; a += kBookCtas * kBookThreads) {
      const int r = row_of(s.held, p.n, a), j = a - s.held[r];
      const int page = pg.table[static_cast<int64_t>(s.from[r]) * pg.max_pages + j];
      odd = odd || page < 0 || page >= pg.n_pages || pg.refs[page] < 1;
      if (a == a0) row0 = r, page0 = page;
      if (OP == kBookCompact) p.old_table[static_cast<int64_t>(r) * pg.max_pages + j] = page;   // what the gather reads
    }
  if (kWalks) odd = __syncthreads_or(odd);

  // ---- the free pages of this CTA's part, one bit each
  int mine = 0;   // free pages of the part
  if (kTakes) {
    for (int w = warp; w < nw; w += kBookThreads / 32) {
      const int page = ((w0 + w) << 5) + lane;
      const uint32_t m = __ballot_sync(kFull, w == warp ? count0 == 0 : page < pg.n_pages && pg.refs[page] == 0);
      if (lane == 0) s.bits[w] = m;
    }
    __syncthreads();
    int base = 0;
    for (int c = 0; c < nw; c += kBookThreads) {
      const int w = c + tid;
      int2 sum;
      const int2 b = block_scan(make_int2(w < nw ? __popc(s.bits[w]) : 0, 0), s.warp_sum, &sum);
      if (w < nw) s.before[w] = base + b.x;
      base += sum.x;
    }
    mine = base;
  }
  cluster_wait();   // every CTA of the cluster runs: its shared memory may be written
  if (tid < kBookCtas) dsmem_st_u32(dsmem_map(&s.count[rank], tid), static_cast<uint32_t>(s.hold ? -2 : odd ? -1 : mine));
  cluster_sync();   // from here on lengths, tables and counts change

  int before = 0, avail = 0;
  bool wrong = bad;
  for (int c = 0; c < kBookCtas; ++c) {
    wrong = wrong || s.count[c] < 0;
    if (c < rank) before += s.count[c];
    avail += s.count[c];
  }
  const bool ok = !wrong && (!kTakes || total <= avail);
  if (rank == 0 && tid == 0) {
    if (!ok && s.count[0] != -2) atomicOr(p.err, (wrong ? kErrRow : kErrPool) | kErrHeld);
    if (p.plan) {
      p.plan->ok = ok;
      p.plan->n_copies = !ok ? 0 : OP == kBookExtend ? p.n : OP == kBookForkDeep ? total : 0;
    }
  }
  if (!ok) return;

  // ---- free page number a goes to need number a
  if (kTakes)
    for (int w = warp; w < nw; w += kBookThreads / 32) {
      if (before + s.before[w] >= total) break;   // the words after it come later still
      const uint32_t m = s.bits[w];
      const int a = before + s.before[w] + __popc(m & ((1u << lane) - 1));
      if (!(m >> lane & 1) || a >= total) continue;
      const int page = ((w0 + w) << 5) + lane;
      const int r = row_of(s.off, p.n, a), j = a - s.off[r];
      int32_t* entry = pg.table + static_cast<int64_t>(s.row[r]) * pg.max_pages + s.pos[r] + j;
      if (OP == kBookExtend && j == 0) {
        const int f = s.len[r] & (P - 1);
        if (s.pos[r] < (s.len[r] + P - 1) >> pg.shift) {   // in the place of a shared last page
          p.copies[r] = make_int4(*entry, page, f, 0);
          atomicSub(&pg.refs[*entry], 1);
        }
      }
      if (OP == kBookForkDeep) {
        const int from = pg.table[static_cast<int64_t>(s.from[r]) * pg.max_pages + j];
        p.copies[a] = make_int4(from, page, min(P, s.len[r] - (j << pg.shift)), 0);
      }
      *entry = page;
      pg.refs[page] = 1;
    }

  // ---- pages that change hands without moving
  if (OP == kBookFork || OP == kBookFree || OP == kBookCompact)
    for (int a = a0; a < held_total; a += kBookCtas * kBookThreads) {
      const int r = a == a0 ? row0 : row_of(s.held, p.n, a), j = a - s.held[r];
      const int page = a == a0                ? page0
                       : OP == kBookCompact ? p.old_table[static_cast<int64_t>(r) * pg.max_pages + j]
                                            : pg.table[static_cast<int64_t>(s.from[r]) * pg.max_pages + j];
      if (OP == kBookFork) {
        atomicAdd(&pg.refs[page], 1);
        pg.table[static_cast<int64_t>(s.row[r]) * pg.max_pages + j] = page;
      } else if (atomicSub(&pg.refs[page], 1) <= 0) {   // fewer holders counted than the call's rows that name it
        atomicAdd(&pg.refs[page], 1);
        atomicOr(p.err, kErrRow);
      }
    }
  if (rank == 0 && i < p.n) {
    pg.len[s.row[i]] = after;
    if (OP == kBookExtend && !copies) p.copies[i] = make_int4(-1, 0, 0, 0);
  }
}

namespace {

using BookKernel = void (*)(BookParams, NoLens);

BookKernel book_kernel(BookOp op) {
  switch (op) {
    case kBookExtend: return k_book<kBookExtend, NoLens>;
    case kBookFork: return k_book<kBookFork, NoLens>;
    case kBookForkDeep: return k_book<kBookForkDeep, NoLens>;
    default: return k_book<kBookFree, NoLens>;
  }
}

}  // namespace

cudaError_t pages_configure() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  for (BookOp op : {kBookExtend, kBookFork, kBookForkDeep, kBookFree}) {
    const cudaError_t e = cudaFuncSetAttribute(book_kernel(op), attr, sizeof(BookSmem));
    if (e != cudaSuccess) return e;
  }
  return cudaFuncSetAttribute(k_book<kBookCompact, BookLens>, attr, sizeof(BookSmem));
}

cudaError_t book_launch(BookOp op, const BookParams& p, const BookLens* lens, cudaStream_t stream) {
  if (p.n <= 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kBookCtas);
  cfg.blockDim = dim3(kBookThreads);
  cfg.dynamicSmemBytes = sizeof(BookSmem);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (op == kBookCompact) return cudaLaunchKernelEx(&cfg, k_book<kBookCompact, BookLens>, p, *lens);
  return cudaLaunchKernelEx(&cfg, book_kernel(op), p, NoLens{});
}

// ---------------------------------------------------------------- copies

namespace {

constexpr int kMoveThreads = 256;
constexpr int kMoveWarps = kMoveThreads / 32;
constexpr int kTaskRows = 32;   // rows of a warp task
constexpr int kInFlight = 8;    // 16-byte accesses per lane in flight (16 rows per warp)
constexpr int kMoveBlocksPerSm = 4;
constexpr int kRow4 = kHeadDim / 8;   // 16-byte units of a row

// 32 rows, row i from in + src(i) to out + dst(i) (16-byte units), where lane i
// holds its own row's `from` and `to` words and a word below 0 skips the row.
template <typename Src, typename Dst>
__device__ __forceinline__ void move_rows(const uint4* in, uint4* out, int from, int to, Src src, Dst dst) {
  const int lane = threadIdx.x & 31, half = lane >> 4, hl = lane & 15;
#pragma unroll
  for (int j0 = 0; j0 < kTaskRows; j0 += 2 * kInFlight) {
    uint4 v[kInFlight];
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const int f = __shfl_sync(kFull, from, j0 + 2 * k + half);
      if (f >= 0) v[k] = ld_stream(in + src(f) + hl);
    }
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const int row = j0 + 2 * k + half;
      const int f = __shfl_sync(kFull, from, row), t = __shfl_sync(kFull, to, row);
      if (f >= 0) st_stream(out + dst(t) + hl, v[k]);
    }
  }
}

cudaLaunchConfig_t move_config(cudaLaunchAttribute* attr, dim3 grid, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kMoveThreads);
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // starts under the previous kernel's tail
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

// Place of a token word (page << shift | slot) in one KV head of a layer, in 16-byte units.
struct PagePlace {
  int64_t page4;   // page stride
  int head4;       // of the KV head
  int shift;
  __device__ __forceinline__ int64_t operator()(int word) const {
    return static_cast<int64_t>(word >> shift) * page4 + head4 + (word & ((1 << shift) - 1)) * kRow4;
  }
};

}  // namespace

// Warp tasks: (copy, layer, tensor, KV head, 32 rows of the page).
__global__ void __launch_bounds__(kMoveThreads, kMoveBlocksPerSm)
    k_page_copy(const __grid_constant__ PagesView pg, const PagePlan* plan, const int4* copies) {
  griddep_launch_dependents();
  griddep_wait();
  const int lane = threadIdx.x & 31;
  const int blocks = max(1, (1 << pg.shift) / kTaskRows);
  const int per = blocks * pg.G * 2 * pg.n_layers;   // tasks of a copy
  const int64_t ntask = static_cast<int64_t>(plan->n_copies) * per;
  for (int64_t task = static_cast<int64_t>(blockIdx.x) * kMoveWarps + (threadIdx.x >> 5); task < ntask;
       task += static_cast<int64_t>(gridDim.x) * kMoveWarps) {
    const int c = static_cast<int>(task / per);
    int rem = static_cast<int>(task - static_cast<int64_t>(c) * per);
    const int b = rem % blocks;
    rem /= blocks;
    const int g = rem % pg.G;
    rem /= pg.G;
    const int layer = rem >> 1;
    const int4 e = copies[c];
    const int slot = b * kTaskRows + lane;
    const bool live = e.x >= 0 && slot < e.z;
    if (!__any_sync(kFull, live)) continue;
    __nv_bfloat16* pool = (rem & 1 ? pg.v : pg.k) + layer * pg.layer_stride;
    const PagePlace place{pg.page_stride / 8, (g << pg.shift) * kRow4, pg.shift};
    move_rows(reinterpret_cast<const uint4*>(pool), reinterpret_cast<uint4*>(pool), live ? e.x << pg.shift | slot : -1,
              live ? e.y << pg.shift | slot : -1, place, place);
  }
}

cudaError_t page_copy_launch(const PagesView& pg, const PagePlan* plan, const int4* copies, int64_t max_copies, int num_sms,
                             cudaStream_t stream) {
  const int64_t tasks = max_copies * max(1, (1 << pg.shift) / kTaskRows) * pg.G * 2 * pg.n_layers;
  if (tasks <= 0) return cudaSuccess;
  const int64_t blocks = (tasks + kMoveWarps - 1) / kMoveWarps;
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = move_config(attr, dim3(static_cast<unsigned>(min(blocks, static_cast<int64_t>(num_sms) * kMoveBlocksPerSm))), stream);
  return cudaLaunchKernelEx(&cfg, k_page_copy, pg, plan, copies);
}

// grid: (blocks, layers, sequences).  Tasks of one (sequence, layer): 2 tensors x
// G x ceil((B + w) / 32) row blocks, one per warp.
__global__ void __launch_bounds__(kMoveThreads, kMoveBlocksPerSm)
    k_page_gather(const __grid_constant__ PagesView pg, const __grid_constant__ SeqBatch b, const int32_t* rows, int row0, int w,
                  int per_head, const PagePlan* plan, const int32_t* old_table, uint32_t* err) {
  griddep_launch_dependents();
  griddep_wait();
  if (!plan->ok) return;
  const SeqView& sv = b.s[blockIdx.z];
  const int seq = blockIdx.z, layer = blockIdx.y;
  const int B = sv.budget, Lp = sv.Lp;
  const int rows_out = B + w;
  const int lane = threadIdx.x & 31;
  const int sets = per_head ? pg.G : 1;
  const int row = rows ? rows[row0 + seq] : row0 + seq;
  const int32_t* idx_l = sv.idx + static_cast<int64_t>(layer) * sets * B;
  const uint32_t* meta_l = sv.meta ? sv.meta + static_cast<int64_t>(layer) * sv.meta_layer_stride : nullptr;
  uint32_t* meta_out_l = sv.meta_out + static_cast<int64_t>(layer) * sets * rows_out;
  const int32_t* was = old_table + static_cast<int64_t>(row0 + seq) * pg.max_pages;
  const int32_t* is = pg.table + static_cast<int64_t>(row) * pg.max_pages;
  const int nblk = ceil_div(rows_out, kTaskRows);
  const int ntask = 2 * pg.G * nblk;
  for (int task = blockIdx.x * kMoveWarps + (threadIdx.x >> 5); task < ntask; task += gridDim.x * kMoveWarps) {
    const int tensor = task / (pg.G * nblk);
    const int rem = task - tensor * pg.G * nblk;
    const int g = rem / nblk, r = (rem - g * nblk) * kTaskRows + lane;
    const int set = per_head ? g : 0;
    int from = -1, to = -1;
    if (r < rows_out) {
      int src = r < B ? idx_l[static_cast<int64_t>(set) * B + r] : Lp + (r - B);
      if (src < 0 || src >= (r < B ? Lp : sv.L)) {   // a kept index must name a past token: report, copy row 0
        atomicOr(err, kErrIndex);
        src = 0;
      }
      if (meta_l && tensor == 0 && g == set)
        meta_out_l[static_cast<int64_t>(set) * rows_out + r] = meta_l[set * sv.meta_group_stride + src];
      const int page = was[src >> pg.shift];
      to = is[r >> pg.shift] << pg.shift | (r & ((1 << pg.shift) - 1));
      if (page >= 0 && page < pg.n_pages) from = page << pg.shift | (src & ((1 << pg.shift) - 1));   // (else reported)
    }
    __nv_bfloat16* pool = (tensor == 0 ? pg.k : pg.v) + layer * pg.layer_stride;
    const PagePlace place{pg.page_stride / 8, (g << pg.shift) * kRow4, pg.shift};
    move_rows(reinterpret_cast<const uint4*>(pool), reinterpret_cast<uint4*>(pool), from, to, place, place);
  }
}

cudaError_t page_gather_launch(const PagesView& pg, const SeqBatch& b, const int32_t* rows, int row0, int w, int per_head,
                               const PagePlan* plan, const int32_t* old_table, int rows_out_max, uint32_t* err,
                               cudaStream_t stream) {
  if (rows_out_max <= 0) return cudaSuccess;
  const int ntask = 2 * pg.G * ceil_div(rows_out_max, kTaskRows);
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = move_config(attr, dim3(static_cast<unsigned>(ceil_div(ntask, kMoveWarps)), b.nlayers, b.nseq), stream);
  return cudaLaunchKernelEx(&cfg, k_page_gather, pg, b, rows, row0, w, per_head, plan, old_table, err);
}

// Warp tasks: (sequence, layer, tensor, 32 of the T * G rows, the KV heads of a
// token together).  The tokens are the last n_tokens of their row.
template <bool STORE>
__global__ void __launch_bounds__(kMoveThreads, kMoveBlocksPerSm)
    k_page_move(const __grid_constant__ PagesView pg, const __grid_constant__ TokensView t, uint32_t* err) {
  griddep_launch_dependents();
  griddep_wait();
  const uint32_t latched = STORE ? *err : 0;   // (looked at when the places are known: its way is as long as theirs)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int nblk = static_cast<int>((static_cast<int64_t>(t.T) * pg.G + kTaskRows - 1) / kTaskRows);
  const int tensors = t.v ? 2 : 1;
  const int64_t per_seq = static_cast<int64_t>(nblk) * tensors * t.nlayers;
  const int64_t ntask = per_seq * t.n;
  const bool rivals = STORE && t.rows && t.n > 1;
  __shared__ uint32_t found[kMoveWarps];
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kMoveWarps; base < ntask;
       base += static_cast<int64_t>(gridDim.x) * kMoveWarps) {
    // A row that two sequences of a store name would hold either's tokens: the block looks for its own sequences'
    // rows among all.  (Loaded here, looked at when the places are known; 64 rows stored in 28 layers 5.0 us, 4.5
    // without the look, 1,024 rows 48 and 43.)
    const int first = static_cast<int>(base / per_seq);
    int named[kMaxCallRows / kMoveThreads];
#pragma unroll
    for (int k = 0; k < kMaxCallRows / kMoveThreads; ++k) {
      const int j = k * kMoveThreads + threadIdx.x;
      named[k] = rivals && j < t.n ? t.rows[j] : -1;
    }
    int seq = first;
    int64_t rem = base - first * per_seq + (base + warp < ntask ? warp : 0);
    for (; rem >= per_seq; rem -= per_seq) ++seq;
    const int blk = static_cast<int>(rem % nblk);
    rem /= nblk;
    const int tensor = tensors == 2 ? static_cast<int>(rem & 1) : 0;
    const int l = static_cast<int>(tensors == 2 ? rem >> 1 : rem);
    const int row = t.rows ? t.rows[seq] : seq;
    int count = t.n_tokens ? t.n_tokens[seq] : t.T;
    const bool row_ok = row >= 0 && row < pg.n_rows;
    const int L = row_ok ? pg.len[row] : 0;
    bool wrong = !row_ok || count < 0 || count > t.T || count > L || L > static_cast<int64_t>(pg.max_pages) << pg.shift;
    if (wrong || base + warp >= ntask) count = 0;
    const int64_t r = static_cast<int64_t>(blk) * kTaskRows + lane;
    const int tok = static_cast<int>(r / pg.G), g = static_cast<int>(r - static_cast<int64_t>(tok) * pg.G);
    int word = -1;   // the token's place in the pages
    if (tok < count) {
      const int at = L - count + tok;
      const int page = pg.table[static_cast<int64_t>(row) * pg.max_pages + (at >> pg.shift)];
      // a page that others hold too is not written to
      if (page < 0 || page >= pg.n_pages || (STORE && pg.refs[page] != 1)) atomicOr(err, kErrRow);
      else word = page << pg.shift | (at & ((1 << pg.shift) - 1));
    }
    if (rivals) {
      uint32_t twice = 0;   // bit: sequence - first
      int64_t left = min(base + kMoveWarps, ntask) - first * per_seq;   // the block's tasks from its first sequence on
      for (int s = first; left > 0; ++s, left -= per_seq) {
        const int row = t.rows[s];
#pragma unroll
        for (int k = 0; k < kMaxCallRows / kMoveThreads; ++k) {
          const int j = k * kMoveThreads + threadIdx.x;   // (one that brings no tokens is no rival)
          if (named[k] == row && j != s && j < t.n && !(t.n_tokens && t.n_tokens[j] == 0)) twice |= 1u << (s - first);
        }
      }
      if (__syncthreads_or(twice)) {
        twice = __reduce_or_sync(kFull, twice);
        if (lane == 0) found[warp] = twice;
        __syncthreads();
        twice = __reduce_or_sync(kFull, found[lane & (kMoveWarps - 1)]);
        __syncthreads();   // (read, before the block's next tasks write it)
        if (count && twice >> (seq - first) & 1) wrong = true, word = -1;
      }
    }
    if (wrong && lane == 0) atomicOr(err, kErrRow);
    if (STORE && __any_sync(kFull, latched & kErrHeld)) word = -1;   // a call was refused: nothing is written
    __nv_bfloat16* pool = (tensor ? pg.v : pg.k) + (t.layer0 + l) * pg.layer_stride;
    __nv_bfloat16* flat = (tensor ? t.v : t.k) + seq * t.seq_stride + l * t.layer_stride;
    const int half = lane >> 4, hl = lane & 15;
#pragma unroll
    for (int j0 = 0; j0 < kTaskRows; j0 += 2 * kInFlight) {
      uint4 v[kInFlight];
      uint4* dst[kInFlight];
#pragma unroll
      for (int k = 0; k < kInFlight; ++k) {
        const int i = j0 + 2 * k + half;
        const int wd = __shfl_sync(kFull, word, i);
        const int tk = __shfl_sync(kFull, tok, i), gg = __shfl_sync(kFull, g, i);
        dst[k] = nullptr;
        if (wd >= 0) {
          const PagePlace place{pg.page_stride / 8, (gg << pg.shift) * kRow4, pg.shift};
          uint4* in_pool = reinterpret_cast<uint4*>(pool) + place(wd) + hl;
          uint4* in_flat = reinterpret_cast<uint4*>(flat + tk * t.token_stride + gg * t.head_stride) + hl;
          v[k] = ld_stream(STORE ? in_flat : in_pool);
          dst[k] = STORE ? in_pool : in_flat;
        }
      }
#pragma unroll
      for (int k = 0; k < kInFlight; ++k)
        if (dst[k]) st_stream(dst[k], v[k]);
    }
  }
}

cudaError_t page_move_launch(bool store, const PagesView& pg, const TokensView& t, uint32_t* err, cudaStream_t stream) {
  const int64_t tasks = ((static_cast<int64_t>(t.T) * pg.G + kTaskRows - 1) / kTaskRows) * (t.v ? 2 : 1) * t.nlayers * t.n;
  if (tasks <= 0) return cudaSuccess;
  const int64_t blocks = (tasks + kMoveWarps - 1) / kMoveWarps;
  cudaLaunchAttribute attr[1];
  // a task per warp: 28 layers x 2,736 tokens stored and loaded 100 us, with a grid that
  // fills the GPU once 109 (where many tasks turn out empty, as in the page copies, such a
  // grid is the better one: 59 us for 64 branches, 60 so)
  cudaLaunchConfig_t cfg = move_config(attr, dim3(static_cast<unsigned>(min(blocks, int64_t(1) << 30))), stream);
  return cudaLaunchKernelEx(&cfg, store ? k_page_move<true> : k_page_move<false>, pg, t, err);
}

}  // namespace starkv
