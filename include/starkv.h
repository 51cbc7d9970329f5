/*
 * starkv.h -- C ABI of the STaR-KV compression stage on one GB300 (sm_103a).
 *
 * STaR-KV (Spatio-Temporal Adaptive Re-weighting) compresses the KV cache of a
 * GUI vision-language model per layer (Algorithm 1, App. A.2):
 *   1. score the last w window queries against every past key over the GQA
 *      groups, pool along tokens and average inside each group  (Sec. 3.3);
 *   2. re-weight by a per-group prior from the online spatial mutual
 *      information of each group's scores with the screen-patch grid (Sec. 3.4);
 *   3. discount stale visual tokens by the temporal stability of their
 *      governing group (Sec. 3.5);
 *   4. reshape by an entropy-derived temperature (Sec. 3.6);
 *   5. keep the global top-B historical tokens plus the recent window and
 *      gather them into a new contiguous cache (Sec. 3.7).
 * An optional per-KV-head selection mode (select_mode = STARKV_SELECT_PER_HEAD,
 * the head-wise top-K of App. A.3 with the STaR-KV factors) lets each group g
 * keep its own B tokens: it ranks s_{g,t} = max(S[g,t] beta_g D_{g,t}, 0)^(1/T_g)
 * with beta_g = (1 - lambda) + lambda G w_g, D_{g,t} of Eq. (9) with phi_g and
 * T_g from the entropy of S[g, .] (Sec. 3.6 on that row).  beta_g is one factor
 * per row, so in this mode the MI prior scales the scores without changing
 * any group's set.
 *
 * Conventions shared by every call
 * --------------------------------
 * - Pointers inside starkv_seq are DEVICE pointers (cudaMalloc / torch CUDA
 *   memory), except for starkv_step_host, where they are HOST pointers.
 *   The caller owns every input and output buffer; the library owns only the
 *   state created by starkv_init_state.
 * - `stream` is a cudaStream_t passed as void* (NULL = legacy default stream).
 *   Calls are asynchronous and stream-ordered; none synchronises the stream.
 * - `workspace` is caller-owned device scratch of at least
 *   starkv_workspace_bytes(...) bytes, 256-byte aligned.  Its contents are
 *   undefined on entry and on exit.  Concurrent calls must not share it.
 * - Layouts (all row-major, contiguous):
 *     k, v        bf16  [n_layers][G][L][d]
 *     q           bf16  [n_layers][H][w][d]   post-RoPE queries of the last w tokens
 *     meta        u32   [n_layers][L]  or [L] shared (meta_layer_stride = 0);
 *                       per-KV-head mode: optionally one row per group,
 *                       [n_layers][G][L] (meta_group_stride = L, see below)
 *     S           f32   [n_layers][G][L_p]     group score map, L_p = L - w
 *     score       f32   [n_layers][P][L_p]     fused score s_t (s_{g,t})
 *     idx         i32   [n_layers][P][B]       kept historical positions, ascending
 *     k_out,v_out bf16  [n_layers][G][B + w][d]
 *     meta_out    u32   [n_layers][P][B + w]
 *   where P = 1 in the global selection mode and P = G in the per-KV-head mode
 *   (row g of idx / meta_out belongs to group g of k_out / v_out).
 *     stats       f32   [n_layers][STARKV_STATS_STRIDE(G)]
 *   Token metadata word: bit 31 = visual, bits 20..30 = frame id f(t),
 *   bits 10..19 = patch row r_t, bits 0..9 = patch column c_t (Sec. 3.1).
 *   Text tokens only need bit 31 clear.
 * - Errors: a call that returns non-OK has launched nothing unless the code is
 *   STARKV_ERR_CUDA (a launch or copy failed part-way).  Invalid arguments are
 *   caught on the host before any launch.  Device-side checks (metadata out of
 *   range, a bounded wait that ran out) latch a code in the state's device
 *   error word, which starkv_check_device_error reads.  starkv_last_error
 *   returns a thread-local message for the last non-OK status.
 * - Supported shapes: d = 128; w >= 1; H % G == 0; (H / G) * w <= 256;
 *   G <= 32 in the global selection mode (G = H is the MHA-head granularity of
 *   the ablation in Sec. 4.2: each group's key/value replicated for each of its
 *   query heads), G <= 8 in the per-KV-head mode; L >= w (L_p = L - w >= 0;
 *   L_p = 0 keeps only the window);
 *   0 <= B <= L_p; L < 2^24; 1 <= R, C <= 1024; R * C <= 16384;
 *   2 <= mi_bins <= 16; mi_bins * mi_grid^2 <= 4096; odd pool_kernel <= 31;
 *   frame ids 0..2047.  Other shapes return STARKV_ERR_UNSUPPORTED.
 *   k, v, q, k_out and v_out must be 16-byte aligned, every other array
 *   4-byte aligned (STARKV_ERR_INVALID_ARG otherwise).
 */
#ifndef STARKV_H
#define STARKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  STARKV_OK = 0,
  STARKV_ERR_INVALID_ARG = 1,  /* a pointer, size or index is invalid          */
  STARKV_ERR_UNSUPPORTED = 2,  /* valid but outside the supported shapes       */
  STARKV_ERR_CUDA = 3,         /* a CUDA runtime call failed                   */
  STARKV_ERR_TIMEOUT = 4,      /* a bounded device-side wait ran out           */
  STARKV_ERR_NOMEM = 5,        /* state allocation failed                      */
  STARKV_ERR_DEVICE = 6        /* a device-side input check failed             */
} starkv_status;

/* Hyper-parameters.  starkv_default_config fills the paper's defaults
 * (App. A.1, Table 7 AgentNetBench / UI-TARS) and this library's readings of
 * the values the paper leaves open (pool_kernel, mi_bins, mi_grid, eps, eps_h). */
typedef struct {
  int32_t n_layers;
  int32_t n_heads;      /* H query heads                                           */
  int32_t n_kv_heads;   /* G KV groups ("subspaces", Sec. 3.1)                     */
  int32_t head_dim;     /* d, must be 128                                          */
  int32_t window;       /* w: observation window = recent window W_rec (Sec. 3.1)  */
  int32_t grid_rows;    /* R: patch rows of one screenshot                         */
  int32_t grid_cols;    /* C: patch columns of one screenshot                      */
  int32_t pool_kernel;  /* AvgPool1D kernel (odd), stride 1, zero padding (Sec 3.3)*/
  int32_t mi_bins;      /* K equal-frequency rank bins (Sec. 3.4)                  */
  int32_t mi_grid;      /* M: SpatialBin grid is M x M (Sec. 3.4)                  */
  int32_t n_warmup;     /* lambda is 0 for the first n_warmup steps (App. A.1)     */
  int32_t n_ramp;       /* then ramps linearly to lambda over n_ramp steps         */
  int32_t max_seqs;     /* number of state slots (independent trajectories)        */
  float lambda;         /* MI prior strength (Eq. final_score)                     */
  float tau;            /* prior softmax temperature (Eq. 7)                       */
  float rho_mi;         /* MI EMA decay (Eq. 6)                                    */
  float rho_t;          /* temporal EMA decay (Eq. 8)                              */
  float delta;          /* temporal decay rate (Eq. 9)                             */
  float d_min;          /* minimum temporal factor D_min (Eq. 9)                   */
  float t_min, t_max;   /* AEB temperature range (Sec. 3.6)                        */
  float eps;            /* epsilon of the min-max prior (Eq. 7)                    */
  float eps_h;          /* epsilon of the AEB entropy (Algorithm 1)                */
  int32_t select_mode;  /* STARKV_SELECT_GLOBAL (the paper's, default) or
                           STARKV_SELECT_PER_HEAD (one top-B set per KV group)     */
  /* Variants of the paper's ablations (Table 3, the AEB ablation), 0 = the
   * method as defined.  The paper names them without a formula; this
   * library's readings, with x = Delta_f phi:
   *   decay_mode 1 (linear):    D = D_min + (1 - D_min) max(0, 1 - delta x)
   *   decay_mode 2 (power law): D = D_min + (1 - D_min) (1 + x)^(-delta)
   *   aeb_mode 1 (confidence):  T = T_min + (T_max - T_min)(1 - p_max), with
   *                             p_max = max_t s_bar_t / (sum_t s_bar_t + eps_h)
   *   mi_span 1:                the MI of Sec. 3.4 over the newest frame's
   *                             visual tokens only                              */
  int32_t decay_mode;
  int32_t aeb_mode;
  int32_t mi_span;
} starkv_config;

/* Values of starkv_config.select_mode. */
enum { STARKV_SELECT_GLOBAL = 0, STARKV_SELECT_PER_HEAD = 1 };

/* One sequence (trajectory) of a batch: inputs and caller-owned outputs.  For
 * per-layer calls (score_layer / select / compact) the `layer` argument picks
 * the [layer] slice of every [n_layers][...] buffer below. */
typedef struct {
  const void* k;                /* bf16 [n_layers][G][L][d]                         */
  const void* v;                /* bf16 [n_layers][G][L][d]                         */
  const void* q;                /* bf16 [n_layers][H][w][d]                         */
  const uint32_t* meta;         /* u32  [n_layers][L] (or [L] if stride is 0)       */
  int64_t meta_layer_stride;    /* elements between layers of meta: 0 or >= L       */
  int32_t L;                    /* cache length, including the w recent tokens      */
  int32_t cur_frame;            /* F: frame id of the current (newest) screenshot   */
  int32_t budget;               /* B: kept historical tokens, 0 <= B <= L - w       */
  int32_t slot;                 /* state slot in [0, max_seqs)                      */
  void* k_out;                  /* bf16 [n_layers][G][B + w][d]       (compact)    */
  void* v_out;                  /* bf16 [n_layers][G][B + w][d]       (compact)    */
  uint32_t* meta_out;           /* u32  [n_layers][P][B + w]          (compact)    */
  int32_t* idx;                 /* i32  [n_layers][P][B]   select writes, compact reads */
  float* S;                     /* f32  [n_layers][G][L_p] score_layer writes, select
                                   reads; may be NULL for starkv_step (workspace)   */
  float* score;                 /* f32  [n_layers][P][L_p] fused s_t, optional (NULL) */
  float* stats;                 /* f32  [n_layers][STARKV_STATS_STRIDE(G)], optional */
  int64_t meta_group_stride;    /* elements between the metadata rows of groups g
                                   and g + 1 of one layer: 0 = every group shares
                                   one row (required in the global mode), else >= L
                                   (per-KV-head mode, where each group's cache holds
                                   its own tokens after a compaction); with a
                                   nonzero meta_layer_stride it must be
                                   >= (G - 1) * meta_group_stride + L                */
  const float* lse;             /* f32 [n_layers][H][w], optional: the softmax
                                   normaliser of each window row (Eq. 2), as the
                                   natural-log log-sum-exp over the past keys t < L_p
                                   of z = Q_{-i,h} . K[g(h), t] / sqrt(d) (the window
                                   keys excluded), e.g. from the layer's own prefill
                                   attention pass, which computes these logits.  When
                                   every sequence of a call gives it, the first
                                   scoring pass (a whole read of K) is skipped.
                                   NULL = computed.                                 */
  float* attn_o;                /* f32 [n_layers][H][w][d], optional: written by
                                   starkv_window_attention (the window rows'
                                   attention output over the past keys); 16-byte
                                   aligned                                          */
  float* attn_lse;              /* f32 [n_layers][H][w]: written by
                                   starkv_window_attention, each window row's
                                   natural-log normaliser over the past keys, the
                                   value `lse` takes                                */
} starkv_seq;

/* Per-layer diagnostics written to starkv_seq.stats (floats):
 *   [0] H_hat (p_max with aeb_mode 1)  [1] T  [2] lambda_n  [3] n (steps seen before this one)
 *   [4] sum_t s_bar_t  [5] visual tokens in L_p  [6] kept count  [7] 0
 *   [8 + g]       MI_g of this step            (Eq. 5)
 *   [8 + G + g]   MI_bar_g after the EMA       (Eq. 6)
 *   [8 + 2G + g]  w_g                          (Eq. 7)
 *   [8 + 3G + g]  phi_g                        (Eq. 8)
 *   [8 + 4G + g]  H_hat of the row group g ranks: s_bar (global mode, the same
 *                 for every g) or S[g, .] (per-KV-head mode)
 *   [8 + 5G + g]  its temperature T
 * In the per-KV-head mode [0] and [1] are the means of [8 + 4G ..] and
 * [8 + 5G ..] over g.                                                         */
#define STARKV_STATS_STRIDE(G) (8 + 6 * (G))

typedef struct starkv_state starkv_state;

/* Fills `cfg` with the defaults for the UI-TARS-1.5-7B GQA shape (H = 28,
 * G = 4, d = 128, w = 32, 52 x 52 patches, 28 layers, 1 slot). */
void starkv_default_config(starkv_config* cfg);

/* Allocates the device-resident per-(slot, layer) state: step counter n, MI EMA
 * MI_bar[G] (Eq. 6), temporal EMA m_g[R*C] per group (Eq. 8), all zero (fresh).
 * The state lives on the current CUDA device; use it only there.
 * Errors: INVALID_ARG / UNSUPPORTED for a bad config, NOMEM, CUDA. */
starkv_status starkv_init_state(const starkv_config* cfg, starkv_state** out, void* stream);

/* Trajectory-level reset of one slot (App. A.4: states are reset per
 * trajectory): zeroes n, MI_bar and m_g of every layer, stream-ordered. */
starkv_status starkv_reset_seq(starkv_state* st, int32_t slot, void* stream);

/* Frees the state (synchronises the device first).  NULL is accepted. */
starkv_status starkv_destroy_state(starkv_state* st);

/* Checkpoint / resume of one slot's carried state (the step counters n, the
 * MI EMAs MI_bar of Eq. 6 and the temporal EMAs m_g of Eq. 8 of every layer),
 * e.g. to continue a trajectory in another process or on another device.
 * Host buffer layout, STARKV_SLOT_STATE_BYTES(n_layers, G, R*C) bytes:
 *   starkv_slot_header (32 B), then
 *   int32  n[n_layers]                 padded to a multiple of 8 bytes
 *   f64    mi_bar[n_layers][G]
 *   f32    m[n_layers][G][R*C]
 * The header records the shape; an import whose header does not match the
 * state's (magic, version, n_layers, G, R, C) or whose buffer is too small is
 * rejected with STARKV_ERR_INVALID_ARG before any copy. */
typedef struct {
  uint32_t magic;       /* STARKV_SLOT_MAGIC */
  uint32_t version;     /* 1 */
  int32_t n_layers, n_kv_heads, grid_rows, grid_cols;
  uint32_t reserved[2]; /* zero */
} starkv_slot_header;

#define STARKV_SLOT_MAGIC 0x31564B53u   /* "SKV1" */
#define STARKV_SLOT_STATE_BYTES(n_layers, G, RC)                              \
  (sizeof(starkv_slot_header) + (((size_t)(n_layers) * 4 + 7) & ~(size_t)7) + \
   (size_t)(n_layers) * (G) * 8 + (size_t)(n_layers) * (G) * (RC) * 4)

/* Bytes of one slot's exported state for this state's shape. */
starkv_status starkv_slot_state_bytes(const starkv_state* st, size_t* bytes);

/* Writes slot `slot`'s state into the HOST buffer `host` (>= the size above):
 * the header at once, the arrays by stream-ordered copies (valid after the
 * stream is synchronised; page-locked memory keeps them asynchronous). */
starkv_status starkv_export_slot(starkv_state* st, int32_t slot, void* host, size_t bytes, void* stream);

/* Replaces slot `slot`'s state with the one in the HOST buffer `host`, written
 * by starkv_export_slot for the same shape (stream-ordered copies; the buffer
 * may be reused once the stream has passed them). */
starkv_status starkv_import_slot(starkv_state* st, int32_t slot, const void* host, size_t bytes, void* stream);

/* Copies the config the state was created with. */
starkv_status starkv_get_config(const starkv_state* st, starkv_config* out);

/* Bytes of device workspace that starkv_score_layer, starkv_select,
 * starkv_compact, starkv_step and starkv_window_attention need for this batch
 * (the maximum of the five).
 * With host != 0: the bytes starkv_step_host needs (adds staging copies). */
starkv_status starkv_workspace_bytes(const starkv_state* st, const starkv_seq* seqs, int32_t nseq,
                                     int32_t host, size_t* bytes);

/* Sec. 3.3, Eqs. (2)-(4): for layer `layer` of
 * every sequence, writes S[g][t] = (G/H) * sum_{h in g} AvgPool1D(
 * sum_{i<w} softmax_t(Q_{-i,h} K_past[g]^T / sqrt(d)))[t]  for t < L_p,
 * softmax over K_past only.  Reads k, q; writes S.  Uses tcgen05 tensor cores
 * (bf16 in, fp32 accumulate) in two passes (log-sum-exp, then normalised sums);
 * the first is skipped when every sequence supplies `lse`. */
starkv_status starkv_score_layer(starkv_state* st, int32_t layer, const starkv_seq* seqs,
                                 int32_t nseq, void* workspace, size_t workspace_bytes,
                                 void* stream);

/* starkv_score_layer for callers that cannot allocate device memory: for
 * example code running where cudaMalloc is forbidden or unavailable, such as a
 * host that hands out only pre-registered buffers, or a plugin inside another
 * runtime that owns every device allocation.  The paper has no counterpart;
 * this is a deployment aid.  Same arguments and results as starkv_score_layer,
 * minus the workspace: the scratch (pass-1 partials and unpooled sums) is one
 * static device array of 16 MiB per device.  The array is reserved on a device
 * when this library's device code is loaded there: at context creation under
 * eager module loading, else (CUDA's default lazy loading) in
 * starkv_init_state, which looks up the array's device address
 * (cudaGetSymbolAddress) with the state's device current; it stays reserved
 * until the process exits.  The call itself allocates no device memory (no
 * cudaMalloc / cudaFree, no allocating library routine).  Every call on a
 * device shares the one array and leaves its last contents there (nothing in
 * it has to start at zero): calls that may overlap on the GPU (different
 * streams, or threads without ordering) race on it and must not be issued.  A
 * batch is rejected with STARKV_ERR_UNSUPPORTED before any launch when it counts
 * more than 16 MiB by a fixed rule, an upper bound of what the kernels use: 2 KiB
 * per (KV group, 128 past tokens begun) and 16 bytes per (KV group, past token), each
 * sequence's tokens rounded up to 4 and its bytes to 256 (1.8 MB per sequence at
 * the 5-screenshot UI-TARS shape); kernel timing must be off (it creates CUDA
 * events).  STARKV_ERR_CUDA if the array could not be reserved when the state
 * was created. */
starkv_status starkv_score_layer_noalloc(starkv_state* st, int32_t layer, const starkv_seq* seqs,
                                         int32_t nseq, void* stream);

/* The attention pass whose logits Eq. (2) scores (Sec. 3.3; App. A.3 counts the
 * compression's Q K^T as shared with the model's attention): for every layer of
 * every sequence and every window row r = (h, i),
 *   attn_o[r]   = sum_{t < L_p} softmax_t(Q_{-i,h} . K[g(h), t] / sqrt(d)) V[g(h), t]
 *   attn_lse[r] = log sum_{t < L_p} exp(Q_{-i,h} . K[g(h), t] / sqrt(d))
 * over the past keys only (the window keys excluded, as in Eq. 2; a model's
 * causal attention for these rows merges in the window keys' part by the
 * usual log-sum-exp rule).  attn_lse is exactly what `lse` takes, so a caller
 * that runs this pass (or its own attention kernel with the same output)
 * lets starkv_step skip its first scoring pass.  Reads k, v, q; writes attn_o
 * (skipped when NULL) and attn_lse (required; -inf and a zero output when
 * L_p = 0).  Tensor cores: Q K^T in bf16, P V with P rounded to fp16 and V
 * converted to fp16 (|v| must stay below 65504), fp32 accumulation, so
 * |attn_o - O| <= 2^-11 sum_t p_t |V_t| + fp32 rounding, and attn_lse carries
 * the fp32 accuracy of the scoring passes.  Workspace from
 * starkv_workspace_bytes. */
starkv_status starkv_window_attention(starkv_state* st, const starkv_seq* seqs, int32_t nseq,
                                      void* workspace, size_t workspace_bytes, void* stream);

/* Sec. 3.3 - 3.7 after the group score map (Eq. 4 to Eq. 10): from
 * S of layer `layer`: s_bar, g*, online MI per group (Eq. 5) -> EMA (Eq. 6) ->
 * prior w (Eq. 7) -> beta; phi_g and the m_g update (Eq. 8) -> D_t (Eq. 9);
 * H_hat and T (Sec. 3.6); s_t = max(s_bar beta D, 0)^(1/T); global top-B with
 * ties to the lower index -> idx ascending (per-KV-head mode: each group's own
 * scores and top-B, see the top of this file).  Writes idx, and score / stats
 * when non-NULL.  Advances this layer's state by one step (n += 1 and both
 * EMAs). */
starkv_status starkv_select(starkv_state* st, int32_t layer, const starkv_seq* seqs,
                            int32_t nseq, void* workspace, size_t workspace_bytes, void* stream);

/* Sec. 3.7, Eq. (11): K' = [K_past[I]; K_rec], V' = [V_past[I]; V_rec] and the
 * same gather of meta, for layer `layer`, from idx.  Bit copies.  In the
 * per-KV-head mode group g gathers its own rows idx[g] (and meta_out[g]). */
starkv_status starkv_compact(starkv_state* st, int32_t layer, const starkv_seq* seqs,
                             int32_t nseq, void* workspace, size_t workspace_bytes, void* stream);

/* Whole compression step of every layer of every sequence (Algorithm 1 for all
 * layers): score, select, compact.  S may be NULL (workspace is used).
 * Equivalent to calling the three per-layer calls for each layer in order. */
starkv_status starkv_step(starkv_state* st, const starkv_seq* seqs, int32_t nseq,
                          void* workspace, size_t workspace_bytes, void* stream);

/* starkv_step with every pointer in `seqs` a HOST pointer (page-locked memory
 * gives asynchronous copies): copies k, v, q, meta to device staging inside
 * `workspace` (size from starkv_workspace_bytes(..., host = 1, ...)), runs the
 * step, and copies k_out, v_out, meta_out, idx (and score / stats / S when
 * non-NULL) back.  Stream-ordered: the host outputs are valid after the stream
 * is synchronised. */
starkv_status starkv_step_host(starkv_state* st, const starkv_seq* seqs, int32_t nseq,
                               void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Paged cache: many sequences' caches in one pool of pages, where they are
 * branched, appended to, compressed and attended over.  (The paper has no
 * counterpart; its compressed caches are what a model decodes over.)
 *
 * A page holds page_size tokens of every layer and KV head under one number:
 *     k, v   bf16  [layer][page][G][page_size][d]   strides of layer and page below
 * Row r of the table is one sequence of len[r] tokens: token j lies in page
 * table[r][j / page_size], slot j % page_size.  refs[p] is the number of rows
 * that hold page p; a page with refs 0 is free.  Entries of a row behind its
 * pages are neither read nor written.
 *
 * Conventions of the calls on it, besides those at the top of this file:
 * - The caller owns pool, table, lengths and counts (DEVICE memory) and starts
 *   them with starkv_pages_reset.  They change in stream order: calls that may
 *   overlap on the GPU must not touch one pool, except that any number may read.
 * - Rows, counts and lengths are read on the device when the call runs, so that a
 *   captured call replays with what the arrays hold then.  `rows` may be NULL for
 *   rows 0 .. n - 1.  A call takes at most 1024 rows (STARKV_ERR_UNSUPPORTED).
 * - What only the device can see is checked there, latched in the device error
 *   word (STARKV_ERR_DEVICE from starkv_check_device_error) and leaves memory
 *   intact.  extend, fork, free, compact and evict are then not carried out at all: too
 *   few free pages, a row out of range or named twice, a length that does not fit, a
 *   page to be shared, let go or copied that is none or that no row holds.  (Counts
 *   below the number of rows that hold a page are not those of this pool; free, compact
 *   and evict report them and lower none below 0.)  A sequence of store or load that
 *   does not fit is passed over; one of the attention calls has zero outputs and lse
 *   -inf.
 * - What is queued behind a refused extend, fork, free, compact or evict counts on
 *   it.  From the refusal until starkv_check_device_error has reported it, the state's
 *   calls that change a pool (extend, fork, free, compact, evict, store) and those that
 *   add to a mass are held back: they leave every byte as it is, and the pool is found
 *   as the refused call found it.  load, bounds and the attention calls run, on the rows
 *   as they are.  (A refusal holds back the state's other pools too, and a store or mass
 *   call that runs at that moment on another stream may be carried out in part: pools
 *   that must not depend on one another take a state each.  starkv_pages_reset is not
 *   held back.)
 * - Supported: page_size 16, 32, 64, 128 or 256; 1 <= n_pages <= 2^20;
 *   1 <= n_rows <= 65536; max_pages * page_size <= 2^24.
 * ------------------------------------------------------------------------- */
typedef struct {
  void* k;                /* bf16, 16-byte aligned                                      */
  void* v;
  int64_t layer_stride;   /* elements between layers, and between the pages of a layer: */
  int64_t page_stride;    /* multiples of 8; a page of a layer is G * page_size * d     */
  int32_t n_pages;
  int32_t page_size;
  int32_t n_rows;
  int32_t max_pages;      /* entries of a table row                                     */
  int32_t* table;         /* [n_rows][max_pages]                                        */
  int32_t* len;           /* [n_rows]                                                   */
  int32_t* refs;          /* [n_pages]                                                  */
} starkv_pages;

/* Tokens outside the pages: for sequence i of n, the last n_tokens[i] tokens of
 * its row, token t of layer l and KV head g at k + i seq_stride + l layer_stride +
 * t token_stride + g head_stride (elements, multiples of 8, not negative), d
 * contiguous elements; v the same.  (starkv_pages_load: rows that do not overlap.) */
typedef struct {
  void* k;                   /* bf16, 16-byte aligned                                  */
  void* v;                   /* or NULL: keys only                                     */
  const int32_t* rows;       /* [n] or NULL                                            */
  const int32_t* n_tokens;   /* [n], 0 .. T, or NULL = T each                          */
  int32_t n, T;
  int64_t seq_stride, layer_stride, token_stride, head_stride;
} starkv_tokens;

/* Queries of the attention calls: for sequence i of n, its row's last n_tokens[i]
 * tokens, token t and head h at q + i q_seq_stride + t q_token_stride + h
 * q_head_stride (elements, multiples of 8, not negative), d contiguous elements;
 * o the same, apart from q and with rows that do not overlap.  What belongs to t >=
 * n_tokens[i] is neither read nor written. */
typedef struct {
  const void* q;             /* bf16, 16-byte aligned, post-RoPE                       */
  void* o;                   /* bf16, 16-byte aligned                                  */
  float* lse;                /* f32 [n][T][H] natural-log normaliser, or NULL          */
  const uint64_t* mask;      /* [n][T], tree attention only                            */
  const int32_t* rows;       /* [n] or NULL                                            */
  const int32_t* n_tokens;   /* [n], 0 .. T, or NULL = T each (another count: device
                                error, and nothing of sequence i is written)           */
  int32_t n, T;
  int64_t q_seq_stride, q_token_stride, q_head_stride;
  int64_t o_seq_stride, o_token_stride, o_head_stride;
} starkv_queries;

/* Bytes of workspace for any call below over at most n rows (sequences), and at
 * most T queries of each. */
starkv_status starkv_pages_workspace_bytes(const starkv_state* st, const starkv_pages* pages, int32_t n, int32_t T,
                                           size_t* bytes);

/* Every row empty, every page free. */
starkv_status starkv_pages_reset(starkv_state* st, const starkv_pages* pages, void* stream);

/* Makes room for n_new[i] >= 0 more tokens of rows[i] (i32 device arrays [n]):
 * len += n_new.  New pages are the free ones with the lowest numbers, in the order
 * of the call's rows.  A last page that is partly filled and that another row
 * holds too (when the call begins) is first copied, its filled slots in every
 * layer.  The new slots hold what they held; starkv_pages_store fills them. */
starkv_status starkv_pages_extend(starkv_state* st, const starkv_pages* pages, const int32_t* rows, const int32_t* n_new,
                                  int32_t n, void* workspace, size_t workspace_bytes, void* stream);

/* Branches: dst[i], an empty row, becomes a copy of src[i] as it is when the call
 * begins.  deep = 0: it shares src's pages.  deep = 1: it gets pages of its own
 * (numbers as for extend) and their filled slots are copied. */
starkv_status starkv_pages_fork(starkv_state* st, const starkv_pages* pages, const int32_t* src, const int32_t* dst, int32_t n,
                                int32_t deep, void* workspace, size_t workspace_bytes, void* stream);

/* Empties rows: len = 0, and one holder less for each of their pages. */
starkv_status starkv_pages_free(starkv_state* st, const starkv_pages* pages, const int32_t* rows, int32_t n, void* stream);

/* starkv_compact of every layer where the cache lies: rows[i] (L = seqs[i].L
 * tokens, which must be its length) keeps the tokens idx and the last w, in that
 * order, in pages of its own (numbers as for extend, taken before the old pages
 * are let go; other holders of those keep them): len = B + w.  Reads idx, L,
 * budget, meta and its strides of seqs (host values, fixed in a captured call), writes
 * meta_out where meta is given; the other buffers may be NULL, and slots are not
 * looked at.  In the per-KV-head mode
 * group g keeps idx[g].  Error (device): an index outside the past tokens keeps token 0. */
starkv_status starkv_pages_compact(starkv_state* st, const starkv_pages* pages, const int32_t* rows, const starkv_seq* seqs,
                                   int32_t nseq, void* workspace, size_t workspace_bytes, void* stream);

/* Bit copies of tokens into the pages (store) or out of them (load), layers
 * [layer0, layer0 + n_layers).  A page that more than one row holds is not
 * written to, nor is a row that two sequences of a store with tokens name (device
 * error).  load may name a row any number of times. */
starkv_status starkv_pages_store(starkv_state* st, const starkv_pages* pages, int32_t layer0, int32_t n_layers,
                                 const starkv_tokens* tokens, void* stream);
starkv_status starkv_pages_load(starkv_state* st, const starkv_pages* pages, int32_t layer0, int32_t n_layers,
                                const starkv_tokens* tokens, void* stream);

/* Attention of drafted tokens over a row's cache, one layer.  The last n =
 * n_tokens[i] <= 64 tokens of the row (L tokens, the drafted ones stored) are a
 * tree: query t sees the keys j < L - n, and drafted token b where bit b of
 * mask[i][t] is set (its own bit too, if it is to see itself; bits from n on are
 * not looked at).  With z_j = q . K[g(h), j] / sqrt(d) over the keys seen,
 *   o = sum_j softmax_j(z) V[g(h), j],   lse = log sum_j exp(z_j);
 * a query that sees none has o = 0 and lse = -inf.  K and V that a query does not
 * see do not reach its output, whatever they hold (V that is not finite and is seen by
 * some queries only costs time: their rows are taken again key by key).  A seen V of
 * infinity gives infinity, or NaN with its opposite.  Sums are held in fp32 against a
 * weight of up to 2^8: values above 2^119 / L may overflow. */
starkv_status starkv_tree_attention(starkv_state* st, const starkv_pages* pages, int32_t layer, const starkv_queries* queries,
                                    void* workspace, size_t workspace_bytes, void* stream);

/* The same with a sliding window and sinks: query t, the token at position i = L -
 * n + t of its row, sees the keys j <= i with j < n_sink or j > i - window
 * (n_sink, window >= 0; window >= L is plain causal attention).  T = 1 is decoding,
 * larger T a chunk of a prompt (T * H / G <= 2^17). */
starkv_status starkv_sink_attention(starkv_state* st, const starkv_pages* pages, int32_t layer, const starkv_queries* queries,
                                    int32_t n_sink, int32_t window, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Attention mass: what each cached token has had of the queries' attention.
 *
 * One f32 per layer, row, KV head and token: token j of row r at mass + layer
 * layer_stride + r row_stride + g group_stride + j, max_pages * page_size tokens a
 * row, rows that do not overlap.  It belongs to the row, not to its pages: a branch
 * takes a copy of its source's rows along, an emptied row leaves values that nothing
 * reads. */
typedef struct {
  float* mass;            /* f32, device memory, 4-byte aligned                        */
  int64_t layer_stride;   /* elements, not negative                                    */
  int64_t row_stride;
  int64_t group_stride;
  float decay;            /* finite, >= 0: factor of what a token has had so far       */
} starkv_mass;

/* Adds the weights of an attention call, one layer: after starkv_tree_attention or
 * starkv_sink_attention with the same queries (q, lse as it was written, mask, rows,
 * n_tokens; o is not looked at), for row rows[i] of L tokens whose last n are the queries,
 *   mass[g][j] = (j < L - n ? decay mass[g][j] : 0)
 *                + sum_t sum_{h in g} [t sees j] exp(q[t, h] . K[g, j] / sqrt(d) - lse[t, h])
 * for j < L, in fp32, the same from call to call.  A row's new tokens start at 0, so
 * that rows need not be cleared; n = 0 leaves a row as it is.  Weights are what the
 * formula has where q, a seen K or lse is not finite; what a query does not see adds
 * nothing, whatever it holds.  A sequence that does not fit, or a row that two sequences
 * with queries name, is left as it is (device error), and so are the tokens of a page
 * that is none; also every row behind a refused call (as for the calls that change a
 * pool).  After STARKV_ERR_TIMEOUT some tokens of the layer have their mass after the call
 * and the others that before it.  T and T * H / G as for the attention. */
starkv_status starkv_tree_mass(starkv_state* st, const starkv_pages* pages, int32_t layer, const starkv_queries* queries,
                               const starkv_mass* mass, void* workspace, size_t workspace_bytes, void* stream);
starkv_status starkv_sink_mass(starkv_state* st, const starkv_pages* pages, int32_t layer, const starkv_queries* queries,
                               int32_t n_sink, int32_t window, const starkv_mass* mass, void* workspace, size_t workspace_bytes,
                               void* stream);

/* Eviction by mass: starkv_pages_compact, with the tokens chosen here.  Every layer of
 * rows[i] keeps the budget past tokens (j < L - w) of greatest mass and the last w; in the
 * per-KV-head mode group g by mass[g], else all groups by the sum over them (in 64 bits).
 * Equal ones: the lower j; a NaN counts as +infinity.  Writes the chosen ones to idx
 * (ascending), and moves the kept tokens' mass to their new places in the row (decay is
 * not looked at).  A refused call changes nothing, idx and mass included. */
starkv_status starkv_pages_evict(starkv_state* st, const starkv_pages* pages, const int32_t* rows, const starkv_seq* seqs,
                                 int32_t nseq, const starkv_mass* mass, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Bounds of pages, and attention over pages that each query chooses by them.
 *
 * Per layer, page and KV head the least and the greatest key of every channel: bf16
 * [layer][page][G][2][d], the least ones first, strides of layer and page below.  They
 * belong to the pages, as K and V do: rows that share a page share them. */
typedef struct {
  void* b;                /* bf16, device memory, 16-byte aligned                      */
  int64_t layer_stride;   /* elements, multiples of 8, not negative                    */
  int64_t page_stride;
} starkv_bounds;

/* Bounds of the pages that hold the last n_tokens[i] (0 .. T; NULL: T) tokens of row
 * rows[i], layers [layer0, layer0 + n_layers), over the slots that hold tokens of that row:
 * after tokens have been stored, and after a row has been compacted or its shared last page
 * copied (extend), for the pages that changed.  What other pages have stays.  NaN where a
 * key is NaN.  A sequence that does not fit, or a page that is none, is passed over (device
 * error).  The pages' refs are not looked at, and a row may be named more than once. */
starkv_status starkv_pages_bounds(starkv_state* st, const starkv_pages* pages, int32_t layer0, int32_t n_layers,
                                  const starkv_bounds* bounds, const int32_t* rows, const int32_t* n_tokens, int32_t n, int32_t T,
                                  void* stream);

/* Bytes of workspace for a sparse attention call of n rows, T queries each and n_chosen pages. */
starkv_status starkv_sparse_workspace_bytes(const starkv_state* st, const starkv_pages* pages, int32_t n, int32_t T, int32_t n_chosen,
                                            size_t* bytes);

/* Attention over chosen pages, one layer.  Query t (of n = n_tokens[i], as for
 * starkv_sink_attention; mask is not looked at) is the token at position i = L - n + t of its
 * row, in the row's page i / page_size.  For each KV head it attends over the tokens j <= i
 * of n_chosen pages (of all pages up to its own, where they are not more): the first n_first,
 * the last n_last up to its own, and of the others those with the greatest
 *   score = sum_c (up_c hi_c + down_c lo_c),  up = sum_{h in g} max(q_h, 0),  down = sum_{h in g} min(q_h, 0),
 * lo and hi the page's bounds: the most that the sum of the heads' logits with one of its keys
 * can be.  Their order is that of 64 bits; equal ones: the lower page; a NaN counts as +infinity.
 * n_first >= 0, n_last >= 1, n_first + n_last <= n_chosen.  chosen (i32 [n][T][G][n_chosen],
 * or NULL) gets the pages' places in the row, ascending, -1 behind them.  o and lse are those of
 * the keys attended over, as for the calls above.  A page that is none (device error) scores 0,
 * and its K and V count as zeros where it is taken. */
starkv_status starkv_sparse_attention(starkv_state* st, const starkv_pages* pages, int32_t layer, const starkv_queries* queries,
                                      const starkv_bounds* bounds, int32_t n_first, int32_t n_last, int32_t n_chosen, int32_t* chosen,
                                      void* workspace, size_t workspace_bytes, void* stream);

/* Reads and clears the state's device error word (synchronises `stream`).
 * Returns STARKV_OK, STARKV_ERR_DEVICE or STARKV_ERR_TIMEOUT. */
starkv_status starkv_check_device_error(starkv_state* st, void* stream);

/* Limit, in nanoseconds, of every bounded device-side wait of this state's
 * kernels (default 1e9).  A wait that runs out stops its kernel early and
 * latches STARKV_ERR_TIMEOUT in the device error word; before it exits or
 * releases tensor memory the kernel still waits for the copies and MMAs it
 * has already issued, for max(limit, 2 s).  (The paged attention's waits for rows
 * that are taken key by key, see there, count from those rows' last unit of 64 keys.) */
starkv_status starkv_set_wait_limit(starkv_state* st, uint64_t limit_ns);

/* Self-test of the failure path that every bounded device wait shares: one
 * thread of a one-block kernel waits on a shared-memory barrier that nothing
 * completes; after `limit_ns` (1e3 .. 1e9) the wait gives up, latches
 * STARKV_ERR_TIMEOUT in the state's device error word and the kernel
 * returns, so the context stays usable.  Stream-ordered; the next
 * starkv_check_device_error reports STARKV_ERR_TIMEOUT (and clears it).
 * STARKV_ERR_INVALID_ARG for a NULL state or a limit out of range. */
starkv_status starkv_selftest_wait(starkv_state* st, uint64_t limit_ns, void* stream);

/* Kernels of the library, for starkv_kernel_times. */
enum {
  STARKV_KERNEL_SCORE_LSE = 0,    /* scoring pass 1: per-row log-sum-exp (Sec. 3.3)        */
  STARKV_KERNEL_SCORE_ACCUM = 1,  /* scoring pass 2: normalised group sums (Eqs. 2-4)      */
  STARKV_KERNEL_POOL = 2,         /* AvgPool1D + group mean (Eqs. 3-4), per-layer calls    */
  STARKV_KERNEL_CALIBRATE = 3,    /* MI, phi, prior, temperature, fused score, top-B
                                     (Sec. 3.4-3.7): one cluster of min(G, 8) CTAs per
                                     layer                                                 */
  STARKV_KERNEL_COMPACT = 4,      /* KV gather (Eq. 11)                                    */
  STARKV_KERNEL_ATTENTION = 5,    /* window-row attention over the past keys (pieces)      */
  STARKV_KERNEL_ATTN_COMBINE = 6, /* merge of its pieces into attn_o / attn_lse            */
  STARKV_KERNEL_PAGE_BOOK = 7,    /* paged cache: tables, counts, free pages               */
  STARKV_KERNEL_PAGE_COPY = 8,    /* its page copies (extend, deep fork)                   */
  STARKV_KERNEL_PAGE_GATHER = 9,  /* its compaction (Eq. 11 on pages)                      */
  STARKV_KERNEL_PAGE_MOVE = 10,   /* tokens into and out of pages                          */
  STARKV_KERNEL_PAGED_ATTENTION = 11,  /* tree, sink and sparse attention                  */
  STARKV_KERNEL_PAGED_COMBINE = 12,    /* merge of its parts                               */
  STARKV_KERNEL_MASS = 13,             /* attention mass                                   */
  STARKV_KERNEL_MASS_SUM = 14,         /* sum of its parts (many queries)                  */
  STARKV_KERNEL_MASS_SELECT = 15,      /* tokens that stay by it                           */
  STARKV_KERNEL_PAGE_BOUNDS = 16,      /* least and greatest keys of pages                 */
  STARKV_KERNEL_PAGE_CHOOSE = 17,      /* pages that queries attend over                   */
  STARKV_NUM_KERNELS = 18
};

/* Kernel timing, a profiling aid.  While `on` is non-zero every kernel launch
 * made for this state is bracketed by a CUDA event pair on its stream. */
starkv_status starkv_set_timing(starkv_state* st, int32_t on);

/* Per kernel kind (arrays of STARKV_NUM_KERNELS): launches made and, while
 * timing was on, their summed device time in milliseconds, since the last
 * call.  Waits for the recorded events.  Launch counts are kept with timing
 * off too (total_ms then stays 0).  Either array may be NULL. */
starkv_status starkv_kernel_times(starkv_state* st, int64_t* launches, float* total_ms);

/* Launches of scoring pass 2 that went through their tiles backwards, since the
 * state's creation (taken when the window rows of a group are at most 128 and the
 * launch's K exceeds the device's L2; the results are the same either way). */
starkv_status starkv_backward_launches(const starkv_state* st, int64_t* launches);

/* Thread-local message describing the last non-OK status on this thread. */
const char* starkv_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* STARKV_H */
