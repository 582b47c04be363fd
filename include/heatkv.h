/*
 * heatkv.h -- C ABI of the B200 (sm_100a) HeatKV hot path.
 *
 * HeatKV (head-tuned KV-cache compression for visual autoregressive, next-scale
 * models) prunes the KV cache per attention head and per source scale with a static
 * schedule derived from calibrated attention statistics.  This library holds the
 * data-parallel part: the calibration reduction (Sec. 3.1), the schedule builder
 * (Sec. 3.2, 3.3, Appendix A), the per-head cache with append / eviction, and the
 * per-scale-step attention over the retained keys.
 *
 * Conventions
 *  - Scales ("steps"), layers and heads are 0-based here: step = k-1 for the paper's
 *    scale k, so t[step] tokens are generated at `step` and c[step] = t[0]+..+t[step].
 *  - Activations are bf16, shaped [n_seq, H, t_step, d] with d contiguous; the other
 *    three strides are given in elements by heatkv_strides (NULL = densely packed).
 *    Base pointers must be 16-byte aligned and strides multiples of 8 elements.  A head or
 *    sequence stride of inputs may be 0: one tensor shared by all heads or sequences.
 *  - Every pointer is marked HOST or DEVICE.  Device buffers belong to the caller (the
 *    library never allocates or frees device memory); the library owns only the host
 *    objects behind heatkv_ctx / heatkv_schedule.  Kernels are enqueued on the given
 *    CUDA stream (a cudaStream_t passed as void*, NULL = default stream) and calls return
 *    without waiting, except the calls documented as synchronising.
 *  - Every function returns HEATKV_OK (0) or a negative heatkv_status.  Nothing throws or
 *    aborts across this boundary; a call that fails leaves cache and context unchanged.
 *  - A context is not thread-safe; use one context per thread or lock around it.
 *  - The kernels of one context share work counters and scratch inside its arena, so they must
 *    not overlap on the GPU: enqueue a context's calls on one stream, or order the streams
 *    with events.  After HEATKV_ERR_DEVICE_TIMEOUT (heatkv_device_status) a context stays in
 *    that state; destroy it and create a new one.
 */
#ifndef HEATKV_H_
#define HEATKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define HEATKV_MAX_K 16          /* at most 16 scales (mask words are 16 bit)        */
#define HEATKV_MAX_BATCH 128     /* sequences per attention / append call            */
#define HEATKV_PAGE_TOKENS 64    /* rows per cache page and per key half-tile        */

typedef enum {
  HEATKV_OK = 0,
  HEATKV_ERR_INVALID_ARG = -1,
  HEATKV_ERR_SHAPE_MISMATCH = -2,
  HEATKV_ERR_BUDGET_INFEASIBLE = -3,   /* b*c_{K-1} < c_s, or the removal list ran out */
  HEATKV_ERR_OUT_OF_PAGES = -4,        /* pool or metadata region exhausted            */
  HEATKV_ERR_BAD_STEP_ORDER = -5,
  HEATKV_ERR_NAN_SCORE = -6,
  HEATKV_ERR_DEVICE_TIMEOUT = -7,      /* a bounded device-side wait gave up           */
  HEATKV_ERR_CUDA = -8,
  HEATKV_ERR_HOST_MEMORY = -9,
  HEATKV_ERR_TOO_LARGE = -10           /* the call needs more built-in scratch than the library holds */
} heatkv_status;

typedef enum { HEATKV_LAYOUT_RAGGED = 0, HEATKV_LAYOUT_PAGED = 1 } heatkv_layout;

typedef enum {
  HEATKV_POLICY_HEATKV = 0,   /* Algorithm 1, head-scale units, orders O_i from S-CAS      */
  HEATKV_POLICY_BINARY = 1,   /* Algorithm 1, head units, one order O from CAS            */
  HEATKV_POLICY_NAIVE = 2,    /* Sec. 3.3 boundary policy: prune before a scale, not after */
  HEATKV_POLICY_EXPLICIT = 3  /* per-head token fraction (no counterpart in the paper)     */
} heatkv_policy;

typedef enum {
  HEATKV_ACCOUNT_PHYSICAL = 0, /* layers not yet run hold what they held at scale start   */
  HEATKV_ACCOUNT_LITERAL = 1   /* Algorithm 2 exactly as printed                          */
} heatkv_accounting;

typedef enum {
  HEATKV_KERNEL_AUTO = 0,      /* tensor-memory kernel for steps of >= 256 queries (>= 128 once a call holds
                                  64 (sequence, head) units; >= 48 in calibration with an attention output),
                                  generic otherwise */
  HEATKV_KERNEL_GENERIC = 1,   /* warp-level MMA kernel for every step                    */
  HEATKV_KERNEL_TCGEN05 = 2    /* tcgen05 / TMEM / TMA kernel wherever its shape rules allow */
} heatkv_kernel_choice;

typedef enum {
  HEATKV_CACHE_BF16 = 0,       /* rows stored verbatim                                            */
  HEATKV_CACHE_FP8_E4M3 = 1    /* rows stored as 8-bit codes plus one exponent byte (see below)    */
} heatkv_cache_dtype;

typedef struct heatkv_ctx heatkv_ctx;
typedef struct heatkv_schedule heatkv_schedule;

typedef struct {
  int32_t L, H, d, K;            /* layers, heads per layer, head dim (64 or 128), scales  */
  int32_t t[HEATKV_MAX_K];       /* tokens per scale, t_k = w_k * h_k (Sec. 3.1)           */
  int32_t s;                     /* sink scales always kept (Sec. 3.2); 0 allowed          */
  int32_t layout;                /* heatkv_layout                                           */
  int32_t kernel;                /* heatkv_kernel_choice                                    */
  float sm_scale;                /* logit scale; <= 0 selects 1/sqrt(d)                    */
  void* arena;                   /* DEVICE, caller-owned, 1024-byte aligned                */
  uint64_t arena_bytes;          /* metadata region + scratch region + K pool + V pool     */
  uint64_t meta_bytes;           /* bytes of the arena set aside for plans; 0 = default    */
  uint64_t scratch_bytes;        /* bytes of the arena for partial results of heads whose key range is
                                    split over several CTAs, 1/32 to 1/8 of it (at most 32 MiB) for
                                    the plans' merged tables; 0 = default (1/8 of the arena, at most
                                    128 MiB); too little only disables both                         */
  int32_t cache_dtype;           /* heatkv_cache_dtype; FP8_E4M3 needs the paged layout                    */
  int32_t reserved0;
  uint64_t stage_bytes;          /* FP8_E4M3 only: bytes of the arena for the bf16 staging rows one attention
                                    call expands its visible keys into; 0 = default (1/8 of the arena)     */
} heatkv_config;

typedef struct {                 /* element strides of the [n_seq, H, t, d] activations    */
  int64_t q_seq, q_head, q_tok;
  int64_t kv_seq, kv_head, kv_tok;   /* shared by k and v                                  */
  int64_t o_seq, o_head, o_tok;
} heatkv_strides;

typedef struct {                 /* which kernels a context has launched so far             */
  uint32_t tcgen05_attention_ready;    /* 1: the tensor-memory attention kernel is set up on this device */
  uint32_t tcgen05_calibration_ready;  /* 1: the tensor-memory calibration kernel is set up               */
  uint64_t attention_tcgen05;    /* launches of the tcgen05 / TMEM / TMA attention kernel (carries the cache
                                    update of heatkv_attention_append in the paged layout)               */
  uint64_t attention_generic;    /* launches of the warp-level attention kernel                          */
  uint64_t calibration_tcgen05, calibration_generic;
  uint64_t append, compact;      /* stand-alone cache-update kernels                                     */
  uint64_t other;                /* small helper kernels (fixed-order reduction of the static-scratch call) */
} heatkv_kernel_stats;

/* The form in which an attention call was launched (heatkv_last_attention). */
typedef enum heatkv_attention_kernel {
  HEATKV_ATTENTION_NONE = 0,           /* no attention call has been launched yet                               */
  HEATKV_ATTENTION_GENERIC = 1,        /* warp-level kernels; the other fields are 0                            */
  HEATKV_ATTENTION_TCGEN05 = 2,        /* attn_tc_kernel                                                        */
  HEATKV_ATTENTION_CTA_PAIRS = 3       /* attn_pair_kernel: whole heads, 256 queries an item                    */
} heatkv_attention_kernel;
typedef struct heatkv_attention_form {
  int32_t kernel;          /* heatkv_attention_kernel                                                               */
  int32_t items;           /* work items of the launch (an upper bound where the call mixes schedules)              */
  int32_t longest_piece;   /* key tiles of the longest piece of a head that was cut (0: none was; where the call
                              mixes schedules the longest run a piece may have)                                     */
  int32_t lone;            /* 1: some items are one query tile of 128, the others a pair of them, and nothing is cut */
} heatkv_attention_form;

typedef struct {
  uint64_t pool_rows;            /* rows (tokens) the K pool and the V pool can hold        */
  uint64_t reserved_rows;        /* rows reserved by open sequences                         */
  uint64_t used_tokens;          /* tokens held right now by open sequences                 */
  uint64_t peak_reserved_rows;   /* high-water mark of reserved_rows                        */
  uint64_t meta_bytes_used;
  uint32_t open_seqs;
  uint32_t plans;                /* schedules whose plan is resident                        */
} heatkv_alloc_stats;

/* fp8 cache (cache_dtype = HEATKV_CACHE_FP8_E4M3).  The paper names quantisation of the cache only as an
 * orthogonal direction (Sec. 5 and the conclusion) and defines no format; this one is the library's own.
 * A cached row (the d values of one token of one head, K or V) is stored as d codes of the OCP 8-bit
 * floating-point format E4M3 (1 sign, 4 exponent bits with bias 7, 3 mantissa bits, subnormals, no
 * infinities, largest finite value 448) plus one signed exponent byte e:
 *     code_j = round-to-nearest-even on the E4M3 grid of x_j * 2^-e,
 *     e = the smallest integer >= -120 with max_j |x_j| * 2^-e <= 448   (all-zero row: e = -120),
 * so a row costs d + 1 bytes instead of 2 d.  Reading gives x^_j = value(code_j) * 2^e, which a bf16 holds
 * exactly.  Attention in such a context is attention over x^ for the cached scales (the step's own K/V come
 * from k_new / v_new unquantised, as always): before the attention kernel runs, the call expands the visible
 * head-scales of its (layer, step) into bf16 staging rows inside the arena (stage_bytes), and the attention
 * kernels read those (the warp-level kernel of the smallest steps reads the codes themselves); the update after the layer
 * quantises the new rows on their way into the pool.  Inputs must be finite.  Only the paged layout is supported; in
 * heatkv_attention_append the update rides on the attention launch of the warp-level kernel (small steps) and on the
 * expansion before the tensor-memory kernel.  A call whose sequences need more staging rows than stage_bytes holds returns
 * HEATKV_ERR_OUT_OF_PAGES (rows needed per sequence: the largest number of visible 64-row half-tiles of any
 * (layer, step) of its schedule, times 64).
 *
 * Context: validates the shape, splits the arena into a metadata region and the K / V
 * pools, zero-fills the pools (enqueued on `stream`).  The arena must outlive the context.
 * With kernel = HEATKV_KERNEL_AUTO or HEATKV_KERNEL_TCGEN05 the tensor-memory kernels are set up here; if that
 * fails on a device of compute capability 10.x (or on any device under HEATKV_KERNEL_TCGEN05) the call returns
 * HEATKV_ERR_CUDA: a context never falls back to the warp-level kernel behind the caller's back.  Which kernel
 * ran is reported by heatkv_kernel_launches. */
int heatkv_create(const heatkv_config* cfg /*HOST*/, void* stream, heatkv_ctx** out /*HOST*/);
int heatkv_destroy(heatkv_ctx* ctx);

/* Sec. 3.1, Eq. 2 -- scale attention mass.  For one (layer, step) and n_seq calibration
 * sequences: attention of the t[step] queries over ALL c[step] keys (no pruning), fused
 * with the per-row probability mass on each source scale; the mean over rows is added to
 * beta_accum[layer][h][step][0..step] for every head (sum over the n_seq sequences; every
 * sequence counts as one data point d).  The attention matrix is never written out.  Against 64 bits the
 * masses of 13 scales are off by 4e-7 of themselves on average without an output, where one exponential in three
 * is a cubic (5e-6 was the largest seen), and by 1e-7 with one (1e-6).
 *   q       DEVICE bf16 [n_seq,H,t[step],d]   strides q_*
 *   k_full  DEVICE bf16 [n_seq,H,c[step],d]   strides kv_*  (all scales up to `step`)
 *   v_full  DEVICE bf16 like k_full, or NULL when `out` is NULL
 *   seg_bias DEVICE fp32 [H][K] additive logit bias per source scale (-inf takes a scale out; one that a query
 *           sees must remain), or NULL
 *   beta_accum DEVICE fp32 [L][H][K][K], zero-initialised by the caller before the first call
 *   out     DEVICE bf16 [n_seq,H,t[step],d] strides o_*: the attention output, or NULL
 * Without an output the o_* strides are not read (they may be left zero).                */
int heatkv_calibrate_scores(heatkv_ctx* ctx, int layer, int step, int n_seq, const void* q,
                            const void* k_full, const void* v_full, const heatkv_strides* st,
                            const float* seg_bias, float* beta_accum, void* out, void* stream);

/* Sec. 3.1, Eq. 2 for the steps step_begin .. step_end - 1 of one layer in one call: offline calibration from
 * recorded activations, where the queries and keys of every scale of a sample are at hand (the beta rows of different
 * steps are independent of one another).  The steps the tensor-memory kernel takes run as ONE launch whose CTAs are
 * dispatched longest first, which evens out the rounds that a launch per step leaves partly filled; the small steps
 * share one launch of the generic kernel.  Results agree with step-by-step heatkv_calibrate_scores calls up to the
 * order of the fp32 sums.
 *   q_all   DEVICE bf16 [n_seq,H,c[step_end-1],d]  the queries of all scales, token axis = the scales one after the
 *           other, strides q_*
 *   k_all   DEVICE bf16 [n_seq,H,c[step_end-1],d]  the keys, same layout, strides kv_*
 *   seg_bias DEVICE fp32 [step_end][H][K]: the bias of step k at seg_bias + k*H*K, or NULL
 *   beta_accum as in heatkv_calibrate_scores.  The o_* strides are not read. */
int heatkv_calibrate_scores_steps(heatkv_ctx* ctx, int layer, int step_begin, int step_end, int n_seq, const void* q_all,
                                  const void* k_all, const heatkv_strides* st, const float* seg_bias, float* beta_accum,
                                  void* stream);

/* No counterpart in the paper: heatkv_calibrate_scores for callers that must not allocate device
 * memory while they run -- code inside a serving loop whose memory pool is fixed at start-up, a plug-in
 * of a host application that owns the allocator, a caller between stream-ordered allocator
 * checkpoints.  It computes the same beta update (no attention output, so no v_full / out), but every
 * CTA writes its partial masses into a 4 MiB array that is part of the library image (held by every GPU
 * that loads the library until the process exits) and a second small kernel adds them to beta_accum in a
 * fixed order; the call itself makes no cudaMalloc / cudaFree and uses no allocating library routine.
 *   Limit: ceil(t[step] / 64) * H * n_seq * 64 partial slots must fit in 2^20 floats, i.e. at most
 *   16 384 (query tile, head, sequence) CTAs; larger calls return HEATKV_ERR_TOO_LARGE and launch nothing.
 *   The first call on a device looks up the array's device address (once per device, on the device that
 *   is current); make that first call before any stream capture.
 *   All calls share the one array and it keeps the last call's contents: every slot a call reads is
 *   written by that call first, so nothing needs clearing, but two calls whose kernels overlap on the
 *   GPU (different streams) race on it -- keep them on one stream or order them yourself.
 * Arguments as in heatkv_calibrate_scores (the o_* strides are not read).  Results agree with it up to the
 * order of the fp32 sums. */
int heatkv_calibrate_scores_static(heatkv_ctx* ctx, int layer, int step, int n_seq, const void* q,
                                   const void* k_full, const heatkv_strides* st, const float* seg_bias,
                                   float* beta_accum, void* stream);

/* Text after Eq. 2, Eq. 3 and Eq. 4 -- copies beta_accum to the host (synchronises
 * `stream`), divides by n_samples = |D| and reduces in fp64:
 *   beta HOST [L][H][K][K], scas HOST [L][H][K] (0 outside s < k < K), cas HOST [L][H].
 * Any of the three outputs may be NULL.  HEATKV_ERR_NAN_SCORE if a value is not finite. */
int heatkv_finalize_scores(heatkv_ctx* ctx, const float* beta_accum /*DEVICE*/, int n_samples,
                           double* beta, double* scas, double* cas, void* stream);

/* Sec. 3.2 (Eq. 5), Sec. 3.3 (Algorithm 1), Appendix A (Algorithm 2) -- pure host code.
 * Ranks heads per source scale by ascending S-CAS (ties: ascending l*H+h), computes N_k,
 * the sets G_k, E_k (GreedyEarlyPruning) and A_k = G_{k-1} u E_k for every scale.
 *   scas HOST [L][H][K]  (HEATKV, NAIVE)      cas HOST [L][H]  (BINARY)
 *   fraction HOST [L][H] (EXPLICIT: the head stores scales 1..j, the largest prefix with
 *            c_j <= ceil(fraction * c_{K-1}), at least the sinks, and never evicts)
 *   b in (0,1]: the budget is B = floor(b * L*H * c_{K-1}) tokens (ignored by EXPLICIT).
 * Only L, H, K, t, s of cfg are read.                                                    */
int heatkv_build_schedule(const heatkv_config* cfg, const double* scas, const double* cas,
                          int policy, int accounting, double b, const double* fraction,
                          heatkv_schedule** out);
int heatkv_schedule_free(heatkv_schedule* sch);

/* Schedule as bit masks, HOST arrays of K*L*H uint16 indexed [step][layer][head]:
 *   attn_mask bit i (i < step): source scale i is in the cache and visible at `step`,
 *             i.e. i is a sink or (i,l,h) is not in A_step;
 *   keep_mask bit i (i <= step): source scale i is stored once the layer ran at `step`,
 *             i.e. i is a sink or (i,l,h) is not in G_step (last step: unchanged, nothing
 *             is appended because the last scale is never cached).
 *   n_k HOST [K] (N_k, 0 for the last step), budget_tokens = B (-1 for EXPLICIT).
 * Any output may be NULL.                                                                */
int heatkv_schedule_masks(const heatkv_schedule* sch, uint16_t* attn_mask, uint16_t* keep_mask,
                          int32_t* n_k, int64_t* budget_tokens);

/* Peak number of cached tokens over all checkpoints (scale start and after every layer)
 * and the pool rows one sequence reserves under `layout`.                                */
int heatkv_schedule_footprint(const heatkv_schedule* sch, int layout, int64_t* peak_tokens,
                              int64_t* reserved_rows);

/* The plan a sequence of this schedule runs under `layout`, as the flat int32 table the
 * kernels read (HOST copy, for inspection and tests): a 24-word header {L, H, K, n_desc,
 * word offsets of: desc, attn_begin, attn_cnt, app_begin, app_cnt, order, move, pre_begin,
 * pre_cnt, post_begin, post_cnt, then n_move, total_words, 1 spare, word offsets of run_desc,
 * run_begin, run_cnt, 3 spare} followed by the tables.
 * desc = {row relative to the reservation, n_valid | source_scale << 8}; move = {src, dst, n, 0};
 * the per-(step, layer, head) tables are indexed (step*L + layer)*H + head.  run_* = attn_* for
 * calls without seg_bias: rows that follow one another share half-tiles across source scales.
 * Call with words == NULL to get *n_words, then with a buffer of that many int32.        */
int heatkv_schedule_plan(const heatkv_schedule* sch, int layout, int32_t* words, int64_t* n_words);
/* The same for a context with the fp8 cache (paged layout): the attention descriptors of every (step, layer) carry
 * staging rows -- consecutive 64-row slots in descriptor order across the layer's heads -- and header word 17 is the
 * word offset of an extra table int32[n_desc] with the pool row behind every descriptor (append descriptors keep
 * pool rows); word 21 is the same for run_desc.  *stage_rows (optional) = staging rows one sequence needs in an attention call: 64 per visible
 * half-tile of its busiest (step, layer).  Pure host code. */
int heatkv_schedule_plan_fp8(const heatkv_schedule* sch, int32_t* words, int64_t* n_words, int64_t* stage_rows);

/* Admit / retire one image.  Opening reserves the sequence's rows for its whole life (the
 * schedule is static, so the reservation and every page table are known up front) and, on
 * first use of a schedule, uploads its plan on `stream`.  A plan keeps its place while a
 * sequence uses it; plans (or their merged tables) that none uses make way when a region is
 * full.  HEATKV_ERR_OUT_OF_PAGES if the pool or the metadata region cannot hold it.      */
int heatkv_seq_open(heatkv_ctx* ctx, const heatkv_schedule* sch, void* stream, int* seq_id);
int heatkv_seq_close(heatkv_ctx* ctx, int seq_id);

/* Sec. 3.3 -- cache update for one layer.
 *   k_new != NULL: after layer `layer` ran at `step`: store the step's K/V for every head
 *     whose (step,l,h) is not in G_step and drop the head-scales of G_step \ A_step of this
 *     layer (Sec. 3.3: these leave right after their own layer has run).  The last step stores
 *     nothing.  k_new, v_new DEVICE bf16 [n_seq,H,t[step],d], strides kv_*.
 *   k_new == NULL: before `step` starts: drop the head-scales of E_step (Sec. 3.3, Algorithm 1:
 *     the early-pruned set, gone before the scale begins) in `layer`, or in all layers when layer < 0.
 * Survivors keep their order.  In the paged layout eviction moves no data.               */
int heatkv_append_compact(heatkv_ctx* ctx, const int* seq_ids /*HOST*/, int n_seq, int layer,
                          int step, const void* k_new, const void* v_new,
                          const heatkv_strides* st, void* stream);

/* Attention of one layer at one step (Sec. 3.1 notation; Sec. 3.3 for the visible set):
 * out = softmax(sm_scale * q K^T + bias) V over the retained prior head-scales (ascending
 * scale, raster order inside) followed by the step's own t[step] keys, which always come
 * from k_new / v_new and are all visible.  bf16 operands, fp32 accumulation, probabilities
 * rounded to bf16 before the PV product.
 *   q, k_new, v_new DEVICE bf16 [n_seq,H,t[step],d]; seg_bias DEVICE fp32 [H][K] (-inf takes a
 *   scale out, as in heatkv_calibrate_scores) or NULL;
 *   out DEVICE bf16 [n_seq,H,t[step],d].                                                 */
int heatkv_scale_attention(heatkv_ctx* ctx, const int* seq_ids /*HOST*/, int n_seq, int layer,
                           int step, const void* q, const void* k_new, const void* v_new,
                           const heatkv_strides* st, const float* seg_bias, void* out,
                           void* stream);

/* heatkv_scale_attention followed by heatkv_append_compact(k_new != NULL) for the same (layer, step), as one
 * call: the order a model issues them in (Sec. 3.3: G_step \ A_step is evicted as soon as its layer has run).
 * In the paged layout both run in ONE kernel launch (the plan releases the pages of G_step \ A_step only
 * after the layer's append, so the new scale never lands on a page this step's attention still reads): on
 * the tensor-memory kernel two spare warps per SM copy the new rows beside the attention work, whatever the
 * update's size; on the generic kernel the copies are extra CTAs of the attention launch while the update
 * is small (up to 8 MiB of K/V, a launch-bound copy), and a larger update keeps its own bandwidth-bound
 * kernel.  In the ragged layout the in-place compaction must follow the attention, so
 * there the separate kernels run.  Arguments as in heatkv_scale_attention. */
int heatkv_attention_append(heatkv_ctx* ctx, const int* seq_ids /*HOST*/, int n_seq, int layer, int step,
                            const void* q, const void* k_new, const void* v_new, const heatkv_strides* st,
                            const float* seg_bias, void* out, void* stream);

/* How the tensor-memory attention kernel would cut the work of heatkv_scale_attention(seq_ids, layer,
 * step) without seg_bias: *split_tiles = longest piece, in 128-key tiles, among the heads whose key range is cut (0: every
 * work item takes a whole head's key range), *items = work items of the launch (an upper bound when the
 * call mixes schedules).  A cut head's pieces leave partial results in the arena's scratch region, where
 * the last to arrive merges them.  The choice (a piece count per head) minimises an estimate of the launch's
 * makespan over the SMs and is cached per (schedule, step, layer, batch size).  A launch of few and short items (at most one per
 * two SMs, 16 key tiles, of 64-wide heads 12) runs uncut on pairs of CTAs instead, so there the figures only say what that saves.
 * One whose items would leave SMs idle may also take query tiles of 128 one by one, with whole key
 * ranges, instead of in pairs (its own items are not counted here).  heatkv_last_attention has what a launch did.  Host only. */
int heatkv_attention_split(heatkv_ctx* ctx, const int* seq_ids /*HOST*/, int n_seq, int layer, int step,
                           int32_t* split_tiles, int32_t* items);

/* The search behind heatkv_attention_split, on its own (pure host code, needs no context and no GPU): given
 * the key tiles (128 keys each) of the heads of one launch in dispatch order (descending), the query tile
 * pairs per head (ceil(t_step / 256)), the sequences of the call and the SMs of the device, writes to
 * pieces[0..n_heads) into how many equal pieces every head's key range is cut (1 = whole head).  per_head = 0
 * restricts the choice to "no piece longer than some run", the rule a call that mixes schedules uses.
 * max_slots / max_ctrs bound the partial-result slots and arrival counters the cut may use (what the
 * context's scratch region holds).  The two optional outputs are the estimated makespans, in key tiles,
 * of the launch with whole heads and with the chosen cut.  Errors: INVALID_ARG for non-positive sizes or
 * tiles that are not sorted in descending order. */
int heatkv_split_plan(const int32_t* tiles /*HOST*/, int n_heads, int n_qp, int n_seq, int n_sm, int per_head,
                      uint64_t max_slots, uint64_t max_ctrs, int32_t* pieces /*HOST*/, double* makespan_whole,
                      double* makespan_cut);

/* The whole choice of such a launch: the search above, then whether query tiles one by one are quicker (pure host code as well).
 * t_q: the step's queries, d: the head dimension (64 or 128).  pieces[0..n_heads) as heatkv_split_plan; *lone = 1 when the launch cuts nothing and takes some query tiles
 * of 128 by themselves, 0 when the cut runs; singles[0..n_heads) = 1 for the heads whose query tiles all go one by one (0 for the
 * others: pairs of query tiles, and an odd last one by itself).  Errors: as heatkv_split_plan. */
int heatkv_lone_plan(const int32_t* tiles /*HOST*/, int n_heads, int t_q, int n_seq, int n_sm, int d, int per_head,
                     uint64_t max_slots, uint64_t max_ctrs, int32_t* pieces /*HOST*/, int32_t* singles /*HOST*/, int32_t* lone);

/* Introspection (host state only unless noted). */
/* (With the fp8 cache a row counts d + 1 bytes instead of 2 d in both figures.)
 * Bytes of K and V the sequence holds right now, two ways: *actual = the pool rows its plan has placed for the
 * head-scales it stores (valid rows of their destination half-tiles) x d x 2 (K and V) x 2 bytes; *closed_form =
 * sum over (layer, head) of kept_tokens x d x 2 x 2 from the schedule's masks (Sec. 3.2: the cache size in
 * tokens).  The two agree unless the plan and the schedule have come apart.  Either may be NULL. */
int heatkv_cache_bytes(heatkv_ctx* ctx, int seq_id, uint64_t* actual, uint64_t* closed_form);
/* The pool rows reserved for the sequence: first row and row count (x d x 2 x 2 bytes of K and V). */
int heatkv_seq_reservation(heatkv_ctx* ctx, int seq_id, uint64_t* first_row, uint64_t* rows);
/* Global token indices c_{i-1}+j of the tokens head (layer, head) holds now; idx HOST with
 * room for c_{K-1} entries. */
int heatkv_retained_indices(heatkv_ctx* ctx, int seq_id, int layer, int head, int32_t* idx, int* n);
/* Gathers the head's cached K and V rows in logical order into DEVICE buffers of
 * n*d bf16 each (enqueued on `stream`). */
int heatkv_export_head(heatkv_ctx* ctx, int seq_id, int layer, int head, void* k_out, void* v_out,
                       void* stream);
/* The same for a context with the fp8 cache (heatkv_export_head answers HEATKV_ERR_INVALID_ARG there, and this
 * call in a bf16 context): the head's n cached rows in logical order as stored, k_codes / v_codes DEVICE
 * uint8 [n][d] (E4M3 codes) and k_exps / v_exps DEVICE int8 [n] (the rows' exponent bytes). */
int heatkv_export_head_fp8(heatkv_ctx* ctx, int seq_id, int layer, int head, void* k_codes, void* v_codes,
                           void* k_exps, void* v_exps, void* stream);
int heatkv_allocator_stats(heatkv_ctx* ctx, heatkv_alloc_stats* out);
/* Kernels launched by this context so far. */
int heatkv_launch_count(heatkv_ctx* ctx, uint64_t* n);
/* The same per kernel, with the state of the tensor-memory kernels' set-up. */
int heatkv_kernel_launches(heatkv_ctx* ctx, heatkv_kernel_stats* out);
/* How many of the attention_tcgen05 launches ran uncut on pairs of CTAs (attn_pair_kernel; see heatkv_attention_split). */
int heatkv_pair_launches(heatkv_ctx* ctx, uint64_t* n);
/* How many of the attention_tcgen05 launches, and of the calibration_tcgen05 launches with an attention output, had work items of one
 * query tile of 128 instead of two (attn_tc_kernel, nothing cut).  None of them counts as a launch on pairs of CTAs. */
int heatkv_lone_launches(heatkv_ctx* ctx, uint64_t* n);
/* What the context's last attention call (heatkv_scale_attention, heatkv_attention_append) launched. */
int heatkv_last_attention(heatkv_ctx* ctx, heatkv_attention_form* out);
/* Appendix on S-CAS stability -- how much the head ordering moves between calibration sets.  scas_runs HOST
 * [n_runs][L][H][K]: S-CAS of n_runs independent calibration sets (heatkv_finalize_scores).  For every prunable
 * source scale k (s <= k <= K-2, 0-based) each run ranks the L*H heads by ascending S-CAS (ties by ascending
 * l*H+h, as heatkv_build_schedule does); out[k] = mean over heads of the standard deviation (population form)
 * of the head's rank position over the runs; 0 for the other k.  out HOST [K].  Pure host code.
 * HEATKV_ERR_NAN_SCORE if a score is not finite. */
int heatkv_rank_dispersion(const double* scas_runs, int n_runs, int L, int H, int K, int s, double* out);
/* Exercises the bounded wait every tensor-memory kernel uses for its hand-overs: a one-thread kernel waits,
 * with a short limit, on a barrier that nothing will ever signal.  Synchronises `stream`.  Returns
 * HEATKV_ERR_DEVICE_TIMEOUT when the wait gave up and set the device status word as designed (the expected
 * outcome; the context is then in the timed-out state described above and should be destroyed), HEATKV_OK if
 * the wait claimed success, HEATKV_ERR_CUDA on any other outcome.  Nothing faults, traps or hangs. */
int heatkv_selftest_wait_expiry(heatkv_ctx* ctx, void* stream);
/* Reads the device-side status word (synchronises `stream`): HEATKV_OK or
 * HEATKV_ERR_DEVICE_TIMEOUT if a bounded wait inside a kernel ran out. */
int heatkv_device_status(heatkv_ctx* ctx, void* stream);
const char* heatkv_strerror(int status);

/* ---------------------------------------------------------------------------------------------------------------------
 * Paged cache for requests of any length.  No counterpart in the paper: the cache above is planned for images, whose lengths are known
 * before they start; prompts, text that is answered token by token and drafted tokens are not.  Here a request's tokens lie in pages of
 * HEATKV_PAGE_TOKENS that its row of a block table lists, every head keeps every token, and G = n_heads / n_kv_heads query heads share a
 * kv head.  These calls need no context and keep nothing between them: all buffers are the caller's, lengths and tables stay on the
 * device, and no call waits for the device unless it says so.
 *
 * One step of a batch: heatkv_paged_tables (pages and slots of the new tokens), then per layer heatkv_paged_store (their K and V into the
 * layer's pool) and heatkv_paged_attention, or heatkv_paged_select and heatkv_paged_sparse_attention.  Requests' new tokens lie one
 * request after another in all token tensors: request i has the tokens q_begin[i] .. q_begin[i + 1] - 1, and the last of them is its token
 * number kv_len[i] - 1.
 *
 * Keys and values below kv_len must be finite; what the pool holds past them, and in pages that no table lists, may be anything, NaN
 * included.  Entries of tables and slot maps outside of the pool are not followed: nothing is stored there, and what is read is zero. */
typedef enum { HEATKV_DTYPE_BF16 = 0, HEATKV_DTYPE_FP16 = 1 } heatkv_dtype;

#define HEATKV_PAGED_MAX_SEQ 4096          /* requests of a call                                        */
#define HEATKV_PAGED_MAX_SELECT 32768      /* pages of a request from which heatkv_paged_select chooses */

typedef struct {                 /* one layer's pool                                                                   */
  void* k;                       /* DEVICE [n_pages][n_kv_heads][64][d], d contiguous, 16-byte aligned; strides below  */
  void* v;                       /* DEVICE, the same shape and strides                                                 */
  int8_t* k_code;                /* DEVICE [n_pages][n_kv_heads][d] page summaries, 16-byte aligned, or NULL: none kept */
  float* k_scale;                /* DEVICE [n_pages][n_kv_heads], or NULL with k_code                                  */
  int64_t page_stride, head_stride, row_stride;   /* elements, multiples of 8                                          */
  int32_t n_pages, n_kv_heads;
  int32_t d;                     /* 64 or 128                                                                          */
  int32_t dtype;                 /* heatkv_dtype of k, v and of the activations that go with them                      */
} heatkv_paged_pool;

typedef struct {                 /* the requests of a step                                                             */
  const int32_t* q_begin;        /* DEVICE [n_seq + 1] first new token of every request, and the last one's end; the first may be
                                    other than 0 (a part of a larger batch's requests: its pointers moved on, n_tokens as it was) */
  const int32_t* kv_len;         /* DEVICE [n_seq] tokens of the request, the new ones included; 0: none               */
  const int32_t* block_table;    /* DEVICE [n_seq][table_pages] page numbers, rows table_stride elements apart         */
  int64_t table_stride;
  int32_t n_seq, table_pages;
  int32_t n_tokens;              /* rows of the token tensors, at least q_begin[n_seq]                                 */
  int32_t max_new;               /* new tokens of the longest request: picks the kernel, with the other sizes; any value gives right results */
} heatkv_paged_batch;

typedef struct {                 /* element strides of [n_tokens][n_heads][d] activations: at least d, multiples of 8 */
  int64_t q_tok, q_head, o_tok, o_head;
} heatkv_token_strides;

/* Block tables and slot maps of a step, from its requests' lengths.  Request i takes need_i = ceil((past_i + new_i) / 64) -
 * ceil(past_i / 64) fresh pages for its new tokens; in request order they come from a ring of free pages.  A request is refused when
 * need_i > 0 and the pages wanted up to and including it exceed the free ones, or when it needs more than table_pages: it takes no
 * pages, its slots are -1 and its kv_len is 0 in this step (so its rows of the attention are zero).
 *   new_tokens, past_tokens DEVICE [n_seq] (negative counts as 0)
 *   free_pages DEVICE [n_pages] the ring; state DEVICE int32[4]: {place of its oldest entry, entries, 0, 0}
 *   state_out DEVICE int32[4]: {place and entries after the call, requests refused, new tokens of all requests}; another buffer than
 *             state, so that a step can be repeated
 *   block_table DEVICE, in and out: entries ceil(past_i / 64) .. are written for the fresh pages
 *   q_begin DEVICE [n_seq + 1], kv_len DEVICE [n_seq], slot_map DEVICE [n_tokens] (page * 64 + row, -1: none; also past the last token),
 *   positions DEVICE [n_tokens] (past_i + place among the new tokens) or NULL
 * What is written (state_out, block_table, q_begin, kv_len, slot_map, positions) shares no memory with the rest. */
int heatkv_paged_tables(const int32_t* new_tokens, const int32_t* past_tokens, int n_seq, const int32_t* free_pages, int n_pages,
                        const int32_t* state, int32_t* state_out, int32_t* block_table, int64_t table_stride, int table_pages,
                        int32_t* q_begin, int32_t* kv_len, int32_t* slot_map, int32_t* positions, int n_tokens, void* stream);

/* Gives back the pages that hold only tokens from keep_len[i] on (0: the request is over; less than kv_len[i]: drafted tokens were
 * turned down), request by request, to the end of the ring.  DEVICE pointers as above; state_out: {.., .., 0, pages given back}.  The
 * tables are left as they are: the caller's lengths say what of them counts. */
int heatkv_paged_release(const int32_t* kv_len, const int32_t* keep_len, int n_seq, const int32_t* block_table, int64_t table_stride,
                         int table_pages, int32_t* free_pages, int n_pages, const int32_t* state, int32_t* state_out, void* stream);

/* K and V rows of new tokens to their slots: k_new, v_new DEVICE [n_tokens][n_kv_heads][d], strides in elements (multiples of 8).
 * Tokens with a slot outside of the pool are left out; no slot may occur twice.  With page summaries kept, every page whose last row is
 * among the slots gets its own: the mean of its 64 keys in 32 bits (a tree sum: rows i and i + 32, then i and i + 16, and so on),
 * scale = max|mean| * (1 / 127), code = round-to-nearest-even(mean / scale).  A page's rows that come with this call must lie one after
 * another in k_new, as heatkv_paged_tables puts them. */
int heatkv_paged_store(const heatkv_paged_pool* pool /*HOST*/, const void* k_new, const void* v_new, int64_t tok_stride,
                       int64_t head_stride, const int32_t* slot_map, int n_tokens, void* stream);

/* Workspace of the two attention calls below on the current device, in bytes (DEVICE, 256-byte aligned).  It must be zero before its
 * first use and may then serve any number of calls that do not overlap on the GPU, of this batch or a smaller one (fewer requests and
 * tokens) with as many heads. */
int heatkv_paged_workspace_bytes(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, uint64_t* bytes);

/* Attention of every request's new tokens over its pages: out = softmax(sm_scale q K^T) V, with causal != 0 over the keys up to the
 * token's own position, else over all kv_len of the request (an image's scale, whose tokens see one another).  Sums and softmax
 * statistics in 32 bits, probabilities rounded to 16 before the product with V.
 *   q DEVICE [n_tokens][n_heads][d], out the same shape, not the same memory; strides NULL: packed.  sm_scale <= 0: 1 / sqrt(d)
 *   lse DEVICE fp32 [n_tokens][n_heads], the natural logarithm of the sum of exponentials, or NULL
 * A row that sees no key (kv_len 0, or shorter than the new tokens), or whose logits are all minus infinity, is zero, its lse minus
 * infinity.  NaN in a query row, or a logit of plus infinity, makes that row and its lse NaN, and no other row.  Rows in front of
 * q_begin[0] and past q_begin[n_seq] are left as they are.  n_heads / n_kv_heads at most 128. */
int heatkv_paged_attention(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                           const heatkv_token_strides* st, int causal, float sm_scale, void* out, float* lse, void* workspace,
                           uint64_t workspace_bytes, void* stream);

/* The pages that every query token attends to, per kv head: the first `sink` pages, the last `local` ones (local >= 1: the token's own
 * page is among them) and, up to n_select in all, those between whose summary scores highest against the query's: the sum of the
 * group's query heads in 32 bits, in head order, as 8-bit codes like a page's; score = (whole-number dot product of the codes) * the
 * page's scale, ties to the lower page.  sel DEVICE int32 [n_tokens][n_kv_heads][n_select]: page places in the request's table row,
 * ascending, -1 after the last (nothing but -1 for tokens that are no request's).  n_select >= sink + local.  Pages between must have
 * summaries (they are whole by then). */
int heatkv_paged_select(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                        const heatkv_token_strides* st, int sink, int local, int n_select, int32_t* sel, void* stream);

/* Causal attention of every new token over the pages that sel lists for it (distinct places in the request's table row; entries below 0,
 * past the token's own page or past the table count for nothing).  Other arguments and results as heatkv_paged_attention.
 * n_heads / n_kv_heads at most 64. */
int heatkv_paged_sparse_attention(const heatkv_paged_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                                  const heatkv_token_strides* st, const int32_t* sel, int n_select, float sm_scale, void* out,
                                  float* lse, void* workspace, uint64_t workspace_bytes, void* stream);

/* Reads the workspace's status word (synchronises `stream`): HEATKV_OK, or HEATKV_ERR_DEVICE_TIMEOUT if a bounded wait inside a kernel
 * ran out.  From the call whose wait ran out on, attention on this workspace leaves rows unwritten, although the calls return HEATKV_OK (they
 * do not wait for the device): results since the last look are not to be used, and the workspace must be zeroed again. */
int heatkv_paged_status(const void* workspace /*DEVICE*/, void* stream);

/* Exercises the bounded waits of the paged kernels as heatkv_selftest_wait_expiry does those of the others: one warp waits, with a short limit,
 * on a barrier that nothing will ever signal.  Synchronises `stream`.  workspace: at least 256 bytes, the status zero.
 * HEATKV_ERR_DEVICE_TIMEOUT when the waits gave up and set the status as designed (the expected outcome; the workspace must then be
 * zeroed again), HEATKV_OK if one claimed success, HEATKV_ERR_CUDA on any other outcome.  Nothing faults, traps or hangs. */
int heatkv_paged_selftest_wait_expiry(void* workspace /*DEVICE*/, void* stream);

/* ---- a cache in 4 bits
 * The same pages with K and V as 4-bit codes: a value is code * scale * 2^exp, whole codes from -7 to 7 kept as code + 8, one scale (an 8-bit e4m3
 * number, not negative) for sixteen neighbouring columns of a row, exp the pool's.  72 bytes a row and head for d = 128 instead of 256.  Every
 * such value with exp 0 is a bf16 and an fp16 number exactly.  scale = e4m3(max |x| 2^-exp * (1 / 7)), to nearest even, at most 448; code = x 2^-exp / scale
 * to the nearest whole number, ties to even, within -7 .. 7; all 0 where the scale is 0.  Rows that are stored must be finite.
 * A page of one head is one block of bytes: codes of K [64][d / 2], codes of V, scales of K [64][d / 16], scales of V.  In every four bytes (a word, lowest
 * byte first, columns c .. c + 7) bits 4 i .. 4 i + 3 hold column c + 2 i for i < 4 and column c + 2 (i - 4) + 1 for the others. */
typedef struct {                 /* one layer's pool                                                                       */
  void* blocks;                  /* DEVICE [n_pages][n_kv_heads][64 (d + d / 8)] bytes, 16-byte aligned; strides below     */
  int64_t page_stride, head_stride;               /* bytes, multiples of 16                                                */
  int32_t n_pages, n_kv_heads;
  int32_t d;                     /* 64 or 128                                                                              */
  int32_t dtype;                 /* heatkv_dtype of the activations that go with it                                        */
  int32_t k_exp, v_exp;          /* from -64 to 64                                                                         */
} heatkv_paged4_pool;

/* K and V rows of new tokens to their slots; arguments as heatkv_paged_store. */
int heatkv_paged4_store(const heatkv_paged4_pool* pool /*HOST*/, const void* k_new, const void* v_new, int64_t tok_stride, int64_t head_stride,
                        const int32_t* slot_map, int n_tokens, void* stream);

/* The reverse: rows of some slots as 16-bit numbers, to k_out, v_out DEVICE [n_tokens][n_kv_heads][d] (strides at least d, multiples of 8; not the
 * same memory).  Tokens with a slot outside of the pool get zeros; a slot may occur more than once. */
int heatkv_paged4_load(const heatkv_paged4_pool* pool /*HOST*/, const int32_t* slot_map, int n_tokens, void* k_out, void* v_out,
                       int64_t tok_stride, int64_t head_stride, void* stream);

/* heatkv_paged_workspace_bytes and heatkv_paged_attention for a cache in 4 bits: the same arguments and results; what the pool holds
 * past kv_len and in pages that no table lists may be any bytes.  sm_scale times 2^k_exp must lie between 1e-27 and 1e22.
 * heatkv_paged_status looks at this workspace, too. */
int heatkv_paged4_workspace_bytes(const heatkv_paged4_pool* pool, const heatkv_paged_batch* batch, int n_heads, uint64_t* bytes);
int heatkv_paged4_attention(const heatkv_paged4_pool* pool, const heatkv_paged_batch* batch, int n_heads, const void* q,
                            const heatkv_token_strides* st, int causal, float sm_scale, void* out, float* lse, void* workspace,
                            uint64_t workspace_bytes, void* stream);

/* ---- rows between steps
 * Requests may list the same page as long as it is full for all of them: a page that is not full, where the next token goes, is listed by one row
 * alone.  The two calls below keep it so.  They read the old lengths and table and write new ones (other buffers, so that a step can be
 * repeated; entries past a row's pages become -1), take pages from the ring's head where rows need fresh ones and append to its end, in page
 * order, those that the old table lists and the new one does not.  Neither touches K and V: the moves (from and to slots, -1: none) are for
 * heatkv_paged_move or heatkv_paged4_move on every layer's pool, before anything else writes to the pools.
 * heatkv_paged_release must not be used while rows share pages (it would give them back for all): heatkv_paged_fork does its work, too.
 *   lengths DEVICE [n_seq] tokens of every row; block_table, table_out DEVICE [n_seq][table_pages], rows table_stride and out_stride apart
 *   free_pages DEVICE [n_pages] in and out, state, state_out DEVICE int32[4] as in heatkv_paged_tables
 *   workspace DEVICE, heatkv_paged_rows_workspace_bytes, 16-byte aligned, zero before its first use; forks and compactions of any sizes that it is
 *   large enough for may take turns on it, none may overlap */
int heatkv_paged_rows_workspace_bytes(int n_seq, int table_pages, int n_pages, uint64_t* bytes);

/* Row i goes on as a copy of row parents[i] (its own number: as it is; none of 0 .. n_seq - 1: it is over) with its first keep_len[i] tokens at most
 * (negative counts as 0; keep_len NULL: all).  Whole pages are shared.  A page that is not full stays with one row: the lowest of those that go
 * on from themselves, else the lowest; every other row, and all of them where some row has all of the page, get a fresh page, in row order, and its
 * tokens' moves: entries 64 i .. of move_from and move_to, DEVICE [64 n_seq].  Where the free pages end, rows lose the tokens of that page: lengths_out
 * says how many they have.  state_out: {place and entries of the ring, rows that lost tokens, pages given back} */
int heatkv_paged_fork(const int32_t* parents, const int32_t* keep_len, const int32_t* lengths, int n_seq, const int32_t* block_table,
                      int64_t table_stride, int table_pages, int32_t* free_pages, int n_pages, const int32_t* state, int32_t* lengths_out,
                      int32_t* table_out, int64_t out_stride, int32_t* state_out, int32_t* move_from, int32_t* move_to, void* workspace,
                      uint64_t workspace_bytes, void* stream);

/* Token t of row i leaves the cache where stays[i][t] (DEVICE bytes, rows stays_stride apart, stays_width of each) is 0; tokens past the width stay.
 * (stays may be NULL where the width is 0.)
 * Pages before the first token that leaves stay as they are; the tokens behind move together into fresh pages, in order.  Rows take their fresh
 * pages in row order; from the first row on for which the free ones, or the n_moves entries of move_from and move_to, do not suffice, every
 * row that needs some is left as it is.  The moves lie one after another, row by row, token by token; -1 past the last.
 * state_out: {place and entries of the ring, rows left as they are, tokens moved}.  A row's K keep the positions that they were encoded
 * with, while the places that heatkv_paged_tables counts go on from the new length. */
int heatkv_paged_compact(const uint8_t* stays, int64_t stays_stride, int stays_width, const int32_t* lengths, int n_seq,
                         const int32_t* block_table, int64_t table_stride, int table_pages, int32_t* free_pages, int n_pages,
                         const int32_t* state, int32_t* lengths_out, int32_t* table_out, int64_t out_stride, int32_t* state_out,
                         int32_t* move_from, int32_t* move_to, int n_moves, void* workspace, uint64_t workspace_bytes, void* stream);

/* K and V of all heads from slot from[i] to slot to[i], DEVICE [n_moves]; nothing where either lies outside of the pool.  No slot may occur twice
 * in `to`, nor in both.  With page summaries kept, pages whose last row is among `to` get theirs. */
int heatkv_paged_move(const heatkv_paged_pool* pool /*HOST*/, const int32_t* from, const int32_t* to, int n_moves, void* stream);
int heatkv_paged4_move(const heatkv_paged4_pool* pool /*HOST*/, const int32_t* from, const int32_t* to, int n_moves, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HEATKV_H_ */
