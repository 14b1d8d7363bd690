/*
 * lazyev -- decode-time hot path of LazyEviction (arXiv 2506.15969) for AMD MI355X (gfx950).
 *
 * C ABI.  Every pointer is marked (host) or (device).  The library owns no device memory:
 * caches, statistics arrays and the workspace are allocated by the caller (for example as
 * torch tensors) and must stay valid until lazyev_destroy.  All calls enqueue work on the
 * stream given at init and return without waiting, except lazyev_stats and
 * lazyev_mri_histogram, which wait for it.
 * Calls on one context must come from one thread at a time.
 *
 * A "unit" is one (layer, sequence, KV head).  Each unit has its own cache of N entries
 * (N is the same for all units of a layer), its own recurrence statistics and its own
 * survivor set.  Notation of the paper: B budget, W observation window, alpha activation
 * threshold, t decode step (1-based), TS timestamp vector, MRI maximum recurrence interval.
 *
 * Layouts (row-major, C = lazyev_capacity(cfg) entries per unit):
 *   k_cache, v_cache   [n_layers][batch][n_kv_heads][C][head_dim]   fp32 or bf16
 *   ts, mri, pos       [n_layers][batch][n_kv_heads][C]             int32
 *   q, out             [batch][n_q_heads][head_dim]                 same dtype as the caches
 *   k_new, v_new       [batch][n_kv_heads][head_dim]
 *   p_out, p_override  [batch][n_q_heads][C]                        fp32
 * Query head h reads KV head h / (n_q_heads / n_kv_heads).
 */
#ifndef LAZYEV_H
#define LAZYEV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LAZYEV_OK          0
#define LAZYEV_EINVAL     -1   /* bad shape, null pointer, B <= W, step or layer out of order   */
#define LAZYEV_ECAPACITY  -2   /* decode_step on a full cache (a due eviction was skipped)        */
#define LAZYEV_EWORKSPACE -3   /* workspace missing or smaller than lazyev_workspace_size        */
#define LAZYEV_EHIP       -4   /* a HIP runtime call failed; lazyev_last_hip_error has the code  */
#define LAZYEV_ENOMEM     -5   /* host memory for the context or a read-back buffer ran out      */
#define LAZYEV_ESCRATCH   -6   /* lazyev_evict_static: the shape exceeds the library's static scratch */
#define LAZYEV_EEXCHANGE  -7   /* lazyev_stats: a block of an earlier decode call gave up waiting for
                                  another block's partial result; that call's outputs are invalid   */

#define LAZYEV_DTYPE_FP32  0
#define LAZYEV_DTYPE_BF16  1

#define LAZYEV_SCORE_H1    1   /* use the H1 term of Eq. 3 */
#define LAZYEV_SCORE_H2    2   /* use the H2 term of Eq. 3 */
/* With LAZYEV_SCORE_H2: use 1 - H2 (and 1 at MRI = 1, 0 at MRI = 0) in place of H2.  The H2 of
 * Sec. 4 item 2 as printed grows with MRI; the sentence introducing it and App. D describe a
 * term that falls with MRI.  Default is the printed formula; this bit selects the other reading. */
#define LAZYEV_SCORE_H2_DECREASING 16
/* Rank the candidates by the attention weight they received at the eviction's own step (largest
 * over the query group) instead of Eq. 3: the rule of the current-attention methods the paper
 * compares against (Sec. 2 (2); App. C "Baselines").  With window = 1 this is their per-step
 * greedy eviction, with a larger window the same rule behind an observation window.  Replaces
 * the H1 / H2 bits.  bf16, head_dim 128 only, and lazyev_evict must directly follow the
 * lazyev_decode_step of the same layer (the weights of older calls are gone). */
#define LAZYEV_SCORE_CURRENT_ATTENTION 32

/* Number of eviction candidates (cache entries outside the last W) per unit whose score keys
 * the selection kernel holds in LDS.  An eviction with more candidates (a prompt far beyond the
 * budget) ranks through the workspace instead: same result, slower selection. */
#define LAZYEV_LDS_CANDIDATES 8192

/* Largest number of bins of lazyev_mri_histogram. */
#define LAZYEV_MAX_HIST_BINS 8192

typedef struct lazyev_ctx lazyev_ctx;              /* opaque, host memory */

typedef struct {
  int32_t n_layers, batch, n_q_heads, n_kv_heads;  /* n_q_heads % n_kv_heads == 0, group <= 8 */
  int32_t head_dim;                                /* 64 or 128                                */
  int32_t budget, window, prompt_len;              /* B > W >= 1 (Sec. 4: B >> W); P >= 0      */
  float   alpha;                                   /* activation test is p >= alpha (Alg. 1)   */
  float   softmax_scale;                           /* 0 selects 1/sqrt(head_dim) (Eq. 4)       */
  int32_t dtype;                                   /* LAZYEV_DTYPE_*: storage of K, V, q, out  */
  int32_t score_flags;                             /* LAZYEV_SCORE_* bits (Table 4 ablation)   */
  void    *k_cache, *v_cache;                      /* (device) see layouts                     */
  int32_t *ts, *mri, *pos;                         /* (device) see layouts                     */
  void    *workspace;                              /* (device) scratch, 256-byte aligned       */
  size_t  workspace_bytes;
  void    *stream;                                 /* hipStream_t; NULL = the default stream   */
} lazyev_config;

typedef struct {
  int32_t  n_layers;            /* in: length of the arrays below                               */
  int32_t *len;                 /* (host, nullable) out: current N of each layer                 */
  int32_t *last_step;           /* (host, nullable) out: last decode step seen by each layer     */
  int64_t *n_evict_events;      /* (host, nullable) out: evictions that fired, per layer         */
  int64_t *n_evicted;           /* (host, nullable) out: entries removed per unit, summed over
                                   the layer's events (with per-sequence timing, where the due
                                   units of an event may differ: the largest per event)         */
  int64_t *n_activations;       /* (host, nullable) out: (entry, step) pairs with p >= alpha,
                                   summed over the layer's units                                */
  int64_t *n_rows_moved;        /* (host, nullable) out: surviving entries that an eviction moved
                                   to a lower slot, summed over the layer's units and events:
                                   each is one K row and one V row read and written             */
} lazyev_stats_t;

/* Entries of cache per unit: C = max(prompt_len, budget) + window.  0 if cfg is invalid. */
int32_t lazyev_capacity(const lazyev_config *cfg /*host*/);

/* Bytes of workspace the configuration needs (split partials, two buffers of per-entry logits,
 * gather lists, counters, records of partials).  0 if cfg is invalid. */
size_t lazyev_workspace_size(const lazyev_config *cfg /*host*/);

/* Creates a context.  The caller has already written the prompt's K/V rows to entries
 * 0..P-1 of every unit.  Enqueues: TS = 0, MRI = 0, pos = i for those entries (the state a
 * token has "as if last important when prefill ended"; the paper starts MRI at 0, Sec. 4),
 * and clears the counters.  N = P for every layer.
 * Errors: EINVAL, EWORKSPACE, EHIP, ENOMEM. */
int lazyev_init(const lazyev_config *cfg /*host*/, lazyev_ctx **out /*host*/);

/* Optional start state from the prompt (the paper starts its clock at the first generated
 * token and is silent on the prompt): runs the tracking loop of Alg. 1 and Eq. 1 over the
 * prompt's own causal attention in `layer`.  Prompt position i (0-based, P positions) is the
 * query of step i + 1 - P <= 0 over the keys 0..i; entry i is born with TS = i + 1 - P, MRI = 0
 * and is updated by every later position whose probability for it reaches alpha in any head of
 * its group, exactly as a decode step would.  Decoding continues at step 1; the activations are
 * added to the layer's count.  Replaces the TS = 0, MRI = 0 that lazyev_init gave the prompt
 * entries; call it after lazyev_init and before the layer's first decode step.
 * q_prompt (device): [batch][P][n_q_heads][head_dim], the prompt's queries in the cache's dtype.
 * p_out / p_override (device, nullable): [batch][n_q_heads][P][P] fp32, row = query position,
 *   column = key; only the lower triangle (key <= query) is written / read; meaning as in
 *   lazyev_decode_step.
 * Not with lazyev_admit / retire.
 * Errors: EINVAL (shape, order, null, P = 0), EHIP. */
int lazyev_prefill_track(lazyev_ctx *ctx, int32_t layer, const void *q_prompt /*device*/,
                         float *p_out /*device, nullable*/,
                         const float *p_override /*device, nullable*/);

/* The same for ONE sequence of a batch with per-sequence timing (lazyev_admit): the prompt of
 * slot `seq` (its prompt_len positions, rows already in the caches) is tracked on the slot's own
 * clock, position i as local step i + 1 - prompt_len.  Call it after lazyev_admit and before the
 * sequence's first decode step in `layer`.
 * q_prompt (device): [prompt_len][n_q_heads][head_dim]; p_out / p_override: [n_q_heads][P][P].
 * Errors: EINVAL (no per-sequence timing, empty slot or prompt, the sequence has decoded in the
 * layer, shape), EHIP. */
int lazyev_prefill_track_seq(lazyev_ctx *ctx, int32_t layer, int32_t seq, const void *q_prompt /*device*/,
                             float *p_out /*device, nullable*/,
                             const float *p_override /*device, nullable*/);

/* One decode step of one layer (Eq. 4; Alg. 1 tracking loop; Eq. 1):
 *   appends (k_new, v_new) as entry N with TS = t, MRI = 0, pos = P + t - 1;
 *   out[h] = softmax(scale * q[h] K^T) V over the N+1 entries of the head's unit;
 *   an entry is active if any query head of its group has probability >= alpha (fp32 compare);
 *   active entries get MRI = max(MRI, t - TS), then TS = t.
 * `out` and the appended K/V rows are complete when the call's work on the stream is.  The
 * single-launch attention kernel (see lazyev_set_variant) works out which entries were active
 * with the NEXT call on the context (any layer) and keeps that as one bit per entry; the updates
 * of ts / mri of a layer's calls are applied together, in the order of the calls, before
 * anything reads them: by lazyev_evict / lazyev_evict_all, lazyev_stats, lazyev_mri_histogram,
 * lazyev_admit / lazyev_retire, after at most min(W, 256) calls of the layer, and at once when
 * p_out or p_override is given.  A caller that reads ts / mri / pos itself calls lazyev_stats
 * first.
 * t must be the layer's previous step + 1 (first step is 1).
 * A call on a stream that is being captured into a HIP graph is recorded with the step, entry and
 * pointers it was made with, and the context goes on from there; every replay computes `out` and
 * the appended rows from what the pointers hold then.  ts / mri / pos follow the order of the
 * calls only if each captured call is replayed once, in its place: what a replay at another time
 * tracks, and what is tracked of the calls around it, is unspecified (but within the buffers).
 * p_out (device, nullable): receives the fp32 probabilities the threshold test used, entries
 *   [0, N+1) of each row.
 * p_override (device, nullable): probabilities to threshold INSTEAD of the computed ones (the
 *   attention output is unaffected); lets a checker feed identical weights to two
 *   implementations.
 * Errors: EINVAL (order, range, null), ECAPACITY (N == C), EHIP. */
int lazyev_decode_step(lazyev_ctx *ctx, int32_t layer, int32_t t,
                       const void *q /*device*/, const void *k_new /*device*/,
                       const void *v_new /*device*/, void *out /*device*/,
                       float *p_out /*device, nullable*/,
                       const float *p_override /*device, nullable*/);

/* Lagged eviction check after decode step t of a layer (Sec. 4; Eq. 3; Eq. 6; Alg. 1):
 * does nothing unless t % W == 0 and N > B.  Otherwise every unit scores entries 0..N-W-1
 * with I = H1 + H2 in binary64, keeps the B-W best (ties: the more recent entry wins) and
 * the last W, and moves K, V, TS, MRI, pos of the survivors to entries 0..B-1 in their
 * original order.  N becomes B.
 * n_evicted (host, nullable): entries removed per unit (N - B, or 0).
 * t must equal the layer's last decode step.
 * Errors: EINVAL, EHIP. */
int lazyev_evict(lazyev_ctx *ctx, int32_t layer, int32_t t, int32_t *n_evicted /*host*/);

/* lazyev_evict for callers that must not allocate and cannot hand over a scratch area of their
 * own for this call: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, same kernels and the same result as lazyev_evict; the one
 * difference is where the kernels' scratch buffer lives.  The selection kernel leaves a gather
 * list (source entry of every survivor, one int32 per cache entry of the layer's units) that the
 * row-move kernel then walks; lazyev_evict keeps it in the caller's workspace, this call keeps
 * it in a device array of LAZYEV_STATIC_SCRATCH_ENTRIES int32 (4 MiB) that is part of the
 * library image: every GPU the library runs on holds its own copy from load time until the
 * process ends.  The call allocates nothing, neither device nor host memory.
 * Limits: batch * n_kv_heads * capacity <= LAZYEV_STATIC_SCRATCH_ENTRIES and at most
 * LAZYEV_LDS_CANDIDATES candidates per unit (capacity - window); beyond them LAZYEV_ESCRATCH and
 * nothing is launched.  The device that was current at lazyev_init must be current (EINVAL).
 * All contexts of a process share one array per GPU and the array keeps the previous call's
 * list: nothing in it has to start at zero (a call overwrites every entry it later reads), but
 * two such calls whose kernels overlap on one GPU (different streams) race.  The per-layer
 * counters lazyev_stats reports stay in the caller's workspace.
 * Errors: those of lazyev_evict, ESCRATCH. */
#define LAZYEV_STATIC_SCRATCH_ENTRIES (1 << 20)
int lazyev_evict_static(lazyev_ctx *ctx, int32_t layer, int32_t t, int32_t *n_evicted /*host*/);

/* The same check (Sec. 4 "MRI-Centric Eviction"; Eq. 3; Eq. 6; the eviction branch of Alg. 1)
 * for EVERY layer after decode step t (every layer must have taken step t).  The paper states
 * Alg. 1 for one attention module; the modules of a model are independent of one another.
 * Where the layers stand at the same point, which is the normal course of a model, the
 * selection and the row move of all layers go in one launch each (the units of different
 * layers are independent); otherwise this is lazyev_evict layer by layer.  Results are those
 * of the per-layer calls.  n_evicted: entries removed per unit of a layer (the largest, if the
 * layers differ).  Errors: those of lazyev_evict. */
int lazyev_evict_all(lazyev_ctx *ctx, int32_t t, int32_t *n_evicted /*host*/);

/* The bookkeeping of Alg. 1 as the host sees it: cache length per layer (the saw-tooth of
 * Fig. 6: at most B + W entries, exactly B after an eviction, Sec. 4 / Eq. 6), evictions that
 * fired, entries removed, activations (entries with A_t[i] >= alpha, first loop of Alg. 1) and
 * rows the compaction moved.  Applies any tracking still pending, waits for the stream, then
 * fills the non-null arrays of *out.  The TS / MRI / pos arrays themselves belong to the caller,
 * who reads them directly after this call (there is no copy-out argument).
 * Errors: EINVAL, EHIP, ENOMEM; EEXCHANGE when a decode call since the last lazyev_stats could
 * not complete its exchange between blocks (not expected on a working GPU; reported once). */
int lazyev_stats(lazyev_ctx *ctx, lazyev_stats_t *out /*host*/);

/* Per-sequence timing, for a batch whose sequences do not start together (the paper decodes one
 * sequence at a time and says nothing about batches; what follows applies Alg. 1 to every
 * sequence on its own clock).  Until the first of these two calls every sequence has the
 * configuration's prompt_len and starts at step 1.
 *
 * lazyev_admit: batch slot `seq` is taken by a sequence whose prompt_len K/V rows the caller
 *   has written (or will have written, on the context's stream, before the sequence's first
 *   step) to entries 0..prompt_len-1 of the slot's units in every layer.  Its first decode step
 *   is the call with t = t0 + 1; every quantity of Alg. 1 then runs on the sequence's local
 *   step t - t0: TS, the W-step schedule, pos = prompt_len + local step - 1.  Enqueues the
 *   state of lazyev_init for the slot in every layer.  A slot that is already taken starts over.
 *   Needs prompt_len <= capacity - window and t0 >= every layer's last decode step.
 * lazyev_retire: the slot is empty from now on: its units take no part in later calls (their
 *   output rows are not written) until it is admitted again.
 *
 * With per-sequence timing in use: lazyev_decode_step skips sequences whose first step lies
 * ahead; lazyev_evict runs for the sequences whose local step is a multiple of W and whose cache
 * exceeds the budget (n_evicted: the largest number removed from one unit) and must be called
 * after every step at which that holds for some sequence (the next lazyev_decode_step of the
 * layer returns ECAPACITY otherwise); lazyev_stats reports the longest cache of each layer.
 * bf16, head_dim 128 and the default attention kernel only.
 * A caller that wants the prompt itself tracked (TS / MRI from the prompt's own attention, and
 * eviction while a prompt longer than the budget is read) admits the sequence with prompt_len 0
 * and feeds the prompt tokens as decode steps.
 * Both apply pending tracking first.  Errors: EINVAL, EHIP. */
int lazyev_admit(lazyev_ctx *ctx, int32_t seq, int32_t prompt_len, int32_t t0);
/* Entries a sequence holds before the append of its local step (>= 1) when every due eviction has
 * run: the closed form host and kernels share (a due eviction leaves exactly `budget` entries,
 * Sec. 4 / Eq. 6, so the length depends on nothing else).  Host only.  -1 for bad arguments. */
int32_t lazyev_cached_before_step(int32_t prompt_len, int32_t local_step, int32_t budget, int32_t window);
int lazyev_retire(lazyev_ctx *ctx, int32_t seq);

/* Distribution of the Maximum Recurrence Interval (Eq. 1) over the cached entries, the
 * statistic from which the observation window W is chosen offline (Sec. 3, Fig. 2(c); Sec. 4
 * "Observation Window": W = the MRI below which 80 % of the tokens fall; run it on a context
 * whose budget covers the whole generation so that no token has been evicted).
 * hist[m] = number of entries 0..N-1, over all units of `layer` (-1: of every layer), whose MRI
 * is m, for m < n_bins - 1; hist[n_bins - 1] counts MRI >= n_bins - 1.  hist[0] are the entries
 * never re-activated since they were appended.
 * Applies any tracking still pending and waits for the stream.
 * Errors: EINVAL (2 <= n_bins <= LAZYEV_MAX_HIST_BINS, layer range, null), EHIP, ENOMEM. */
int lazyev_mri_histogram(lazyev_ctx *ctx, int32_t layer, int32_t n_bins, int64_t *hist /*host*/);

/* Observation window from such a histogram (Sec. 4 "Observation Window": W is set to the MRI
 * below which 80 % of the tokens fall): over the entries that were re-activated at least once
 * (MRI >= 1; an entry with MRI = 0 never recurred), the smallest W with at least `quantile` of
 * them at MRI <= W.  *window = 0 if no entry was ever re-activated; an answer of n_bins - 1 means
 * the histogram was too short.  Host arithmetic only, no GPU work.
 * Errors: EINVAL (null, n_bins < 2, quantile outside (0, 1], a negative count). */
int lazyev_window_from_histogram(const int64_t *hist /*host*/, int32_t n_bins, double quantile,
                                 int32_t *window /*host*/);

/* Score of Eq. 3 for n (t - TS, MRI) pairs, on the device, with the same code the eviction
 * uses; result as binary64.  For checking the scoring arithmetic in isolation.
 * Errors: EINVAL, EHIP. */
int lazyev_score_pairs(const int32_t *delta_t /*device*/, const int32_t *mri /*device*/,
                       double *score /*device*/, int64_t n, int32_t score_flags,
                       void *stream);

/* ---- Rows around a decode step: norms and rotation, a cache in pages, attention over pages.  The calls of this
 * section keep no state: they need no context (but lazyev_decode_step_shared), enqueue on the stream they are given (which
 * belongs to the current device) and return without waiting.  Two calls may run at once, on any streams, if neither writes what
 * the other reads or writes (the workspace of lazyev_pages_attend included).  They can be captured into a HIP graph; a replay
 * works on what the pointers hold then, with the lengths of the captured call.  No alignment beyond the element's
 * is asked for (multiples of 16 bytes are faster) but for a cache's pages and the workspace. */

/* Heads of the tokens of a batch, head_dim elements each: element e of head h of token i of sequence s lies at
 * rows[s * seq_stride + i * token_stride + h * head_stride + e] (strides in elements, of any sign, so that a head
 * may be a view into a joint projection), its result at `to` by the to_ strides: any places, the entries of
 * a cache for instance, of which no two heads share one.  `to` may be `rows` with the same strides; an
 * overlap of any other kind gives unspecified rows.
 * weight (nullable): [head_dim] of the rows' type: the head is normed, x / sqrt(mean(x^2) + eps) * weight.  The squares are summed in
 * fp32: elements of up to 2^60 in size, and, where eps does not outweigh them, from 2^-60 on. */
typedef struct {
  const void *rows;             /* (device)                                                             */
  void       *to;               /* (device)                                                             */
  int64_t     seq_stride, token_stride, head_stride;
  int64_t     to_seq_stride, to_token_stride, to_head_stride;
  const void *weight;           /* (device, nullable)                                                   */
  int32_t     n_heads;
} lazyev_heads;

#define LAZYEV_ROPE_NONE   0    /* no rotation                                                          */
#define LAZYEV_ROPE_HALVES 1    /* elements j and j + dims / 2 are turned together, j < dims / 2        */
#define LAZYEV_ROPE_PAIRS  2    /* elements 2 j and 2 j + 1                                             */
/* The pair j of a token at position p is turned by the angle p * inv_freq[j]: (x, y) becomes (x cos - y sin, y cos + x sin).
 * The angle is worked out in binary64, so positions may be as far as they like.  Elements from dims on stay. */
typedef struct {
  int32_t      layout;          /* LAZYEV_ROPE_*                                                        */
  int32_t      dims;            /* a multiple of 16, at most head_dim (layout NONE: ignored)            */
  const float *inv_freq;        /* (device) [dims / 2] fp32 (layout NONE: ignored)                      */
  float        eps;             /* of the norms, >= 0                                                   */
} lazyev_rotation;

/* Norms of the query and key heads and the rotation by the token's position, in one pass: what lazyev_decode_step and
 * lazyev_prefill_track take their rows after.  Arithmetic in fp32, rounded once to the rows' type.
 * Token i of sequence s is at position start + positions[s * n_tokens + i], or start + i without `positions`.
 * q or k may be null (not both).  head_dim 64 or 128, dtype LAZYEV_DTYPE_*.  n_seqs or n_tokens 0: nothing to do; n_seqs * n_tokens
 * is at most 2^30, here and in lazyev_pages_append.
 * Errors: EINVAL, EHIP. */
int lazyev_norm_rope(int32_t n_seqs, int32_t n_tokens, int32_t head_dim, int32_t dtype,
                     const lazyev_heads *q /*host, nullable*/, const lazyev_heads *k /*host, nullable*/,
                     const lazyev_rotation *rotation /*host*/, const int32_t *positions /*device, nullable*/,
                     int32_t start, void *stream);

/* A cache in pages: entry i of table row s is place i % page_size of page table[s * table_stride + i / page_size],
 * for every KV head.  Rows of the table may share pages.  A page number outside 0 .. n_pages - 1 stands for no page: its
 * entries are not written and no token sees them.
 * The caches of a context are such a pool too, per layer: n_pages = batch pages of page_size = capacity entries, so the same
 * calls fill a sequence's prompt (table row {sequence}) and attend over it. */
typedef struct {
  int32_t n_kv_heads, head_dim, dtype;             /* head_dim 64 or 128                                */
  int32_t n_pages, page_size;                      /* page_size up to 2^20, 2^32 rows of all pages and heads */
  int32_t n_seqs, table_stride;                    /* rows of the table, entries from one to the next   */
  void    *k_pages, *v_pages;                      /* (device) [n_pages][n_kv_heads][page_size][head_dim], 16-byte aligned */
  const int32_t *table;                            /* (device) [n_seqs][table_stride]                   */
} lazyev_pages;

/* Writes the keys and values of n_tokens tokens of every table row to the row's entries start .. start + n_tokens - 1: the keys
 * normed (k->weight) and rotated on the way, by the position position0 + i of the i-th token, the values as they are
 * (v->weight null).  k and v describe the source only: their `to` members are ignored.
 * A page that several of the written entries lead to (one number twice in the table) holds unspecified parts of their rows.  The
 * sources do not overlap the written entries.
 * start + n_tokens <= table_stride * page_size.  Errors: EINVAL, EHIP. */
int lazyev_pages_append(const lazyev_pages *pages /*host*/, int32_t start, int32_t n_tokens,
                        const lazyev_heads *k /*host*/, const lazyev_heads *v /*host*/,
                        const lazyev_rotation *rotation /*host*/, int32_t position0, void *stream);

/* Attention of n_tokens tokens of every table row over the row's first `length` entries (Eq. 4 for many queries at once: the
 * entries are read once for the tokens that share them):
 *   out[s][i][h] = softmax(scale * q[s][i][h] K^T) V,  lse[s][i][h] = ln(sum of exp(scale * q[s][i][h] k))
 * over the entries below visible[s * n_tokens + i] (null: all; values beyond 0 .. length count as the nearest of the two).
 * A batch's decode step over its common prefix: one table row, every sequence's query a token of it.  A prompt after the
 * prefix: likewise.  A prompt over itself: visible = i + 1.
 * A token that sees nothing, or nothing but logits of -inf, gets zeros, and lse = -inf.  What a token does not see has no influence on it, whatever it holds.
 * joined_out, joined_lse (nullable, together): the output and lse of the same queries over other entries, for instance the
 *   sequences' own caches; out and lse are then those over both.  They may be `out` and `lse` themselves.  No other argument
 *   overlaps what the call writes (out is not q: EINVAL).
 * Values of up to 2^89 in size stay in the range of fp32 on the way; of larger ones sums may leave it as infinities.
 * scale 0 selects 1/sqrt(head_dim).  Sums, maxima and the output are fp32 until out is rounded to its type; for the product with V
 * weights of 128 x bf16 rows are rounded to bf16 (as in lazyev_decode_step), those of 64 x bf16 rows taken as two bf16 terms.  n_q_heads is any multiple of the pages' n_kv_heads up to 64 times;
 * n_tokens * n_q_heads / n_kv_heads is at most 65535 * 32, n_seqs * n_kv_heads 2^22, n_seqs * n_tokens * n_q_heads 2^30, length 2^30.
 * Workspace: lazyev_pages_attend_workspace bytes, 256-byte aligned, needing no initial contents (0 bytes: may be null).
 * Errors: EINVAL (length 0 .. table_stride * page_size among them), EWORKSPACE, EHIP. */
int lazyev_pages_attend(const lazyev_pages *pages /*host*/, int32_t length, int32_t n_tokens, int32_t n_q_heads,
                        const int32_t *visible /*device, nullable*/,
                        const void *q /*device, [n_seqs][n_tokens][n_q_heads][head_dim]*/,
                        const void *joined_out /*device, nullable, like q*/,
                        const float *joined_lse /*device, nullable, [n_seqs][n_tokens][n_q_heads]*/,
                        void *out /*device, like q*/, float *lse /*device, nullable*/, float scale,
                        void *workspace /*device*/, size_t workspace_bytes, void *stream);
/* Bytes for such a call; 0 also for arguments that the call refuses. */
size_t lazyev_pages_attend_workspace(const lazyev_pages *pages /*host*/, int32_t length, int32_t n_tokens,
                                     int32_t n_q_heads);

/* lazyev_decode_step of a batch whose sequences share a prefix: the same append and the same tracking, with attention over
 * the first prefix_len entries of the pages' one table row AND the sequences' own caches.  The softmax is over both: p of the
 * activation test (and p_out) is the weight that an own entry has beside the prefix.  The prefix takes no part in tracking and is
 * never evicted.  (lazyev_prefill_track knows no prefix: its weights are those of the prompt alone, so that after one it counts
 * more activations than the test beside the prefix would, unless p_override holds the weights.)  `out` is not q.  prefix_len 0 is lazyev_decode_step.  With per-sequence timing, sequences that take no part are left alone.
 * The pages' head_dim, dtype and n_kv_heads are the context's and n_seqs is 1; scale is the context's.  Own and prefix parts
 * are rounded to the rows' type once each.
 * workspace: lazyev_pages_attend_workspace(prefix, prefix_len, batch, n_q_heads) bytes, on the context's stream.
 * Errors: those of lazyev_decode_step, EWORKSPACE, EINVAL (a prefix that does not fit the context; the two-kernel attention
 * of lazyev_set_variant 0).  Nothing is enqueued on an error but EHIP. */
int lazyev_decode_step_shared(lazyev_ctx *ctx, int32_t layer, int32_t t, const void *q /*device*/,
                              const void *k_new /*device*/, const void *v_new /*device*/, void *out /*device*/,
                              const lazyev_pages *prefix /*host*/, int32_t prefix_len,
                              void *workspace /*device*/, size_t workspace_bytes,
                              float *p_out /*device, nullable*/, const float *p_override /*device, nullable*/);

/* ---- A long cache in pages: which of its blocks a token reads, and which of its entries stay.  The calls keep no state, as those of the section
 * above, of which the same holds (streams, graphs, calls at once, alignment, page numbers that stand for no page).
 *
 * Blocks.  Block b of a table row is its entries b * block .. b * block + block - 1, whatever pages they lie in.  Per KV head its bounds are
 * the smallest and the largest of each element of its keys. */
typedef struct {
  int32_t n_kv_heads, head_dim, dtype;             /* head_dim 64 or 128                                */
  int32_t n_seqs, n_blocks;                        /* blocks of a table row and KV head that `bounds` has room for */
  int32_t block;                                   /* entries of a block: 16, 32, 64 or 128             */
  void    *bounds;                                 /* (device) [n_seqs][n_kv_heads][n_blocks][2][head_dim] of the rows' type, 16-byte aligned */
} lazyev_blocks;

/* Bounds of the blocks that the entries start .. start + n_tokens - 1 of every table row lie in, over those entries; where `start` lies inside a block, that
 * block's bounds are extended, so that the same call after every append keeps all of them.  Other blocks are left alone.  (Entries that change otherwise, by
 * an eviction for instance, are counted in anew from their block's first one on.)  A NaN among a block's keys is in its bounds; entries of no page are
 * not counted: a block of nothing else has bounds of +inf and -inf.
 * Sizes agree between pages and blocks; start + n_tokens <= n_blocks * block and at most 2^30; n_seqs * n_kv_heads at most 2^22, and times the blocks that the entries lie
 * in 2^25.  Errors: EINVAL, EHIP. */
int lazyev_blocks_bound(const lazyev_pages *pages /*host*/, const lazyev_blocks *blocks /*host*/, int32_t start, int32_t n_tokens,
                        void *stream);

/* The blocks that tokens read, by a bound of what their logits can be: for a block, a token and a KV head
 *   score = max over the heads of the group of (sum of q[e] largest[e] where q[e] > 0, and of q[e] smallest[e] where q[e] < 0).
 * A token that sees v entries (visible as in lazyev_pages_attend) has ceil(v / block) blocks.  If these are more than n_chosen, it reads the first
 * n_first, the last n_last (of which one may be seen in part: it has no score) and those of the others with the highest scores,
 * of equal ones the lowest; otherwise all.  The ranks are those of the exact sums: in binary64, which the scores are worked out
 * in where a rounded one does not decide.  A sum that is no number counts as +inf: such a block is read rather than passed over.
 * Bounds are read of the blocks that some token ranks; what others hold has no influence (but may be read).
 * chosen (device): [n_seqs][n_tokens][n_kv_heads][n_chosen], ascending, -1 behind the last.
 * n_first >= 0, n_last >= 1, n_first + n_last <= n_chosen <= 2^20; length 0 .. n_blocks * block, at most 2^30; heads and tokens as in lazyev_pages_attend;
 * n_seqs * n_kv_heads * (length / block / 128 + 1) at most 2^22.
 * Workspace: lazyev_blocks_choose_workspace bytes, 256-byte aligned, needing no initial contents (0 bytes: may be null).
 * Errors: EINVAL, EWORKSPACE, EHIP. */
int lazyev_blocks_choose(const lazyev_blocks *blocks /*host*/, int32_t length, int32_t n_tokens, int32_t n_q_heads,
                         const int32_t *visible /*device, nullable*/, const void *q /*device, [n_seqs][n_tokens][n_q_heads][head_dim]*/,
                         int32_t n_first, int32_t n_last, int32_t n_chosen, int32_t *chosen /*device*/, void *workspace /*device*/,
                         size_t workspace_bytes, void *stream);
/* Bytes for such a call; 0 also for arguments that the call refuses. */
size_t lazyev_blocks_choose_workspace(const lazyev_blocks *blocks /*host*/, int32_t length, int32_t n_tokens, int32_t n_q_heads,
                                      int32_t n_last, int32_t n_chosen);

/* lazyev_pages_attend over the entries of listed blocks alone: for every token and KV head those of the blocks chosen[s][i][kvh][..] that the token
 * sees, visible and all else as there (a token that sees nothing of its blocks gets zeros and lse = -inf; what it does not see has no influence).  A number that is
 * no block of the row's first `length` entries, -1 for instance, stands for none; a number twice counts its entries twice.
 * Equal calls give equal bits; but lists of several tokens are gone over together, so that the order of a token's sums, and with it their roundings,
 * may depend on what else a call lists.
 * block: 16, 32, 64 or 128; n_chosen >= 1, n_chosen * block at most 2^30; a group of up to 64 heads; n_seqs * n_tokens * n_kv_heads at most 2^22.
 * Pools of up to 2^32 - 1 rows.  Errors: those of lazyev_pages_attend. */
int lazyev_blocks_attend(const lazyev_pages *pages /*host*/, int32_t length, int32_t block, int32_t n_chosen,
                         const int32_t *chosen /*device, [n_seqs][n_tokens][n_kv_heads][n_chosen]*/, int32_t n_tokens, int32_t n_q_heads,
                         const int32_t *visible /*device, nullable*/, const void *q /*device*/, const void *joined_out /*device, nullable*/,
                         const float *joined_lse /*device, nullable*/, void *out /*device*/, float *lse /*device, nullable*/, float scale,
                         void *workspace /*device*/, size_t workspace_bytes, void *stream);
size_t lazyev_blocks_attend_workspace(const lazyev_pages *pages /*host*/, int32_t length, int32_t block, int32_t n_chosen,
                                      int32_t n_tokens, int32_t n_q_heads);

/* The attention weight that every entry received, over the tokens that see it and the heads of its group:
 *   weights[s][kvh][e] = (e < known and decay is not 0 ? decay * old[s][kvh][e] : 0) + sum of exp(scale * q k - lse),  e < length
 * with the lse that lazyev_pages_attend gave these queries; one over more than the row's entries, a joined one, gives
 * the weights beside those.  An lse over chosen blocks alone (lazyev_blocks_attend) gives the weights beside those blocks: right for the entries that the token read; any other one
 * that it sees (but did not read) gets exp(its logit - lse) too, which nothing bounds (+inf is possible), and which a sum with decay 1 keeps.  Who evicts by weights
 * takes the lse over all entries.  Called for a prompt and then for every step, with decay 1, it keeps the sum of all weights; with decay 0 those of
 * the call alone.  A token whose lse is -inf adds nothing, nor does any token to an entry that it does not see or that lies in no page.
 * old, weights: fp32, `stride` elements from one KV head to the next (at least length), and n_kv_heads times that from one row to the next; weights may be
 * old (known 0: old may be null).  No other argument overlaps weights.  scale as in lazyev_pages_attend, decay finite.
 * Logits, weights and sums are fp32; the sums are taken in an order that depends on sizes alone.  length up to 2^30, n_seqs * n_kv_heads * (length / 128 + 1) below 2^24,
 * heads and tokens as in lazyev_pages_attend.
 * Workspace: lazyev_pages_weigh_workspace bytes, 256-byte aligned, needing no initial contents (0 bytes: may be null).  Errors: EINVAL, EWORKSPACE, EHIP. */
int lazyev_pages_weigh(const lazyev_pages *pages /*host*/, int32_t length, int32_t n_tokens, int32_t n_q_heads,
                       const int32_t *visible /*device, nullable*/, const void *q /*device*/,
                       const float *lse /*device, [n_seqs][n_tokens][n_q_heads]*/, float scale, const float *old /*device*/, int32_t known,
                       float decay, float *weights /*device*/, int64_t stride, void *workspace /*device*/, size_t workspace_bytes,
                       void *stream);
size_t lazyev_pages_weigh_workspace(const lazyev_pages *pages /*host*/, int32_t length, int32_t n_tokens, int32_t n_q_heads);

/* Eviction by weight: of the first n entries of every table row and KV head (n = lengths[s], values beyond 0 .. length counting as the nearest of the two; null:
 * length), `keep` stay if there are more: the newest, whose position is above the largest one - n_recent, the first, whose position is below n_first, and of the
 * others those of the largest weights, a NaN being the largest; equal ones (and, if there are more than `keep` of them, newest and first ones) in
 * the entries' order.  Positions are those of `positions`, null: the entries' own numbers.
 * Entries that stay below `keep` are left where they are; those from `keep` on go, in their order, to the places that became free, lowest first, with
 * their keys and values.  So no more rows are moved than entries go; the order of entries is not that of positions any more, which
 * attention does not ask for.  Entries from `keep` on are left as they are.
 * sources (device): [n_seqs][n_kv_heads][keep], the entry that each place holds now, -1 from n on.
 * weights, positions (device): `stride` elements from one KV head to the next (at least length; length 0: may be null).  weights_to, positions_to (device, nullable): weights and positions
 *   of the places, 0 and -1 from n on, `to_stride` elements from one KV head to the next (at least keep); they may be weights and positions with the same
 *   stride, and overlap nothing else.  Rows of entries of no page are not moved.
 * Not for the caches of a context while it goes on with them: their statistics and positions (and its number of entries) would stay as they are, beside other entries'
 *   keys and values.  lazyev_evict is that call.
 * Pages that are in the table more than once (a prefix that sequences share): rows are moved for all table rows and KV heads at once, in no order.  So no entry that
 *   one of them moves, from or to, may lie in such a page, or that place's keys and values are undefined afterwards, a mixture of several entries' even.  Shared entries that
 *   all stay where they are (the first ones, n_first of them or more) are safe; others are copied to pages of their own before.
 * keep >= 1, n_recent, n_first >= 0, n_recent + n_first <= keep; n_seqs * n_kv_heads below 2^22, n_seqs * n_kv_heads * (keep / 64 + 1) below 2^24; length up to 2^30.
 * Workspace: lazyev_pages_evict_workspace bytes, 256-byte aligned, needing no initial contents.  Errors: EINVAL, EWORKSPACE, EHIP. */
int lazyev_pages_evict(const lazyev_pages *pages /*host*/, int32_t length, const int32_t *lengths /*device, nullable*/, int32_t keep,
                       int32_t n_recent, int32_t n_first, const float *weights /*device*/, const int32_t *positions /*device, nullable*/,
                       int64_t stride, int32_t *sources /*device*/, float *weights_to /*device, nullable*/,
                       int32_t *positions_to /*device, nullable*/, int64_t to_stride, void *workspace /*device*/, size_t workspace_bytes,
                       void *stream);
size_t lazyev_pages_evict_workspace(const lazyev_pages *pages /*host*/, int32_t keep);

void lazyev_destroy(lazyev_ctx *ctx);              /* frees host memory only; NULL is allowed */
const char *lazyev_strerror(int code);
int lazyev_last_hip_error(const lazyev_ctx *ctx);  /* hipError_t of the last EHIP, else 0 */

#ifdef __cplusplus
}
#endif
#endif /* LAZYEV_H */
