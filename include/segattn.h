/*
 * segattn.h -- C ABI of libsegattn: segment-level causal attention for AMD MI355X (gfx950).
 *
 * The library implements the attention step of segmented execution (Sec. 3.1, Eq. 1: the
 * same forward operator F(x_i, C_{i-1}, R_{i-1}) at training and inference time) for one
 * attention layer:
 *
 *   - Eq. 12 (Appendix C): O = softmax(Q K^T * scale + M) V, where the mask M lets a
 *     segment query see every prefix row and the rows of its own segment up to itself;
 *   - Eq. 13 (Appendix C): the prefix a head sees -- the carried KV tail C_{i-1} (last T
 *     key/value rows of the previous segment; Sec. 3.4 "Local Continuity Channel"), the
 *     forward-only past KV (Sec. 3.4 "Long-Range Channel"), or nothing;
 *   - the cross-segment state itself: tail hand-off and append-only past pool
 *     (Sec. 3.4, Appendix D "Memory layout"; the paper applies no eviction, the evict call
 *     here is an extension).
 *
 * Conventions that hold for every entry point
 *   Pointers   Every q/k/v/out/lse/cache pointer is a DEVICE pointer unless the comment says
 *              "host".  All of them are borrowed for the duration of the enqueued work; the
 *              library never allocates or frees device memory.  The caller allocates one
 *              cache arena of segattn_cache_bytes() bytes (256-byte aligned) and keeps it
 *              alive until segattn_destroy().
 *   Streams    `stream` is a hipStream_t passed as void* (NULL = the default stream).  Work is
 *              only enqueued; no entry point synchronises with the device.  All calls on one
 *              context must be issued on one stream or be ordered by the caller.
 *   Layouts    Dense, token-major:  q, out [B, rows, Hq, D];  k, v [B, rows, Hkv, D];
 *              lse [B, Hq, rows].  q/k/v are bf16.  out is bf16, or fp32 when the
 *              configuration sets out_fp32 or fp32_check.  lse is fp32, the natural logarithm of
 *              sum_j exp(scale * q.k_j) over the visible keys.  Query head h reads KV head
 *              h / (Hq / Hkv).
 *   Errors     Every call validates its arguments and the context state before it enqueues
 *              anything and returns a segattn_status; nothing aborts or throws.  After EINVAL,
 *              ECAPACITY or ESTATE nothing was enqueued and the context is unchanged.  EHIP means
 *              the HIP runtime refused a launch or a copy, possibly after earlier kernels of the
 *              same call had entered the stream: the device counters of the cache may then be
 *              ahead of the context's bookkeeping, so the context is marked not ready and every
 *              stateful call returns ESTATE until segattn_reset() or seg_kv_set_lengths().
 *   Threads    A context is not thread-safe; distinct contexts are independent.
 */
#ifndef SEGATTN_H
#define SEGATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct segattn_ctx segattn_ctx; /* opaque; host-side bookkeeping only */

typedef enum {
  SEGATTN_OK = 0,
  SEGATTN_EINVAL = 1,    /* bad argument or unsupported configuration               */
  SEGATTN_ECAPACITY = 2, /* a PAST head would hold more than past_capacity rows      */
  SEGATTN_ESTATE = 3,    /* call not valid in the current cache state                */
  SEGATTN_EHIP = 4,      /* the HIP runtime reported an error on launch / copy       */
  SEGATTN_ESCRATCH = 5   /* the problem does not fit the library's built-in scratch   */
} segattn_status;

/* Per-KV-head access policy (Eq. 13), a bit mask.  SEG: own segment only (a long-range head
 * outside a long-range layer).  TAIL: plus the carried tail (a local head).  PAST: plus every
 * row the head's past pool holds (a long-range head in a long-range layer; here the whole
 * history rather than a retrieved top-k subset).  TAIL|PAST sees the union of positions. */
enum { SEGATTN_SEG = 0, SEGATTN_TAIL = 1, SEGATTN_PAST = 2 };

typedef struct {
  int32_t batch;           /* B >= 1                                                      */
  int32_t n_q_heads;       /* Hq, a multiple of n_kv_heads                                */
  int32_t n_kv_heads;      /* Hkv, 1..128                                                 */
  int32_t head_dim;        /* D, 64 or 128                                                */
  int32_t seg_len;         /* S >= 1: segments start at multiples of S (Sec. 3.5)         */
  int32_t tail_len;        /* T, 0 <= T <= S: rows of the carried tail (the paper's M)    */
  int64_t past_capacity;   /* rows a PAST head's pool can hold (history + open segment);
                              must be >= S when any head is PAST; < 2^31                  */
  const uint8_t *kv_policy;/* host, [Hkv] policy bit masks; copied                        */
  float scale;             /* score scale; 0 means 1/sqrt(D) (Eq. 12)                     */
  int32_t fp32_check;      /* 1: fp32 FMA arithmetic and fp32 `out` (validation mode)     */
  int32_t out_fp32;        /* 1: `out` is fp32 (the unrounded accumulator) also in bf16
                              MFMA mode; implied by fp32_check                            */
  int32_t retrieved_capacity; /* 0: a PAST head attends to its whole pool.  R_max > 0:
                              retrieval mode (Sec. 3.4 "Long-Range Channel"): a PAST head
                              attends to [retrieved prefix ; own segment] (Eq. 13, second case),
                              the prefix being the rows seg_kv_past_select() gathered, at most
                              R_max of them; no head may then have both TAIL and PAST       */
  float rope_theta;        /* 0: positions are not the library's business.  > 0: base of the
                              rotary embedding (Appendix E): seg_rope_apply() rotates by it, and
                              in retrieval mode the gathered K rows are re-rotated (see
                              seg_kv_past_select)                                              */
  /* Launch-shape overrides for tests and A/B timing; 0 everywhere = the library chooses.  Results
   * do not depend on them beyond rounding order. */
  int32_t prefill_waves;   /* 4 or 8: waves per workgroup of the head_dim-128 bf16 forward kernel
                              (a forced shape also keeps seg_attn_fwd from cutting prefixes, and
                              it as well as a forced queue mode every call from the forms for small
                              launches)                                                           */
  int32_t item_queues;     /* forward and dQ kernels as a resident grid that takes its work items
                              from per-XCD queues: 1 never, 2 whenever a launch has more than one
                              item, 3 the same with a grid a third of the items (so that small
                              inputs loop and take over items of other queues too)               */
} segattn_config;

/* ---- context --------------------------------------------------------------------------- */

/* Bytes of device memory the cache arena needs for this configuration (0 if invalid).
 * Per TAIL/SEG head: (T + S) rows of K and of V; per PAST head: past_capacity rows (in
 * retrieval mode also retrieved_capacity + S rows: retrieved prefix and a copy of the open
 * segment); plus per-(sequence, head) counters, the split-K workspace of the decode path and,
 * where one segment alone cannot fill the chip with the query blocks of its PAST heads (few
 * sequences, few PAST heads) and the pool can hold 2048 rows or more, at most 34 MB of workspace
 * in which seg_attn_fwd merges the pieces it cuts such a head's prefix into. */
size_t segattn_cache_bytes(const segattn_config *cfg);

/* Create a context over a caller-allocated arena (device, >= segattn_cache_bytes(), aligned
 * to 256 bytes).  The cache starts empty (C_0 = R_0 = empty) once segattn_reset() has been
 * enqueued; create itself touches no device memory.  EINVAL on a bad configuration. */
segattn_status segattn_create(const segattn_config *cfg, void *cache_dev, size_t cache_bytes,
                              segattn_ctx **out_ctx);
void segattn_destroy(segattn_ctx *ctx); /* frees host bookkeeping only, never the arena */

/* Empty the cache of every sequence: no tail, no past, no open segment. */
segattn_status segattn_reset(segattn_ctx *ctx, void *stream);

/* ---- prefill ---------------------------------------------------------------------------- */

/* Attention for the next m rows of the open segment of every sequence (Eq. 12 / Eq. 13).
 * q [B,m,Hq,D], k,v [B,m,Hkv,D]; out [B,m,Hq,D]; lse [B,Hq,m].  Row t of the call sits at
 * in-segment offset fill+t, where fill is the number of rows already committed to the open
 * segment; it sees the head's prefix held in the cache, those fill rows, and rows 0..t of k/v.
 * Requires 1 <= m and fill + m <= S for every sequence (ESTATE otherwise).  Reads the cache,
 * does not change it: follow with seg_kv_commit() on the same stream.
 * (All prefill entry points, head_dim 128: the library runs workgroups of eight or of four waves
 * depending on how much work the launch has; segattn_config.prefill_waves forces one of them.) */
segattn_status seg_attn_fwd(segattn_ctx *ctx, const void *q, const void *k, const void *v,
                            int32_t m, void *out, float *lse, void *stream);

/* Stateless whole-sequence form: one launch over all ceil(n/S) segments of q [B,n,Hq,D],
 * k,v [B,n,Hkv,D] by absolute position; only the last segment may be short.  Needs no
 * context and no cache: each segment's prefix is read from k/v directly (the tail is rows
 * [s-T, s) and the past rows [0, s) of a segment starting at s).  out [B,n,Hq,D] (bf16, or
 * fp32 if cfg->out_fp32 or cfg->fp32_check), lse [B,Hq,n].  cfg->past_capacity is ignored. */
segattn_status seg_attn_fwd_seq(const segattn_config *cfg, const void *q, const void *k,
                                const void *v, int64_t n, void *out, float *lse, void *stream);

/* Packed ragged batch (sequences of different lengths, no padding): q [total,Hq,D], k,v
 * [total,Hkv,D], out [total,Hq,D], lse [Hq,total]; sequence b = rows cu_seqlens[b] ..
 * cu_seqlens[b+1]-1 with its own segment grid (segments start at multiples of S inside the
 * sequence).  cu_seqlens: DEVICE int32 [cfg->batch + 1], ascending, cu_seqlens[0] = 0; total and
 * max_seqlen (the longest sequence, which sizes the launch) are host values.  An empty sequence
 * is allowed.  Otherwise as seg_attn_fwd_seq. */
segattn_status seg_attn_fwd_varlen(const segattn_config *cfg, const void *q, const void *k,
                                   const void *v, const int32_t *cu_seqlens, int64_t total,
                                   int64_t max_seqlen, void *out, float *lse, void *stream);

/* Policy array of one layer from the paper's head/layer sets (Sec. 3.4): KV heads in
 * long_heads are long-range heads, the others local (TAIL); a long-range head is PAST in a layer
 * of L_long and within-segment only (SEG) elsewhere.  Host only: long_heads [n_long] KV-head
 * indices, policy_out [n_kv_heads].  EINVAL on a bad index. */
segattn_status segattn_layer_policy(int32_t n_kv_heads, const int32_t *long_heads, int32_t n_long,
                                    int32_t layer_in_l_long, uint8_t *policy_out);

/* ---- positions --------------------------------------------------------------------------- */

/* RoPE re-indexing for prefix concatenation (Sec. 3.4, Appendix E).  Rotates q [B,rows,Hq,D] and
 * k [B,rows,Hkv,D] in place: row t of sequence b by the position pos0[b] + t, channel pair
 * (i, i + D/2) by position * theta^(-2i/D), theta = cfg->rope_theta (> 0).  pos0: device int64 [B]
 * or NULL (all zero).  Rotating every token by its absolute position before seg_attn_fwd* /
 * seg_kv_commit / seg_attn_decode reproduces the paper's re-indexed positions (prefix 0..P-1,
 * segment P..P+m-1) exactly for the carried tail and for a whole-history prefix, because RoPE
 * scores depend on position differences only; a retrieved prefix is turned to the positions
 * just before its segment by seg_kv_past_select.  Values are never rotated. */
segattn_status seg_rope_apply(const segattn_config *cfg, void *q, void *k, int64_t rows,
                              const int64_t *pos0, void *stream);

/* Rotary positions in the forms that models are trained with.  Pair i, i < rotary_dim / 2, of a head at
 * position p is turned by the angle p * f_i and multiplied by `magnitude`:
 *   (a, b) -> magnitude * (a cos - b sin, a sin + b cos).
 * Without scaling f_i = theta^(-2i / rotary_dim).  For contexts longer than the trained ones the frequencies
 * become f_i * (kept_i + (1 - kept_i) / factor) with
 *   LINEAR        kept_i = 0 (all positions divided by factor);
 *   BY_ROTATIONS  kept_i rises linearly from 0 to 1 while the rotations that pair i makes within trained_len
 *                 positions, trained_len * f_i / (2 pi), rise from `low` to `high`;
 *   BY_INDEX      kept_i falls linearly from 1 to 0 while the index i rises from that of the pair that makes
 *                 `high` rotations (rounded down, not below 0) to that of the one that makes `low` (rounded
 *                 up, not above rotary_dim - 1).
 * Frequencies are formed and angles reduced in double precision. */
enum { SEGATTN_ROPE_PLAIN = 0, SEGATTN_ROPE_LINEAR = 1, SEGATTN_ROPE_BY_ROTATIONS = 2, SEGATTN_ROPE_BY_INDEX = 3 };
typedef struct {
  double theta;          /* > 0 (BY_INDEX: not 1)                                                    */
  int32_t rotary_dim;    /* channels of a head that are turned, from the first on: a multiple of 16
                            up to D; 0 means D.  The others are passed on as they are                */
  int32_t interleaved;   /* 0: pair i is channels i and i + rotary_dim / 2; 1: channels 2i and 2i + 1 */
  int32_t scaling;       /* SEGATTN_ROPE_*                                                           */
  double factor;         /* > 0; not used by PLAIN                                                   */
  double trained_len;    /* > 0, low, high: BY_ROTATIONS and BY_INDEX only                           */
  double low, high;      /* 0 < low < high                                                           */
  double magnitude;      /* >= 0; 0 means 1                                                          */
  const double *inv_freq;/* host, [rotary_dim / 2] or NULL: the f_i themselves (copied); theta and
                            scaling are then not looked at                                           */
} segattn_rope;

/* Turns q [B*rows,Hq,D] and k [B*rows,Hkv,D] (B * rows < 2^31 - 4096) into q_out and k_out (either pair may be NULL).  An output may
 * be its own input (same pointer and stride: in place); apart from that its rows must not overlap an input's or the other
 * output's (EINVAL).  Row t of sequence b is at position pos0[b] + t (device int64 [B]; NULL: all 0), or row
 * j of all at pos[j] (device int64 [B*rows]: packed batches, caches that were evicted from; not both).  The
 * strides are in elements between token rows, 0 for dense, so that q and k can be parts of one projection's
 * output; heads are dense inside a row; rows and pointers on 16 bytes.  fp32 = 0: bf16, 1: float, in and out.
 * inverse = 1 turns by the negative angles (and multiplies by the magnitude all the same): applied to the gradients of
 * q_out and k_out it gives those of q and k, for bf16 and fp32 results of seg_attn_bwd_* alike.  cfg's rope_theta is not
 * used. */
segattn_status seg_rope_rotate(const segattn_config *cfg, const segattn_rope *rope, const void *q,
                               int64_t q_stride, const void *k, int64_t k_stride, int64_t rows,
                               const int64_t *pos0, const int64_t *pos, int32_t inverse, int32_t fp32,
                               void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride,
                               void *stream);

/* ---- backward (training) ---------------------------------------------------------------- */

/* Gradients of seg_attn_fwd_seq for truncated backpropagation over segments (Sec. 3.2,
 * Definition "K-truncated consistent objective"): given dout = dL/dout [B,n,Hq,D] (bf16) and
 * the forward's out and lse, writes dq [B,n,Hq,D] and dk, dv [B,n,Hkv,D] (bf16, or fp32 if
 * cfg->out_fp32 or cfg->fp32_check; `out` has that same type).  Every visible key contributes to
 * dq.  dk and dv collect the pairs inside a query's own segment and, for a head with the TAIL
 * bit, its carried tail -- the differentiable interface state; rows a query reaches only through
 * the PAST bit are forward-only and receive nothing (no-gradient lemma, Appendix B).  A window
 * of K+1 segments passed as one sequence is therefore exactly the graph truncation depth K
 * backpropagates through.  The g query heads of a group add up in dk, dv.  workspace: device,
 * at least seg_attn_bwd_workspace_bytes(cfg, n) bytes, 256-byte aligned, overwritten. */
size_t seg_attn_bwd_workspace_bytes(const segattn_config *cfg, int64_t n);
segattn_status seg_attn_bwd_seq(const segattn_config *cfg, const void *q, const void *k,
                                const void *v, const void *out, const float *lse,
                                const void *dout, int64_t n, void *dq, void *dk, void *dv,
                                void *workspace, size_t workspace_bytes, void *stream);

/* seg_attn_bwd_seq for callers that cannot allocate device memory or pass a workspace: code
 * under HIP graph capture, tight serving or training loops, harnesses that forbid hipMalloc.
 * Same arguments without the workspace, same kernels, same results bit for bit; the two [B,Hq,n]
 * fp32 row statistics that the backward kernels hand to each other live in an array inside the
 * library's device image instead (SEGATTN_BWD_STATIC_SCRATCH_BYTES per GPU, held from the moment
 * the library is loaded until the process ends).  The call allocates and frees nothing.
 * SEGATTN_ESCRATCH, before anything is enqueued, if the two statistics -- 2 * B * Hq * n * 4
 * bytes -- exceed the array (8 MiB: e.g. four 8192-token training windows of 32 query heads).  All calls on one GPU share that
 * GPU's array: calls whose kernels may overlap (different streams, several host threads) race on
 * it and must be ordered by the caller; the array keeps the last call's contents and nothing in
 * it needs clearing, since every call overwrites what it reads. */
#define SEGATTN_BWD_STATIC_SCRATCH_BYTES (8u << 20)
segattn_status seg_attn_bwd_seq_static(const segattn_config *cfg, const void *q, const void *k,
                                       const void *v, const void *out, const float *lse,
                                       const void *dout, int64_t n, void *dq, void *dk, void *dv,
                                       void *stream);

/* The same backward pass for a packed ragged batch (layout and cu_seqlens as for
 * seg_attn_fwd_varlen: q, out, dout, dq [total,Hq,D]; k, v, dk, dv [total,Hkv,D]; lse [Hq,total]);
 * every sequence is differentiated on its own, as one window of consecutive segments.
 * workspace: device, >= seg_attn_bwd_varlen_workspace_bytes(cfg, total), 256-byte aligned. */
size_t seg_attn_bwd_varlen_workspace_bytes(const segattn_config *cfg, int64_t total);
segattn_status seg_attn_bwd_varlen(const segattn_config *cfg, const void *q, const void *k,
                                   const void *v, const void *out, const float *lse,
                                   const void *dout, const int32_t *cu_seqlens, int64_t total,
                                   int64_t max_seqlen, void *dq, void *dk, void *dv,
                                   void *workspace, size_t workspace_bytes, void *stream);

/* ---- cache operations -------------------------------------------------------------------- */

/* Append m rows k,v [B,m,Hkv,D] to the open segment of every sequence.  When that makes the
 * segment complete (S rows) it is closed: the tail of every non-PAST head becomes the
 * segment's last T rows and the rest is dropped (this is what bounds memory, Sec. 3.5
 * "Memory Complexity"); a PAST head keeps all rows (append-only pool).  ESTATE if
 * fill + m > S for some sequence, ECAPACITY if a PAST pool would overflow. */
segattn_status seg_kv_commit(segattn_ctx *ctx, const void *k, const void *v, int32_t m,
                             void *stream);

/* The same for a whole prompt handed over at once: k,v [B,n,Hkv,D], every sequence's open segment
 * empty (ESTATE otherwise).  Leaves exactly the state that n/S calls of seg_kv_commit with S rows
 * and one with the remaining n%S rows would leave (pools of the PAST heads grown by the whole
 * segments, the tail of the last whole segment, the open rows), in two launches.  It is the
 * companion of seg_attn_fwd_seq: prefill in one launch, commit in one call, then decode.
 * ECAPACITY if a pool cannot take n more rows. */
segattn_status seg_kv_commit_seq(segattn_ctx *ctx, const void *k, const void *v, int64_t n,
                                 void *stream);

/* Append `rows` explicit rows k,v [B,rows,D] (e.g. rows gathered by a retrieval step,
 * Appendix D "Output") to the past pool of one PAST head, for every sequence.  Only valid
 * between segments (no open segment: ESTATE otherwise); EINVAL if the head is not PAST. */
segattn_status seg_kv_past_append(segattn_ctx *ctx, int32_t kv_head, const void *k,
                                  const void *v, int64_t rows, void *stream);

/* Retrieval mode only.  Retrieved prefix for the next segment (Appendix D "Output"): for every
 * sequence and every PAST head gather the R pool rows idx names into the head's retrieved
 * prefix.  idx: device int32 [B, n_past, R], n_past = the PAST heads in ascending KV-head
 * order; entries are pool row numbers (absolute positions, or the order of
 * seg_kv_past_append), distinct, each below the head's pool size and not evicted.  The
 * prefix rows take the order of the list (softmax does not depend on it).  The prefix serves
 * the segment that starts next (prefill calls and decode steps alike) and is dropped when
 * that segment closes; without a call the prefix is empty.  R = 0 empties it.  Valid between
 * segments only (ESTATE with an open segment); EINVAL if the context is not in retrieval
 * mode or R > retrieved_capacity; ECAPACITY if R exceeds the visible pool rows of some
 * sequence and head.  The lists are not read on the host: an out-of-range entry is clamped
 * into the pool (never an out-of-bounds access), a repeated entry counts twice.
 * With rope_theta > 0 the pool is taken to hold keys rotated by their absolute position (pool
 * row number = position, as seg_rope_apply + seg_kv_commit leave them) and list entry r is
 * re-rotated to position s - R + r, s the position at which the next segment starts: the
 * positions 0..R-1 / R..R+m-1 of Appendix E up to a common shift. */
segattn_status seg_kv_past_select(segattn_ctx *ctx, const int32_t *idx, int32_t R, void *stream);

/* Sizes of the top-k retrieval operator (Appendix D).  The paper names the steps and gives
 * L_q in [24, 64] and R = 512 (Appendix F); every other size is the caller's choice. */
typedef struct {
  int32_t n_queries;   /* L_q >= 1: the last L_q query rows of the previous segment are used     */
  int32_t pool_window; /* >= 1: sliding-window mean pooling, window = stride = this many rows     */
  int32_t tail_avg;    /* >= 1: one more summary, the mean of the last tail_avg rows              */
  int32_t n_anchors;   /* 1..32: rows with the highest scores                                      */
  int32_t win_before;  /* >= 0: an anchor a contributes rows a - win_before .. a + win_after       */
  int32_t win_after;   /* >= 0                                                                     */
} segattn_retrieval;

/* Bytes of device workspace seg_kv_retrieve needs for this context (0 if the sizes are invalid:
 * the summaries of one KV group, ceil(L_q / pool_window) + 1 per query head, must not exceed 64). */
size_t seg_kv_retrieve_workspace_bytes(const segattn_ctx *ctx, const segattn_retrieval *r);

/* Top-k retrieval operator (Appendix D): choose, for every sequence and every PAST head, the R
 * pool rows that form the retrieved prefix, and write them to idx_out (device int32
 * [B, n_past, R], ascending) in the form seg_kv_past_select takes.  q_prev: device bf16
 * [B, m, Hq, D], the queries of the previous segment (m >= 1).  Steps, as read here: query
 * summaries = means of consecutive pool_window-row windows of the last L_q rows plus the mean of
 * the last tail_avg rows, for every query head of the group, rounded to bf16; score of a pool
 * row = its best dot product with a summary over the visible pool (one bandwidth-bound pass over
 * the head's K rows); anchors = the n_anchors best rows (ties: lower row), which is what
 * per-summary top-k, de-duplication and anchor choice yield for any k >= n_anchors; anchors in
 * descending score order add their windows (clipped, rows already in skipped) until R rows are
 * in; the earliest visible rows pad to R.  ECAPACITY if some pool holds fewer than R visible
 * rows; EINVAL on bad sizes, a context without PAST heads, or a pool capacity above 2^20 rows.
 * workspace: device, >= seg_kv_retrieve_workspace_bytes(), 256-byte aligned, overwritten. */
segattn_status seg_kv_retrieve(segattn_ctx *ctx, const segattn_retrieval *r, const void *q_prev,
                               int32_t m, int32_t R, int32_t *idx_out, void *workspace,
                               size_t workspace_bytes, void *stream);

/* ---- retrieval mode for a whole prompt, stateless ------------------------------------------------
 * During prefill every segment's queries and every earlier key are present at once, so the
 * per-segment chain retrieve -> select -> attend -> commit (the calls above; they remain the form
 * for decoding) collapses into two calls with no context and no cache:
 *
 * seg_kv_retrieve_seq: the top-k retrieval operator (Appendix D, same reading and sizes as
 * seg_kv_retrieve) for every segment i >= 1 of q [B,n,Hq,D], k [B,n,Hkv,D] at once: the queries
 * are the last L_q rows of segment i-1, the pool of a PAST head is its keys [0, i S).  idx_out:
 * device int32 [B, n_seg, n_past, R], n_seg = ceil(n / S), PAST heads in ascending KV-head order;
 * the lists of segment 0 (no history) are not meaningful.  Requires 1 <= R <= S, at least one PAST
 * head and none with TAIL as well (Eq. 13), n <= 2^20; workspace: device, 256-byte aligned,
 * >= seg_kv_retrieve_seq_workspace_bytes() (0 if the sizes are invalid).
 *
 * seg_attn_fwd_seq_retrieved: seg_attn_fwd_seq in which a PAST head attends to [the R rows idx
 * names for its segment ; own segment] (Eq. 13, second case) instead of its whole history; the
 * first segment has no prefix.  idx as above (from seg_kv_retrieve_seq or the caller's own):
 * positions before the segment's start, distinct; an out-of-range entry is clamped into the
 * history, never read out of bounds.  The rows are first gathered into the workspace (device,
 * 256-byte aligned, >= seg_attn_fwd_seq_retrieved_workspace_bytes(): 2 R D bf16 per (sequence,
 * segment, PAST head)), with cfg->rope_theta > 0 re-rotated from their absolute positions to the
 * R positions just before the segment as seg_kv_past_select does; then one attention launch. */
size_t seg_kv_retrieve_seq_workspace_bytes(const segattn_config *cfg, const segattn_retrieval *r,
                                           int64_t n);
segattn_status seg_kv_retrieve_seq(const segattn_config *cfg, const segattn_retrieval *r,
                                   const void *q, const void *k, int64_t n, int32_t R,
                                   int32_t *idx_out, void *workspace, size_t workspace_bytes,
                                   void *stream);
size_t seg_attn_fwd_seq_retrieved_workspace_bytes(const segattn_config *cfg, int64_t n, int32_t R);
segattn_status seg_attn_fwd_seq_retrieved(const segattn_config *cfg, const void *q, const void *k,
                                          const void *v, int64_t n, const int32_t *idx, int32_t R,
                                          void *workspace, size_t workspace_bytes, void *out,
                                          float *lse, void *stream);

/* Hide the n_oldest oldest rows of one PAST head's pool from now on (all sequences).  Pure
 * bookkeeping: nothing is copied and the rows' storage is not reused.  If the head also has
 * the TAIL bit, rows inside the current tail window stay visible.  Evicting more rows than
 * the pool holds hides all of them. */
segattn_status seg_kv_past_evict(segattn_ctx *ctx, int32_t kv_head, int64_t n_oldest,
                                 void *stream);

/* Budget form of the same eviction (an extension: the paper's pool grows without eviction,
 * Sec. 3.4): per sequence, hide the oldest rows of the head's pool until at most max_rows
 * remain visible (a sequence holding fewer is left alone).  Called after each commit it keeps
 * a sliding budget of the most recent max_rows rows.  Rows of the current tail window of a
 * TAIL|PAST head stay visible even if max_rows is smaller. */
segattn_status seg_kv_past_keep_recent(segattn_ctx *ctx, int32_t kv_head, int64_t max_rows,
                                       void *stream);

/* Host copies of the cache counters (any pointer may be NULL): past [B,Hkv] = visible pool
 * rows of PAST heads (closed segments only; 0 for other heads), tail [B] = rows in the
 * carried tail, seg_fill [B] = rows in the open segment. */
segattn_status seg_kv_lengths(const segattn_ctx *ctx, int64_t *past, int32_t *tail,
                              int32_t *seg_fill);

/* Declare the cache contents after the caller has written K/V rows into the arena itself
 * (restore from a snapshot, benchmark set-up): host arrays closed_rows [B] = rows in closed
 * segments (a multiple of S), tail [B] (<= min(T, closed_rows)), seg_fill [B] (< S; 0 in
 * retrieval mode).  Row placement is given by segattn_cache_span().  The retrieved prefix
 * starts empty. */
segattn_status seg_kv_set_lengths(segattn_ctx *ctx, const int64_t *closed_rows,
                                  const int32_t *tail, const int32_t *seg_fill, void *stream);

/* Where the rows of (sequence b, KV head h) live inside the arena: K row r is the D bf16
 * values at byte offset *k_off + r*D*2, V likewise from *v_off; *cap_rows rows exist.
 * PAST head: row index = absolute position of the token (history, then the open segment).
 * Other heads: rows [T - tail, T) hold the tail, rows [T, T + seg_fill) the open segment. */
segattn_status segattn_cache_span(const segattn_ctx *ctx, int32_t b, int32_t kv_head,
                                  size_t *k_off, size_t *v_off, int64_t *cap_rows);

/* Bytes of K/V rows currently held (visible or not yet dropped) over all sequences and
 * heads: the quantity Sec. 3.5 bounds by S + T per local head plus the pool of PAST heads
 * (in retrieval mode plus the retrieved prefix and the segment mirror of those heads). */
size_t segattn_resident_bytes(const segattn_ctx *ctx);

/* ---- decode ----------------------------------------------------------------------------- */

/* One decoding step for every sequence (Eq. 2's conditioning on x_<t, C_{i-1}, R_{i-1}):
 * q [B,Hq,D], k_new,v_new [B,Hkv,D] belong to the newest token.  Appends the row to the open
 * segment, attends over [prefix | open segment] with a split-K kernel and a combine pass,
 * writes out [B,Hq,D] and lse [B,Hq], and closes the segment when it reaches S rows (same
 * rule as seg_kv_commit).  ECAPACITY if a PAST pool would overflow. */
segattn_status seg_attn_decode(segattn_ctx *ctx, const void *q, const void *k_new,
                               const void *v_new, void *out, float *lse, void *stream);

/* ---- paged cache -------------------------------------------------------------------------
 *
 * Keys and values in pages of a pool that the caller owns, for programs that serve many sequences from one
 * allocation.  No context: what a sequence holds is said by device arrays that the calls read and write in
 * stream order, so a captured step can be replayed while the cache grows.
 *   rows   int32 [B,Hkv]: rows that the (sequence, KV head) holds.  Row r of it is row r % page_rows of
 *          the page that entry r / page_rows of its table names.
 *   pages  page 0..n_pages-1 holds page_rows rows of every KV head, and table is int32 [B,max_pages]; or
 *          (per_head) page_rows rows of one head, and table is int32 [B,Hkv,max_pages].  An entry outside
 *          0..n_pages-1 names no page: rows there are not seen, not written and not moved.  A sequence's entries
 *          behind its last row need not be set, nor those of a head without the PAST bit before its window.
 * A head's policy keeps its meaning.  A head without the PAST bit sees the rows from max(0, s - T) on (TAIL)
 * or from s on (SEG), where s is the start of the segment of the newest row, so its row numbers have to be the
 * tokens' positions; a PAST head sees every row it holds (TAIL|PAST too), in any order.  The configuration's
 * validation mode, retrieval mode, past_capacity and rope_theta do not apply here (the first two: EINVAL).
 * Pages may be shared between sequences as long as nobody appends to, evicts from or accumulates weights of
 * them: those calls change the page for everyone who names it, in no fixed order.
 * The current device has to be the stream's and the pointers' (EINVAL for another device's stream).
 * Limits (EINVAL): B * Hkv < 2^24; rows of at most 2^26 bytes (row_stride), head_stride and page_stride below 2^40
 * elements, a pool below 4e18 bytes. */
enum { SEGATTN_PAGES_BF16 = 0, SEGATTN_PAGES_E4M3 = 1 };
typedef struct {
  void *k, *v;            /* device, 16-byte aligned: rows of D elements                             */
  int32_t type;           /* bf16, or e4m3 (4 significant bits, largest 448, NaN, no infinity)       */
  int32_t page_rows;      /* >= 1; multiples of 32 are fastest                                       */
  int32_t n_pages;        /* in the pool                                                             */
  int32_t max_pages;      /* entries of a table; max_pages * page_rows < 2^31 - 4096                 */
  int32_t per_head;       /* 1: a page holds the rows of one KV head                                 */
  int64_t page_stride;    /* of k and v, in elements, a multiple of 16 bytes: between pages,         */
  int64_t head_stride;    /* between the heads of a page (not used with per_head)                    */
  int64_t row_stride;     /* and between rows, >= D; all three 0: dense [n_pages][heads][page_rows][D] */
  uint8_t *k_scale, *v_scale; /* e4m3: device [n_pages][heads][page_rows], heads = 1 with per_head:
                             the row's elements times 2^(byte - 127), byte 1..254                     */
  float *mass;            /* device, same layout, or NULL: attention weight a row has received        */
  int32_t *pos;           /* device, same layout, or NULL: position of a row's token                  */
  const int32_t *table;   /* device                                                                  */
} segattn_pages;

/* Appends the tokens k,v [total,Hkv,D] (dense bf16): sequence b's are rows cu_seqlens[b] .. cu_seqlens[b+1]-1
 * (device int32 [B+1], ascending from 0; max_seqlen: the most of one sequence, total: all, host values), or NULL
 * for one token per sequence (total = B, max_seqlen = 1).  They become rows rows[b,h] on of every KV head, and
 * rows_out[b,h] = rows[b,h] + their number (rows_out may be rows).  Token i of a sequence is at position
 * pos0[b] + i (device int64 [B]; NULL: all 0; below 2^31), which pos gets and, with a rope, the key is turned by; q
 * [total,Hq,D] (NULL: none) is then turned into q_out (q itself, or apart from q, k and v).  Without a rope keys are taken as they are
 * (and q is not needed).  mass, where there is one, starts at 0.  e4m3: a row is stored with the smallest
 * power of two 2^e >= 2^-119 for which its largest finite magnitude is at most 448 * 2^e, every element rounded
 * once to nearest even; what is not finite becomes NaN, and what is rounded to 2^128 (from 1.9375 * 2^127 on), beyond bf16 and fp32
 * alike, is infinite to seg_attn_decode_paged.  bf16: turned keys are rounded once.  A row that has
 * no place (no page, or behind the table's last row) is dropped, and rows_out stops at the table's last row. */
segattn_status seg_kv_paged_append(const segattn_config *cfg, const segattn_pages *pages,
                                   const segattn_rope *rope, const void *q, const void *k, const void *v,
                                   const int32_t *cu_seqlens, int64_t total, int64_t max_seqlen,
                                   const int64_t *pos0, const int32_t *rows, void *q_out, int32_t *rows_out,
                                   void *stream);

/* One decoding step over a paged cache that already holds the newest token's rows (seg_kv_paged_append):
 * q [B,Hq,D] bf16; out [B,Hq,D] bf16 or fp32 (cfg->out_fp32); lse [B,Hq].  A query head that sees no row has
 * zeros and -infinity; one that sees a row of K or V with infinities or NaN may have NaN where the formula has an
 * infinity.  max_rows (host, <= max_pages * page_rows): the most rows of a head; it sizes the launch and the workspace, and of a head that holds more only the first max_rows are seen.  accumulate = 1: pages->mass
 * of every row of a PAST head grows by the weight that the row has for this token, summed over the query heads
 * of its group (at least one PAST head, max_rows times the heads of a group below 2^29 -
 * 2^12; EINVAL without mass).  At most 128 query heads per KV head, B * Hq < 2^30, and B * Hkv times (the 32-row tiles of max_rows,
 * plus one) below 2^31.
 * workspace: device, >= ..._workspace_bytes() (0: invalid arguments), 256-byte aligned, overwritten: calls that
 * may overlap need one each. */
size_t seg_attn_decode_paged_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages,
                                             int64_t max_rows, int32_t accumulate);
segattn_status seg_attn_decode_paged(const segattn_config *cfg, const segattn_pages *pages, const void *q,
                                     const int32_t *rows, int64_t max_rows, int32_t accumulate, void *out,
                                     float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* Eviction by accumulated attention weight, in place.  Of every PAST head that holds more than keep_rows rows
 * exactly keep_rows stay: those at the keep_recent newest positions (above the largest position held minus
 * keep_recent), those at positions below keep_first, and of the others the ones with the largest mass (a
 * negative or NaN mass counts as 0; among equals the lower row stays).  Rows that stay and lie at row keep_rows or behind
 * move, in order, into the rows below that became free, also in order, with their scales, mass and position; no
 * other row changes place.  rows_out[b,h] = min(rows[b,h], keep_rows) for a PAST head and rows[b,h] for the others
 * (rows_out may be rows); pages that hold no row any more are the caller's again.  keep_recent + keep_first <=
 * keep_rows.  pages->mass and pages->pos are required, and at least one PAST head.  max_rows as above: rows
 * behind it are not looked at, and none of a head where max_rows <= keep_rows.
 * Where the table has holes, a row without a page is not there: rows below keep_rows without one take a place each that
 * nothing can move to, so as many rows fewer stay (of the protected ones, where not even those have a place, the newest
 * positions first).  workspace as above. */
size_t seg_kv_paged_evict_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages,
                                          int64_t max_rows, int64_t keep_rows);
segattn_status seg_kv_paged_evict(const segattn_config *cfg, const segattn_pages *pages, const int32_t *rows,
                                  int64_t max_rows, int64_t keep_rows, int64_t keep_recent,
                                  int64_t keep_first, int32_t *rows_out, void *workspace,
                                  size_t workspace_bytes, void *stream);

/* ---- paged cache: tables kept on the device ------------------------------------------------
 *
 * users: device int32 [n_pages], how many table entries name a page; a page is free where that is 0 or less.  The two
 * calls below keep it for the tables that they change, of at most 2^31 - 4097 entries a sequence: a program that lets a second table name a page adds 1, and a
 * program whose tables name pages before its first call sets it.  pages->table is written (its entries behind a
 * sequence's last row have to be unnamed, say -1, where pages are wanted: a named one is taken to be reserved
 * already).  Both are in stream order and depend on nothing but their inputs. */

/* Pages for tokens that are going to be appended: m of sequence b, cu_seqlens, total and max_seqlen as for
 * seg_kv_paged_append (there may be fewer tokens than total: cu_seqlens[B] <= total; total may be 0 with cu_seqlens, and is
 * at most B * max_seqlen).  Head h wants the entries of rows rows[b,h] ..
 * rows[b,h] + m - 1, or (newest_only = 1) of those of them that the newest token sees under the head's policy.
 * Wanted entries that name no page are counted sequence by sequence (with per_head: head by head in it); a
 * sequence is granted its pages if it needs none, or if the free pages are enough for it and all sequences before it
 * together, and if its rows fit its table (a sequence whose rows do not fit counts as needing none).  The entries of granted sequences,
 * in order, get the free pages in ascending order, users of which become 1.  granted[b] (device int32 [B]): 1 or 0; a sequence
 * that is not granted changes nothing.  slots: device int64 [total,Hkv] or NULL: where the rows of a token will be in
 * arrays that hold one value per row of the pool (mass, pos, k_scale; rows of a dense pool): ((page * heads) + h) * page_rows + row in
 * page, h = 0 and heads = 1 with per_head; -1 where the table names no page and for sequences that were not granted.  Tokens from
 * cu_seqlens[B] on keep theirs.  workspace: device, >= ..._workspace_bytes() (0: invalid arguments), 256-byte aligned, overwritten. */
size_t seg_kv_paged_reserve_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages);
segattn_status seg_kv_paged_reserve(const segattn_config *cfg, const segattn_pages *pages, int32_t *users,
                                    const int32_t *cu_seqlens, int64_t total, int64_t max_seqlen,
                                    const int32_t *rows, int32_t newest_only, int32_t *granted, int64_t *slots,
                                    void *workspace, size_t workspace_bytes, void *stream);

/* Pages that no head needs any more, given back: an entry that names a page stays if it holds rows of a head (with
 * per_head: of its head) from the first one that its newest row sees (0 for a PAST head) up to rows[b,h] - 1; any
 * other becomes -1 and its page loses a user.  rows[b,h] = 0 ends a sequence.  Entries reserved for rows to come
 * are given back too: call it before reserving, or with the rows that the reservation was for. */
segattn_status seg_kv_paged_release(const segattn_config *cfg, const segattn_pages *pages, int32_t *users,
                                    const int32_t *rows, void *stream);

/* ---- paged cache: attention over chosen blocks ----------------------------------------------
 *
 * Long-range heads that read a few blocks of their history instead of all of it, chosen anew for every token: a block is
 * block_rows consecutive rows of a (sequence, KV head), and what it promises a query is bounded from the upper and
 * lower bounds of its keys in every channel.  Only PAST heads have blocks; the others keep their windows.  One token or many
 * per sequence: cu_seqlens, total and max_seqlen as for seg_kv_paged_append (cu_seqlens[B] <= total; what belongs to the
 * tokens from cu_seqlens[B] on is neither read nor written; total may be 0 with cu_seqlens, the arrays of tokens may then be NULL, and
 * is at most B * max_seqlen), and the tokens' rows have been appended: token i of
 * the m of sequence b is row r = rows[b,h] - m + i of head h, and sees no row behind its own.  max_rows (host, <= max_pages *
 * page_rows): the most rows of a head; it sizes launches and workspaces, and of a head that holds more only the first
 * max_rows are seen (a token whose row lies behind them is taken for the last of them, its window with it).  At most 128 query heads per
 * KV head; chunks with more than 16 are taken token by token.  A workspace whose size was asked for the largest total, max_seqlen,
 * max_rows, n_chosen and batch that a program uses serves its smaller calls too (with the same heads, types and blocks).  What a call
 * writes, its workspace among it, shares no byte with its other arrays (SEGATTN_EINVAL; of the pool's K and V the caller sees to that). */
typedef struct {
  int32_t block_rows;     /* a multiple of 16 that divides page_rows; 64 is a good size           */
  int8_t *bounds;         /* device, 16-byte aligned, [n_pages][heads][page_rows / block_rows][2][D]: upper, then lower
                             bounds of a block's keys; heads = 1 with per_head                      */
  uint8_t *scale;         /* device [n_pages][heads][page_rows / block_rows]: times 2^(byte - 127)    */
} segattn_blocks;

/* Bounds of the blocks that are complete (all their rows below rows[b,h]) and hold a row from rows_from[b,h] on (device int32
 * [B,Hkv]; NULL: 0), for every PAST head: after an append with what rows was before it, after an eviction
 * with NULL.  With e >= -80 the smallest exponent with |k| <= 127 * 2^e for all keys of the block, the bounds are the channels'
 * largest key / 2^e rounded up and smallest key / 2^e rounded down, and scale = e + 127.  Elements that are not finite in 32
 * bits count as 0.  max_new (host): the most rows of rows_from .. rows - 1 of a head; of a head with more only the first ones'
 * blocks are done (the first ceil(max_new / block_rows)).  Blocks in rows without a page are left out.  B * Hkv times ceil(max_new /
 * block_rows) below 2^40. */
segattn_status seg_kv_paged_summarize(const segattn_config *cfg, const segattn_pages *pages,
                                      const segattn_blocks *blocks, const int32_t *rows_from,
                                      const int32_t *rows, int64_t max_new, void *stream);

/* The n_chosen blocks (1 .. 4096) of every token and PAST head: chosen, device int32 [total,n_past,n_chosen], PAST heads in ascending
 * order, block numbers (row / block_rows) in ascending order, -1 behind the last.  Of the blocks 0 .. own (that of the token's
 * own row) all are taken if they are at most n_chosen; else the first keep_first, the last keep_recent (>= 1, so that no
 * bounds of a block are read that the token cannot see whole; keep_first + keep_recent <= n_chosen), and of the others those
 * with the highest scores, among equals the lower ones.  With the queries q [total,Hq,D] (bf16) of the KV head's group rounded to
 * q8 = q / 2^e, to nearest even, e the smallest exponent with |q| <= 127 * 2^e for all of them (elements that are not finite
 * count as 0), block j's score is
 *     2^(scale_j - 127) * max over the group of sum over channels of q8 * (q8 > 0 ? upper_j : lower_j),
 * formed and compared exactly for scales as seg_kv_paged_summarize writes them: an upper bound of the block's largest score but for the
 * rounding of q.  A block without a page has the lowest score.
 * workspace: device, >= ..._workspace_bytes() (0: invalid arguments), 256-byte aligned, overwritten: calls that may overlap need one each.  It
 * has 4 bytes for each token, PAST head and block of max_rows, but no more than 256 MiB or (where that is more) 16 tokens': more go in parts. */
size_t seg_kv_paged_choose_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages,
                                           const segattn_blocks *blocks, int64_t total, int64_t max_rows,
                                           int32_t n_chosen);
segattn_status seg_kv_paged_choose(const segattn_config *cfg, const segattn_pages *pages,
                                   const segattn_blocks *blocks, const void *q, const int32_t *cu_seqlens,
                                   int64_t total, int64_t max_seqlen, const int32_t *rows, int64_t max_rows,
                                   int32_t n_chosen, int32_t keep_first, int32_t keep_recent, int32_t *chosen,
                                   void *workspace, size_t workspace_bytes, void *stream);

/* Attention of the tokens q [total,Hq,D] (bf16): a query head of a PAST KV head sees the rows up to its token's own
 * in the n_chosen (1 .. 65536, n_chosen * block_rows < 2^31 - 4096) listed blocks (chosen as above or the caller's own, in any order: an entry below 0 or behind the
 * token's block is no block, one that is listed twice counts twice); of another KV head the rows of the token's
 * window, max(0, s - T) (TAIL) or s up to its own, s the start of its segment.  out [total,Hq,D] bf16 or fp32 (cfg->out_fp32), lse
 * [total,Hq]; rows without a page are not seen, and a query head that sees no row has zeros and -infinity; one that
 * sees a row of K or V with infinities or NaN may have NaN where the formula has an infinity, others are not touched by it.  Of
 * blocks only block_rows is looked at.  chosen may be NULL where no head has the PAST bit (n_chosen is then not looked at).
 * workspace as above: up to 2.25 GiB.  Of that 1 GiB is for chunks of which a listed block is taken once for all tokens that list it (more
 * tokens than it holds go in parts), 8 bytes for each block of their histories that max_rows leaves room for (1 GiB at most, beyond which
 * lists are taken token by token), 70 MB for windows. */
size_t seg_attn_paged_chosen_workspace_bytes(const segattn_config *cfg, const segattn_pages *pages,
                                             const segattn_blocks *blocks, int64_t total, int64_t max_seqlen,
                                             int64_t max_rows, int32_t n_chosen);
segattn_status seg_attn_paged_chosen(const segattn_config *cfg, const segattn_pages *pages,
                                     const segattn_blocks *blocks, const void *q, const int32_t *cu_seqlens,
                                     int64_t total, int64_t max_seqlen, const int32_t *rows, int64_t max_rows,
                                     const int32_t *chosen, int32_t n_chosen, void *out, float *lse,
                                     void *workspace, size_t workspace_bytes, void *stream);

/* ---- misc ------------------------------------------------------------------------------- */
/* Diagnostic for benchmarks: stream `bytes` of device memory at buf (16-byte aligned) with one of
 * the two access patterns of the library's HBM-bound kernels and nothing else.  mode 0: every
 * 16-byte piece read once, non-temporal (the decode and retrieval scans); sink: device, >= 4
 * bytes, practically never written.  mode 1: every piece read and written back in place with two
 * sign bits flipped (the in-place rotation of seg_rope_apply); two calls restore the buffer.
 * Timing it gives the rate the part sustains for the pattern. */
segattn_status segattn_bandwidth_probe(void *buf, size_t bytes, int32_t mode, void *sink, void *stream);

/* Diagnostic for benchmarks: the shader clock the part holds while other work runs.  Launches
 * SEGATTN_CLOCK_PROBE_WAVES single-wave workgroups (one per XCD) on `stream`; each sleeps until
 * `microseconds` (1 .. 10,000,000, else EINVAL) of the device's constant-rate wall clock have
 * passed, then stores two uint64 into counts (device, 2 x SEGATTN_CLOCK_PROBE_WAVES uint64,
 * 8-byte aligned): the shader clocks and the wall-clock ticks it saw.  *wall_clock_khz (host,
 * required) receives the wall clock's rate: clock [MHz] = clocks / ticks * wall_clock_khz / 1000.
 * Launch it on a stream of its own just before the work to be observed; it occupies one wave
 * slot with a handful of registers on eight compute units and ends by itself. */
#define SEGATTN_CLOCK_PROBE_WAVES 8
segattn_status segattn_clock_probe(uint32_t microseconds, uint64_t *counts, int32_t *wall_clock_khz, void *stream);

/* Diagnostic for benchmarks: the dense bf16 rate of the matrix pipes with nothing else busy.
 * Launches two 256-thread workgroups per compute unit on `stream`; every wave runs `iterations`
 * (1 .. 10,000,000, else EINVAL) rounds of eight independent 32x32x16 bf16 products from
 * registers, no memory access in the loop.  operands = 0: pseudo-random values in [-1, 1), a
 * different one in every lane and register (the switching activity of real data); 1: one constant
 * everywhere (almost no switching: the part draws less power and holds a higher clock).  *flops
 * (host, required) receives the floating-point operations of the launch; sink: device, >= 4
 * bytes, practically never written.  Timing the launch gives the rate; with segattn_clock_probe
 * beside it, the clock the part holds for it. */
segattn_status segattn_mfma_probe(int32_t iterations, int32_t operands, void *sink, int64_t *flops, void *stream);

const char *segattn_strerror(segattn_status st);
/* Name and average device time bookkeeping are not kept by the library; the version string
 * names the kernels' target ISA, e.g. "segattn 0.1 gfx950". */
const char *segattn_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SEGATTN_H */
