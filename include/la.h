/*
 * la.h -- C ABI of libla: block selection and block-sparse attention for
 * autoregressive (AR) chunk generation on AMD Instinct MI355X (gfx950).
 *
 * The operation is the block-sparse attention of Light Interaction (Sec. 3.3): a chunk of Lq query tokens (the frames being
 * denoised) attends to Lk keys laid out as
 *     [n_text text tokens][historical visual context][current chunk: last Lq keys].
 * Tokens are cut into 1-D blocks of `block` consecutive tokens.  Per (batch, head,
 * query block i) the library
 *   1. pools each query block and each historical key block into its mean
 *      (Sec. 3.3, pooling equation);
 *   2. scores s_{i,m} = q_bar_i . k_bar_m / sqrt(d) over the M historical blocks
 *      (Sec. 3.3, selection equation);
 *   3. keeps a subset S_i of the historical blocks: either the shortest
 *      highest-scoring prefix whose softmax mass over the M scores reaches tau
 *      (la_select_blocks), or the floor(r*M) highest scores, the paper's own
 *      Top-floor(rM) rule (la_select_blocks_topk);
 *   4. attends over C_i = text blocks u current-chunk blocks u S_i (Sec. 3.3,
 *      context-union equation), the same block set for K and V.
 *
 * Conventions shared by every call
 *   - Tensors are device pointers, contiguous, row-major, layout [B, H, L, d]
 *     for q, k, v and o; bf16 is raw IEEE bfloat16 (16-bit), 16-byte aligned.
 *   - The caller owns every buffer.  The library allocates no memory and keeps
 *     no state between calls; scratch space comes in through `ws`/`ws_bytes`
 *     (size from la_workspace_bytes; 256-byte alignment).
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = default stream) and the
 *     call returns without synchronising.  Outputs are ready when the stream is.
 *   - Arguments are validated before anything is enqueued: on any error the call
 *     returns a non-zero la_status and enqueues nothing, writes nothing.
 *     LA_ERR_HIP reports a failed kernel launch (outputs are then undefined).
 *   - No floating-point atomics: results are bit-reproducible run to run.
 *   - Calls are thread-safe (no global state).
 *   - The selection and attention calls enqueue kernel launches only (no memset,
 *     copy, allocation or synchronisation), so a caller may capture them in a
 *     HIP graph; replays give the same results as the calls.  Exceptions:
 *     la_sparse_attn_schedule (a reading tool) enqueues copies, and the first
 *     la_select_blocks_noalloc call on a device looks up its scratch address
 *     (make that call before capturing).
 */
#ifndef LA_H_
#define LA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum la_status {
  LA_OK = 0,
  LA_ERR_ARG = 1,        /* null pointer, tau <= 0 or NaN, bad r, misaligned pointer */
  LA_ERR_SHAPE = 2,      /* unsupported or inconsistent shape (see la_shape) */
  LA_ERR_WORKSPACE = 3,  /* ws too small or NULL while needed */
  LA_ERR_HIP = 4         /* a HIP launch failed */
} la_status;

/* Element types, where a call takes more than bf16. */
typedef enum la_dtype { LA_DTYPE_F32 = 0, LA_DTYPE_BF16 = 1 } la_dtype;

/* Problem shape.
 *   B, H        batch and heads (>= 1); every (b, h) is independent (Sec. 3.3:
 *               pooling and selection run per attention head).
 *   Lq, Lk      query tokens and key tokens, 1 <= Lq <= Lk - n_text.
 *   d           head dimension: 64 or 128.
 *   block       tokens per block, the same tiling for queries and keys: 64 or 128.
 *               NQ = ceil(Lq/block) query blocks, NK = ceil(Lk/block) key blocks.
 *   n_text      leading text-condition keys, always kept (the paper's T).
 *   frame_tokens  0: every kept key is visible to every query.  F > 0: frame-causal
 *               inside the chunk, query token t (chunk position) sees chunk key
 *               n (n >= Lk - Lq) only if (n - (Lk - Lq)) / F <= t / F; context keys
 *               stay visible.  Used by the attention calls only.
 * Key block m is forced (always kept, never scored) when it overlaps the text
 * tokens [0, n_text) or the chunk [Lk - Lq, Lk); the others are the M historical
 * candidates, block indices [ceil(n_text/block), floor((Lk-Lq)/block)).
 * Limits: NK <= 16384, M <= 4096, B*H <= 65535, and B*H*ceil(Lq/256)*NK*(block/64)
 * < 2^31 (the 64-key tiles of the attention work plan have 32-bit indices). */
typedef struct la_shape {
  int32_t B, H, Lq, Lk, d;
  int32_t block;
  int32_t n_text;
  int32_t frame_tokens;
} la_shape;

/* Bytes of scratch space the selection and attention calls need for this shape
 * (the maximum over them; the attention pass keeps its work plan and the partial
 * results of work split across workgroups there).  One ws may serve all calls in
 * stream order; a selection call overwrites an attention plan held in the same ws.
 * Returns 0 for an invalid shape. */
size_t la_workspace_bytes(const la_shape* shape);

/* Cumulative-mass block selection.
 *   q      bf16 [B, H, Lq, d];  k  bf16 [B, H, Lk, d]      (inputs)
 *   tau    in (0, +inf): per query block keep the shortest prefix of historical
 *          blocks, ordered by score descending (lower block index first on equal
 *          scores), whose softmax mass (softmax over the M scores) is >= tau.
 *          tau >= 1 keeps every historical block.
 *   mask   uint8 [B, H, NQ, NK] or NULL: 1 = key block kept, 0 = skipped.
 *   counts int32 [B, H, NQ]: number of kept key blocks per query block.
 *   idx    int32 [B, H, NQ, NK]: per query block, the kept key-block indices in
 *          ascending order in the first counts[] slots; later slots untouched.
 * Returns LA_ERR_ARG for tau <= 0 or NaN. */
la_status la_select_blocks(const la_shape* shape, const void* q, const void* k, float tau,
                           uint8_t* mask, int32_t* counts, int32_t* idx,
                           void* ws, size_t ws_bytes, void* stream);

/* la_select_blocks with no workspace argument, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  The scratch it needs (pooled queries and the score matrix,
 * la_workspace_bytes' selection part) is a device array of LA_NOALLOC_SCRATCH_BYTES
 * inside the library, one per GPU, held from the library's load until the process ends;
 * the call itself allocates nothing.
 *   Arguments, rule, outputs and errors as la_select_blocks; shapes whose selection
 *   scratch exceeds LA_NOALLOC_SCRATCH_BYTES (4 B * B*H*NQ*(d + M), rounded up to 256 B per
 *   part) return LA_ERR_WORKSPACE.  Every benchmark shape fits (at most 10.6 MB).
 *   The scratch belongs to the current device (hipGetDevice), which must be the device
 *   of q, k and the stream.  All calls on one GPU share it: calls that may overlap on one
 *   GPU (concurrent streams, or threads enqueueing at once) race; calls ordered on one
 *   stream do not.  Nothing carries over between calls (each call writes every scratch
 *   byte it reads). */
#define LA_NOALLOC_SCRATCH_BYTES (16u << 20)
la_status la_select_blocks_noalloc(const la_shape* shape, const void* q, const void* k, float tau,
                                   uint8_t* mask, int32_t* counts, int32_t* idx, void* stream);

/* The paper's Top-floor(rM) rule (Sec. 3.3, selection equation): keep the
 * keep_blocks = floor(r*M) highest-scoring historical blocks, computed by the
 * caller and clamped to [0, M] here (0 keeps only the forced blocks).  Same
 * outputs as la_select_blocks.  keep_blocks < 0 is LA_ERR_ARG. */
la_status la_select_blocks_topk(const la_shape* shape, const void* q, const void* k,
                                int32_t keep_blocks, uint8_t* mask, int32_t* counts,
                                int32_t* idx, void* ws, size_t ws_bytes, void* stream);

/* Block-sparse attention forward over the kept blocks.
 *   q bf16 [B, H, Lq, d]; k, v bf16 [B, H, Lk, d]                 (inputs)
 *   counts int32 [B, H, NQ], idx int32 [B, H, NQ, NK]: kept key blocks per query
 *          block in the first counts[] slots (as written by la_select_blocks or
 *          la_mask_to_list).  The set of listed blocks is used: order and repeats
 *          do not matter, entries outside [0, NK) are ignored and counts[] is
 *          clamped to [0, NK].  One list serves both K and V (Sec. 3.3).
 *   scale  logit scale; <= 0 selects 1/sqrt(d).
 *   o      bf16 [B, H, Lq, d]: o_t = sum_n softmax_n(q_t . k_n * scale) v_n over
 *          the keys of the kept blocks visible to t; 0 when none is.
 *   lse    float [B, H, Lq] or NULL: natural-log sum of exp(logits) per query
 *          token, -inf when no key is visible.
 * Softmax in fp32, products in bf16 with fp32 accumulation. */
la_status la_sparse_attn_fwd(const la_shape* shape, const void* q, const void* k, const void* v,
                             const int32_t* counts, const int32_t* idx, float scale,
                             void* o, float* lse, void* ws, size_t ws_bytes, void* stream);

/* la_sparse_attn_fwd in its three steps, for callers that time or reuse them.
 * The work plan depends only on the lists: units of 256 query rows (query blocks of a
 * head grouped by the first historical entry of their lists, the first kept historical
 * block for the ascending lists the selection writes, in frame-causal calls behind their
 * frame where that leaves fewer tiles; any order gives the same results),
 * the union of their lists as
 * 64-key tiles, and the split of the work over one persistent workgroup per CU of the
 * current device: whole units in rounds (the workgroups of one XCD start consecutive
 * units of a head together), the remaining and the longest units in equal-work shares
 * cut anywhere.  It lives in ws and is for the device it was built on.
 *
 * la_sparse_attn_plan: builds the plan for `shape` from counts/idx (read as in
 *   la_sparse_attn_fwd) into ws.
 * la_sparse_attn_run: the attention pass over the plan in ws (built by
 *   la_sparse_attn_plan for the same shape; it may be run for several q, k, v that
 *   share the lists).  Writes o and lse for the query rows of units processed whole by
 *   one workgroup, and partial results (O, running max, sum) into ws for the others.
 * la_sparse_attn_merge: merges those partials into o and lse (the buffers given to the
 *   run; lse may be NULL if it was NULL there).
 * Plan, run and merge must follow each other on one stream with the same ws, with no other
 * call using that ws in between (a selection call overwrites the plan): a run on a plan the
 * workspace no longer holds writes wrong values, though every access stays inside q, k, v, o,
 * lse and ws.  Arguments, alignment and errors as for la_sparse_attn_fwd. */
la_status la_sparse_attn_plan(const la_shape* shape, const int32_t* counts, const int32_t* idx,
                              void* ws, size_t ws_bytes, void* stream);
la_status la_sparse_attn_run(const la_shape* shape, const void* q, const void* k, const void* v,
                             float scale, void* o, float* lse, void* ws, size_t ws_bytes,
                             void* stream);
la_status la_sparse_attn_merge(const la_shape* shape, void* o, float* lse, void* ws,
                               size_t ws_bytes, void* stream);

/* The schedule of the plan in ws, for tools and tests that check or study it; it changes
 * nothing.  Units u < U = B H ceil(Lq / 256) own T tiles in all, ordered in one tile
 * sequence; the run's P persistent workgroups (one per CU of the current device, a multiple
 * of 8, at most 256) each take a range of whole units and a share cut anywhere.  Written:
 *   *P, *U    (host)  the two counts the arrays below are sized by;
 *   tstart    int32 [U + 1] (device): position of unit u's first tile; tstart[U] = T;
 *   ucount    int32 [U]     (device): 64-key tiles of unit u's list union that some row of it
 *             sees (a unit with 0 still runs one tile, so it takes max(1, ucount[u]) positions);
 *   dp_start  int32 [P + 1] (device): workgroup l runs the whole units on [dp_start[l],
 *             dp_start[l + 1]) (rounds: its XCD's consecutive units);
 *   sk_start  int32 [P + 1] (device): and its share [sk_start[l], sk_start[l + 1]) of the
 *             remaining tiles, which starts at dp_start[P].
 * Any of the four arrays may be NULL (not copied); the copies run on `stream`.  The values
 * describe the plan la_sparse_attn_plan(_valid) built for `shape` on this device, as long as
 * no other call has used ws since; otherwise they are meaningless.  LA_ERR_ARG if P or U is
 * NULL; workspace errors as for la_sparse_attn_run. */
la_status la_sparse_attn_schedule(const la_shape* shape, const void* ws, size_t ws_bytes,
                                  int32_t* P, int32_t* U, int32_t* tstart, int32_t* ucount,
                                  int32_t* dp_start, int32_t* sk_start, void* stream);

/* Compacts a block mask (uint8 [B, H, NQ, NK], non-zero = kept) into the
 * counts/idx form la_sparse_attn_fwd reads.  Needs no workspace. */
la_status la_mask_to_list(const la_shape* shape, const uint8_t* mask, int32_t* counts,
                          int32_t* idx, void* stream);

/* ------------------------------------------------------------------------------
 * 3-D block layout (Sec. 3.3: visual tokens in non-overlapping (B_t, B_h, B_w)
 * blocks; the fused Q-Prep, KV-Prep and Untile Scatter of its operator fusion).
 *
 * Linear (AR) order: keys are [n_text text tokens][T_ctx context frames][T_q chunk
 * frames], queries are the T_q chunk frames; a frame is Hs x Ws tokens in raster
 * order, token (t, y, x) of a run of frames at (t Hs + y) Ws + x.
 * Blocks: the text in 1-D blocks of `block` tokens; each run of frames (context,
 * chunk) in 3-D blocks of bt x bh x bw tokens, in raster order of their block
 * coordinates, cut at the grid edges (fewer tokens there).  Inside a 3-D block,
 * tokens are in raster order.
 * Block-major (tiled) buffers give every block `block` slots: its tokens first, in
 * the order above, then zero padding.  Key blocks: NT = ceil(n_text/block) text
 * blocks, NC context blocks, NQ chunk blocks; query blocks: the NQ chunk blocks.
 * The tiled problem is the la_shape written by la_grid3d_shape (Lq = NQ block,
 * Lk = (NT + NC + NQ) block, n_text = NT block, frame_tokens = 0), so text and
 * chunk blocks are forced and the NC context blocks are the historical candidates.
 * The padding of key blocks is masked through the per-block valid counts
 * (la_grid3d_valid, la_sparse_attn_fwd_valid); padded query rows are dropped by
 * la_untile_o_3d.
 * -------------------------------------------------------------------------- */
typedef struct la_grid3d {
  int32_t B, H, d;       /* batch, heads, head dimension (64 or 128) */
  int32_t n_text;        /* text tokens (>= 0) */
  int32_t T_ctx, T_q;    /* context frames (>= 0) and chunk frames (>= 1) */
  int32_t Hs, Ws;        /* latent frame height and width in tokens (>= 1) */
  int32_t bt, bh, bw;    /* 3-D block extents (>= 1), bt*bh*bw <= block */
  int32_t block;         /* slots per block in the tiled buffers: 64 or 128 */
} la_grid3d;

/* Part bits of la_prep_kv_3d: which regions of the tiled K/V buffers to write. */
enum { LA_PART_TEXT = 1, LA_PART_CONTEXT = 2, LA_PART_CHUNK = 4, LA_PART_ALL = 7 };

/* Host-only.  Validates the grid and writes the la_shape of the tiled problem.
 * LA_ERR_ARG for NULL pointers, LA_ERR_SHAPE for an invalid grid or a tiled shape
 * la_shape does not accept. */
la_status la_grid3d_shape(const la_grid3d* grid, la_shape* tiled);

/* Host-only.  Valid tokens per block, into host arrays: qvalid int32 [NQ] (may be
 * NULL) and kvalid int32 [NT + NC + NQ] (may be NULL). */
la_status la_grid3d_valid(const la_grid3d* grid, int32_t* qvalid, int32_t* kvalid);

/* Fused Q-Prep (Sec. 3.3, operator fusion; pooling equation): one pass over the
 * chunk queries that writes them block-major and pools every query block.
 *   q        bf16 [B, H, T_q Hs Ws, d], linear order                    (input)
 *   q_tiled  bf16 [B, H, NQ block, d]: block-major, padding slots zero
 *   qbar     float [B, H, NQ, d] or NULL: mean of each block's tokens (fp32 sums) */
la_status la_prep_q_3d(const la_grid3d* grid, const void* q, void* q_tiled, float* qbar, void* stream);

/* Fused KV-Prep (Sec. 3.3, operator fusion; pooling equation): reads K and V
 * together, writes the regions named in `parts` of the block-major buffers and
 * pools the K blocks it writes.  Regions not named are left untouched (a text or
 * context region written once can be kept across calls).
 *   k, v      bf16 [B, H, n_text + (T_ctx + T_q) Hs Ws, d], linear order   (inputs)
 *   k_tiled, v_tiled  bf16 [B, H, (NT + NC + NQ) block, d]
 *   kbar      float [B, H, NT + NC + NQ, d] or NULL: block means of K (rows of the
 *             written regions only)
 *   parts     non-zero subset of LA_PART_ALL, else LA_ERR_ARG. */
la_status la_prep_kv_3d(const la_grid3d* grid, const void* k, const void* v, uint32_t parts,
                        void* k_tiled, void* v_tiled, float* kbar, void* stream);

/* Block means of a 1-D block layout (Sec. 3.3, pooling equation), for callers that keep the
 * key means of the context across calls (the context keys do not change between the
 * denoising steps of a chunk; the paper computes them once, when K enters its KV buffer) and
 * select with la_select_pooled.
 *   which  LA_POOL_Q: x = q bf16 [B, H, Lq, d] -> xbar float [B, H, NQ, d];
 *          LA_POOL_K: x = k bf16 [B, H, Lk, d] -> xbar float [B, H, NK, d].
 *   A ragged last block is the mean of its valid rows.  Sums in fp32, then one multiply by
 *   1 / rows: the same values la_select_blocks pools internally, so selecting from them with
 *   la_select_pooled gives la_select_blocks' result.
 * A bad `which`, NULL or misaligned pointers are LA_ERR_ARG.  Needs no workspace. */
enum { LA_POOL_Q = 0, LA_POOL_K = 1 };
la_status la_pool_blocks(const la_shape* shape, const void* x, int32_t which, float* xbar, void* stream);

/* Block selection from pooled means (Sec. 3.3, selection equation), for block
 * layouts pooled elsewhere (la_pool_blocks, la_prep_q_3d, la_prep_kv_3d).
 *   shape  the tiled shape; qbar float [B, H, NQ, d], kbar float [B, H, NK, d] (rows
 *          of the M historical blocks are read).
 * Rules, outputs and errors as la_select_blocks / la_select_blocks_topk. */
la_status la_select_pooled(const la_shape* shape, const float* qbar, const float* kbar, float tau,
                           uint8_t* mask, int32_t* counts, int32_t* idx, void* ws, size_t ws_bytes,
                           void* stream);
la_status la_select_pooled_topk(const la_shape* shape, const float* qbar, const float* kbar,
                                int32_t keep_blocks, uint8_t* mask, int32_t* counts, int32_t* idx,
                                void* ws, size_t ws_bytes, void* stream);

/* la_sparse_attn_fwd / la_sparse_attn_plan for key blocks with padding.
 *   kvalid  int32 [NK] device array: key block m holds valid keys at its first
 *           kvalid[m] slots (clamped to [0, block]); the others are invisible.
 *           NULL = every slot valid (the plain calls).
 * la_sparse_attn_run and la_sparse_attn_merge serve both plans unchanged. */
la_status la_sparse_attn_fwd_valid(const la_shape* shape, const void* q, const void* k, const void* v,
                                   const int32_t* counts, const int32_t* idx, const int32_t* kvalid,
                                   float scale, void* o, float* lse, void* ws, size_t ws_bytes,
                                   void* stream);
la_status la_sparse_attn_plan_valid(const la_shape* shape, const int32_t* counts, const int32_t* idx,
                                    const int32_t* kvalid, void* ws, size_t ws_bytes, void* stream);

/* Fused Untile Scatter (Sec. 3.3, operator fusion): block-major attention output back
 * to linear order; padding slots are dropped.
 *   o_tiled   bf16 [B, H, NQ block, d]; lse_tiled float [B, H, NQ block] or NULL (inputs)
 *   o         bf16 [B, H, T_q Hs Ws, d]; lse float [B, H, T_q Hs Ws] (written when both
 *             lse pointers are given) */
la_status la_untile_o_3d(const la_grid3d* grid, const void* o_tiled, const float* lse_tiled, void* o,
                         float* lse, void* stream);

/* ------------------------------------------------------------------------------
 * Rotary positions: what turns queries and keys by their tokens' positions before an attention call.
 * Pair j of a head's first `rot` values is turned by positions[axis of j][token] * freqs[j] radians,
 *   (a, b) -> amplitude (a cos - b sin, b cos + a sin);
 * the pairs are (j, j + rot / 2), or with interleaved = 1 (2 j, 2 j + 1); the values from `rot` on are
 * copied.  Angles are computed and reduced in 64 bits, so far positions keep their precision; their sines
 * and cosines and the products are fp32.  A negative position turns back, and turning by -p undoes (and
 * is the gradient of) turning by p at amplitude 1.
 * -------------------------------------------------------------------------- */
typedef struct la_rope_shape {
  int32_t B, L;              /* sequences of L tokens (<= 2^26 - 4) that share their positions (packed tokens:
                                B = 1) */
  int32_t Hq, Hk;            /* heads of q and of k; 0: that tensor is not given */
  int32_t d;                 /* 64 or 128 */
  int32_t rot;               /* values of a head that are turned: a multiple of 16, 16 to d */
  int32_t interleaved;       /* 0 or 1 */
  int32_t dtype;             /* la_dtype of q and k and their outputs */
  int32_t axes;              /* rows of positions, 1 to 3 */
  int32_t section[3];        /* pairs of each axis, in the order of the pairs; they add up to rot / 2 */
  int64_t q_batch, q_token, q_head, qo_batch, qo_token, qo_head;    /* strides in elements, multiples of 8 */
  int64_t k_batch, k_token, k_head, ko_batch, ko_token, ko_head;
} la_rope_shape;

/*   q, k       rows of d contiguous values with the strides above (0: a broadcast), 16-byte aligned
 *   q_out, k_out  the same, rows that lie apart; each may be its input (with its strides)
 *   positions  int32 [axes, L] (device);  freqs  double [rot / 2] (device): radians per position.
 * One kernel launch.  LA_ERR_SHAPE for shapes and strides that do not fit, LA_ERR_ARG for pointers, a
 * bad dtype and an amplitude that is not finite. */
la_status la_rope(const la_rope_shape* shape, const void* q, void* q_out, const void* k, void* k_out,
                  const int32_t* positions, const double* freqs, float amplitude, void* stream);

/* ------------------------------------------------------------------------------
 * Packed sequences: attention over whole prompts, and over a cache in 4 bits.
 *
 * Tokens of S sequences of different lengths lie behind one another, q and o [Tq, Hq, d], k and v
 * [Tk, Hkv, d] in bf16 with the strides below (d contiguous); query head h reads key head
 * h / (Hq / Hkv).  Sequence s has the rows [cu_q[s], cu_q[s + 1]) of q and o.  The starts and
 * lengths are int32 device arrays and are read by the kernels.  They have to ascend from 0; starts
 * are clamped to the rows there are, and a sequence that would end before it starts has no rows, so
 * no value of them reads or writes outside the tensors.
 * Rows that no sequence covers (behind the last one) are not written.
 * Causal: query i of lq sees key n of lk where n <= i + lk - lq (the last query sees the last key).
 * A query that sees no key gives o = 0 and lse = -inf.  Values of keys outside the sequence do not
 * matter, whatever they hold; a key that some query of the sequence sees has to be finite.
 * -------------------------------------------------------------------------- */
typedef struct la_seqs {
  int32_t S;                 /* sequences (>= 0) */
  int32_t Tq, Tk;            /* rows of q and o, and of k and v (>= 0); these and S at most 2^31 - 4096 */
  int32_t Hq, Hkv;           /* heads, at most 65535: Hq a multiple of Hkv */
  int32_t d;                 /* 64 or 128 */
  int32_t causal;            /* 0 or 1 */
  int64_t q_token, q_head;   /* strides in elements, multiples of 8: a token's >= d and < 2^24, */
  int64_t o_token, o_head;   /* a head's >= 0 (0: the heads share one row; not for o) */
  int64_t k_token, k_head;
  int64_t v_token, v_head;
} la_seqs;

/* Bytes of scratch that la_prompt_attn needs (partial results of work that is split between
 * workgroups); 0 where it needs none (few keys), and for an invalid la_seqs. */
size_t la_prompt_ws_bytes(const la_seqs* seqs);

/* Attention over whole prompts: softmax(q k^T scale) v of every sequence over its own keys.
 *   cu_q, cu_k  int32 [S + 1]: first row of every sequence in q and in k; cu_k may be cu_q.
 *   scale       <= 0 selects 1/sqrt(d).
 *   o           bf16, strides o_token and o_head;  lse  float [Tq, Hq] or NULL: natural-log sum of
 *               exp(logits).
 * Softmax in fp32, products in bf16 with fp32 accumulation (the weights are rounded to bf16 for the one
 * with v).  Kernel launches only (one or two): a caller may capture the call; calls that may overlap need
 * a ws each. */
la_status la_prompt_attn(const la_seqs* seqs, const void* q, const void* k, const void* v,
                         const int32_t* cu_q, const int32_t* cu_k, float scale, void* o, float* lse,
                         void* ws, size_t ws_bytes, void* stream);

/* A learned bias by relative position, added to the logits (scale q.k) of la_prompt_attn: query i stands at place
 * i + lk - lq among its sequence's keys, and key n at distance n - that place,
 *   bias[h] = weight[bucket[clamp(distance, lo, hi) - lo]][h].
 * What the buckets are is the caller's: one for every distance, or ever wider ones.  A bucket outside
 * [0, buckets) has no bias (and takes no gradient).  A weight of -inf hides its distances; finite weights beyond
 * +-2^14 (-1e9 or a type's lowest value as a mask) count as +-2^14, which hides where other logits are within 16000 of
 * those hidden, and where a row sees nothing else leaves it the softmax of its q.k; +inf and NaN are not supported.  A
 * positive scale below 2^-60 is LA_ERR_ARG with a bias. */
typedef struct la_rel_bias {
  int32_t lo, hi;            /* lo <= hi <= lo + 512, both within +-2^20 */
  int32_t buckets;           /* rows of the weights: 1 to 2^20 */
  int32_t dtype;             /* la_dtype of the weights and of their gradient */
} la_rel_bias;

/* la_prompt_attn with a bias.
 *   bucket  int32 [hi - lo + 1], weight [buckets, Hq] (device).  `bias` NULL: la_prompt_attn.
 * The scratch is la_prompt_bias_ws_bytes(seqs, bias). */
size_t la_prompt_bias_ws_bytes(const la_seqs* seqs, const la_rel_bias* bias);
la_status la_prompt_attn_bias(const la_seqs* seqs, const la_rel_bias* bias, const void* q, const void* k, const void* v,
                              const int32_t* cu_q, const int32_t* cu_k, const int32_t* bucket, const void* weight,
                              float scale, void* o, float* lse, void* ws, size_t ws_bytes, void* stream);

/* Gradients of la_prompt_attn and la_prompt_attn_bias: with x the logits, P = exp(x - lse),
 * delta = do.o - dlse and dS = P (do.v - delta) over the pairs that see each other,
 *   dq = scale dS k,   dk = scale dS^T q,   dv = P^T do   (dk and dv summed over the query heads of a key head),
 *   dweight[b][h] = the sum of dS over the pairs of bucket b and head h, over all sequences.
 * The probabilities are recomputed from q, k and lse, whose rounding moves a row's by up to 0.2 % where |lse| is 2^14 (in
 * proportion elsewhere); they and dS are rounded to bf16 for their products, sums are fp32 (dweight's 64 bits between
 * workgroups) and in a fixed order: results repeat bit for bit on one device. */
typedef struct la_prompt_grads {
  int64_t do_token, do_head;   /* strides in elements, as in la_seqs: those of do may be a broadcast's (head 0) */
  int64_t dq_token, dq_head;
  int64_t dk_token, dk_head;
  int64_t dv_token, dv_head;
} la_prompt_grads;

/* Bytes of scratch that la_prompt_attn_bwd needs; 0 for invalid arguments.  bias NULL: none. */
size_t la_prompt_bwd_ws_bytes(const la_seqs* seqs, const la_rel_bias* bias);

/*   dout    bf16 [Tq, Hq, d] (do_token, do_head): the gradient of o.
 *   q, k, v, cu_q, cu_k, scale, and bucket and weight (with a bias): as in the forward call.
 *   o, lse  what the forward call left (o with o_token and o_head; lse float [Tq, Hq]).
 *   dlse    float [Tq, Hq] or NULL: the gradient of lse.
 *   dq [Tq, Hq, d], dk, dv [Tk, Hkv, d]  bf16, not overlapping each other or an input.  Rows that no sequence
 *           covers are not written; keys that no query sees get zeros.
 *   dweight [buckets, Hq] in the weights' type, with a bias: written whole.
 * A query that sees no key (lse = -inf) has no gradients and gives none, whatever its rows of do and dlse hold (NaN, say).
 * Kernel launches only: a caller may capture the call; calls that may overlap need a ws each. */
la_status la_prompt_attn_bwd(const la_seqs* seqs, const la_prompt_grads* grads, const la_rel_bias* bias,
                             const void* dout, const void* q, const void* k, const void* v, const void* o,
                             const float* lse, const float* dlse, const int32_t* cu_q, const int32_t* cu_k,
                             const int32_t* bucket, const void* weight, float scale, void* dq, void* dk, void* dv,
                             void* dweight, void* ws, size_t ws_bytes, void* stream);

/* A cache of keys and values in 4 bits, in pages that the sequences share.
 *   Values are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6, and their negatives) times a power of two that the 32
 *   values of a block of a row share: 4.25 bits per value.  The power is the smallest 2^e with the block's
 *   largest magnitude below 7 2^e, so that it is rounded by less than half a step (e is held to -125 .. 125);
 *   values are rounded to nearest, ties to the even code.  A block with a value that is not finite reads as NaN.
 *   cache  uint8 [n_pages, Hkv, la_kv4_page_bytes(d, page)], 16-byte aligned: per page and key head
 *            K codes [page][d / 2]              two values to a byte, the lower 4 bits first;
 *            K scales [d / 32][page]            2^(byte - 127), 255 = NaN;
 *            V codes [page / 4][16][4][d / 32]  quads of tokens: chunk c (values c d / 16 ..) of each in turn;
 *            V scales [d / 32][page].
 *   table  int32 [S, max_pages]: token n of sequence s lies on page table[s][n / page].  A page number
 *          outside [0, n_pages) is a page that does not exist: tokens on it are not written, and are
 *          read, by la_kv4_attn too, as rows of zeros.
 *   lens   int32 [S]: tokens of each sequence, the new ones included. */
typedef struct la_kv4 {
  int32_t n_pages;           /* >= 1 */
  int32_t page;              /* tokens of a page: a power of two, 16 to 1024 */
  int32_t max_pages;         /* pages of a row of the table, >= 1; a sequence ends at max_pages * page tokens, and at
                                2^31 - 4096 */
} la_kv4;

/* Bytes of one key head's part of a page, page (d + d / 16); 0 for an unsupported d or page. */
size_t la_kv4_page_bytes(int32_t d, int32_t page);

/* Enters rows of k and v into the cache.
 *   k, v  bf16 [Tk, Hkv, d] (la_seqs: S, Tk, Hkv, d and their strides are used; Hq is 0 or a multiple of
 *         Hkv; the rest is not looked at, here and for la_kv4_read).
 *   cu    int32 [S + 1]: rows [cu[s], cu[s + 1]) are the last tokens of sequence s, so that the last
 *         row is token lens[s] - 1.  Tokens before 0 or past the table are dropped.
 * Two rows must not go to one place (a page that two sequences share is entered by one of them).  Tk is
 * at most 2^28 - 32, here and for la_kv4_read. */
la_status la_kv4_append(const la_seqs* seqs, const la_kv4* kv, const void* k, const void* v, const int32_t* cu,
                        const int32_t* lens, const int32_t* table, void* cache, void* stream);

/* The values that the last cu[s + 1] - cu[s] tokens of every sequence stand for, into rows of k and v:
 * la_kv4_append's places, read back (exactly: every value of the cache is a bf16 value).  Tokens that
 * have no place come as zeros; rows of no sequence are not written. */
la_status la_kv4_read(const la_seqs* seqs, const la_kv4* kv, const void* cache, const int32_t* cu,
                      const int32_t* lens, const int32_t* table, void* k, void* v, void* stream);

/* Bytes of scratch that la_kv4_attn needs; 0 where it needs none (tables of few tokens), and for
 * invalid arguments. */
size_t la_kv4_ws_bytes(const la_seqs* seqs, const la_kv4* kv, int32_t max_q);

/* Attention of every sequence's queries over its cache: la_prompt_attn with the keys and values that
 * the cache stands for (the strides of k and v in la_seqs are not looked at; Tk is not used, and may be 0 or
 * any valid number).  With causal = 1 the last query sees the last of lens[s] tokens.
 *   max_q  no sequence has more query rows; those of one that has are not written.
 * Whether work is split, and which kernel takes it, goes by what the table can hold, so a table no wider than
 * the sequences need makes small calls faster. */
la_status la_kv4_attn(const la_seqs* seqs, const la_kv4* kv, int32_t max_q, const void* q, const void* cache,
                      const int32_t* cu_q, const int32_t* lens, const int32_t* table, float scale, void* o,
                      float* lse, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------------
 * The scalar policy around the path: adaptive context management (Sec. 3.1) and the
 * denoising cache (Sec. 3.2).  Only the latent dynamics runs on the GPU; the other
 * calls are host-only scalar rules (no GPU, no stream), exact in double precision.
 * Camera-pose similarities are inputs: the paper instantiates them with an FOV
 * overlap measure it does not define.
 * -------------------------------------------------------------------------- */
/* Workspace bytes of la_latent_mse (fp64 partial sums; 256-byte aligned). */
#define LA_LATENT_MSE_WS_BYTES 8192

/* Latent dynamics D_t = MSE(z_{t-1}, z_{t-2}) (Sec. 3.1, latent-dynamics equation): the mean
 * over all n values of (z_a - z_b)^2.
 *   z_a, z_b  device arrays of n values of `dtype` (fp32 or bf16), 16-byte aligned; any
 *             layout, the same for both (the mean runs over every latent dimension).
 *   out       device double: D_t.  Squares are summed in fp32 within 16-byte chunks and in
 *             fp64 beyond; the order is fixed by n, so the result is bit-reproducible.
 *   ws        LA_LATENT_MSE_WS_BYTES of device scratch.
 * n < 1, a bad dtype, NULL or misaligned pointers are LA_ERR_ARG. */
la_status la_latent_mse(const void* z_a, const void* z_b, int64_t n, int32_t dtype, double* out,
                        void* ws, size_t ws_bytes, void* stream);

/* Host-only.  Moving average D_bar_t = alpha D_t + (1 - alpha) D_bar_{t-1} (Sec. 3.1,
 * smoothing equation); D_bar_prev NULL starts the average with D_t.  alpha in (0, 1],
 * D_t >= 0, else LA_ERR_ARG. */
la_status la_dynamics_ema(double D_t, const double* D_bar_prev, double alpha, double* D_bar);

/* Host-only.  Temporal window L_t = clip(floor(L_m kappa / (D_bar + kappa)), 1, L_m)
 * (Sec. 3.1, window equation).  kappa > 0, L_m >= 1, D_bar >= 0, else LA_ERR_ARG. */
la_status la_temporal_window(double D_bar, double kappa, int32_t L_m, int32_t* L_t);

/* Host-only.  Pose gate (Sec. 3.1 retrieved-memory gate, Sec. 3.2 reuse condition):
 * *revisiting = 1 when max_j similarities[j] >= tau_pose (keep the retrieved memory, allow
 * denoising reuse), 0 for pure exploration or n = 0 (discard the retrieved memory).
 * similarities: host array of n floats; NaN entries are LA_ERR_ARG. */
la_status la_pose_revisiting(const float* similarities, int32_t n, float tau_pose, int32_t* revisiting);

/* Host-only.  Denoising-cache schedule over K steps (Sec. 3.2, reuse equation): source[i] =
 * the step whose model output step i uses, i for an evaluated step and 0 for the reused
 * intermediate steps 1..K-2 when reuse != 0 and K > 2; the model is evaluated at steps i with
 * source[i] == i.  source: host array of K int32.  K < 1 is LA_ERR_ARG. */
la_status la_denoise_schedule(int32_t K, int32_t reuse, int32_t* source);

/* Static description of a status code. */
const char* la_status_string(la_status status);

/* ABI version of this header: 1. */
int32_t la_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* LA_H_ */
