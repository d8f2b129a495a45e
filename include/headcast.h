/*
 * headcast.h -- C ABI of the HeadCast routed-attention library for MI355X (gfx950).
 *
 * HeadCast (arXiv 2607.20125) classifies every attention head of an
 * autoregressive video-diffusion model once (Sec. 4.2), splits the KV cache
 * along the head dimension into per-archetype buffers (Sec. 4.3) and then runs
 * each head on its own attention path (Sec. 4.4):
 *
 *   Sink    -- attends to the L keys of block 0 (the frozen sink block),
 *   Dummy   -- attends to the L keys of the current block,
 *   Spatial -- attends, in every frame of the window, to the positions within
 *              a (2r+1) x (2r+1) square around the query (clipped at borders),
 *   Global  -- attends to the whole sliding window (W blocks, current included).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  * One block holds L = frames_per_block * grid_h * grid_w tokens.  Token t of
 *    a block sits at frame f, row y, column x with t = f*grid_h*grid_w + y*grid_w + x.
 *  * q, k, v tensors are bfloat16, row-major [n_heads][tokens][head_dim], in
 *    device memory owned by the caller.  Outputs are float32 [n_heads][L][head_dim].
 *    Every device pointer must be 16-byte aligned (the kernels move 16-byte
 *    vectors); a misaligned one is HC_E_INVAL, checked before any work is queued.
 *  * A window is passed in logical order: block 0 first, then the retained
 *    blocks from oldest to newest, the current block last.  Before the window
 *    first fills (cur_block < window_blocks - 1) it holds blocks 0..cur_block.
 *  * Softmax scale s defaults to 1/sqrt(head_dim); all arithmetic on bf16
 *    inputs accumulates in float32 (QK^T and PV on the matrix cores).  Each
 *    work group first runs the softmax with its offset fixed at 0 (exact while
 *    no exponential overflows or underflows, which it checks on its row sums
 *    and accumulators) and otherwise reruns its keys as an online softmax with
 *    a running max and sum.  Partial results over key ranges are merged with
 *    their maxima and sums.
 *  * Streams: `hc_stream` is a hipStream_t (NULL = the null stream).  Work is
 *    enqueued asynchronously on it unless an entry point says otherwise.
 *  * Graph capture: once hc_attention has run on a layer at its current window
 *    fill, hc_append_block of the current block (the rewrite of a denoising
 *    step) and hc_attention only enqueue kernels on the given stream (no
 *    allocation, copy, memset or synchronisation) and may be captured into a HIP
 *    graph.  The context's host state (current block, window fill) changes when
 *    a call is made, not when a graph replays it, so a captured sequence must not
 *    advance the block; the first hc_attention at a new window fill builds the
 *    layer's work list (it allocates, and waits for the device where an older list
 *    may be in use or the layer's cache was last written on another stream) and
 *    runs eagerly.  Partial results are shared by a context's layers: a call that
 *    sets a table or builds a list may move them, so a graph is captured after the
 *    last such call of any layer and replayed until the next.
 *  * Errors: every entry point returns an hc_status; nothing is thrown across
 *    the ABI.  On failure the context keeps a message (hc_last_error) and the
 *    layer state is left as it was before the call, with two exceptions: after
 *    HC_E_DEVICE the device memory contents of that layer are unspecified, and
 *    after HC_E_NOMEM or HC_E_DEVICE from hc_set_head_types or
 *    hc_classify_heads the layer may have no head table (its old buffers are
 *    released before the new ones are allocated, so replacing a table never
 *    needs the memory of two); it then answers HC_E_STATE until a table is set.
 *  * A context is not thread-safe; use one context per stream of work.
 */
#ifndef HEADCAST_H
#define HEADCAST_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hc_ctx hc_ctx;
typedef void *hc_stream;   /* hipStream_t */

typedef enum {
  HC_OK = 0,
  HC_E_INVAL = -1,   /* bad argument: null pointer, bad layer, bad size, bad label   */
  HC_E_STATE = -2,   /* call not valid in the layer's current state                  */
  HC_E_ORDER = -3,   /* block index neither the current block nor the next one       */
  HC_E_NOMEM = -4,   /* an allocation failed (device or host memory)                  */
  HC_E_DEVICE = -5   /* a HIP runtime call failed (message in hc_last_error)          */
} hc_status;

/* Head archetypes (Sec. 3.2 observations, Sec. 4.2 decision rule). uint8 per head. */
enum { HC_SINK = 0, HC_DUMMY = 1, HC_SPATIAL = 2, HC_GLOBAL = 3 };

/* Per-head classification statistics written by hc_classify_heads (Eq. 3, Eq. 4). */
enum {
  HC_STAT_COS_SINK = 0,    /* mean token cosine of the Sink proxy vs O_ref      */
  HC_STAT_COS_DUMMY = 1,   /* mean token cosine of the Dummy proxy vs O_ref     */
  HC_STAT_COS_SPATIAL = 2, /* mean token cosine of the Spatial proxy vs O_ref   */
  HC_STAT_P5 = 3,          /* 5th percentile of the Spatial token cosines       */
  HC_STAT_MSE = 4,         /* mean squared difference O_spatial - O_ref         */
  HC_STAT_SCORE = 5,       /* P5 - gamma * MSE                                  */
  HC_N_STATS = 6
};

typedef struct {
  int32_t n_layers;          /* layers the context manages (>= 1)                      */
  int32_t n_heads;           /* heads per layer, 1..64                                 */
  int32_t head_dim;          /* 64 or 128                                              */
  int32_t grid_h, grid_w;    /* latent tokens per frame = grid_h * grid_w              */
  int32_t frames_per_block;  /* 1..4 latent frames per block (Sec. 5.1 uses 3)         */
  int32_t window_blocks;     /* W >= 2, counts the frozen sink block and the current   */
  int32_t spatial_radius;    /* r of the deployed Spatial path, 0..12                  */
  int32_t proxy_radius;      /* r_p of the classification Spatial proxy, 0..12 (Sec. 5.1: 2) */
  float theta_sink;          /* Eq. 5 thresholds (Sec. 5.1: 0.95, 0.95, 0.95, 0.755)  */
  float theta_dummy;
  float theta_spatial;
  float theta_score;
  float gamma;               /* MSE weight of Eq. 4 (Sec. 5.1: 5)                     */
  float softmax_scale;       /* 0 => 1/sqrt(head_dim)                                 */
  int32_t spatial_cell;      /* 0: Spatial heads use the centred (2r+1)^2 window (the
                              * Sec. 4.2 proxy geometry).  c in 2..64: the deployed cell
                              * variant of Sec. 4.4 -- every frame is cut into c x c
                              * cells (round(grid/c) per axis, halves rounded up, the last
                              * cell ending at the border) and a query attends to its own
                              * cell in every window frame (Sec. 5.1: c = 10).  At most 64
                              * cells per axis.  The classification proxy always uses the
                              * centred window of radius proxy_radius.                  */
  int32_t sd_blocks;         /* 1: a Sink head attends to block 0 and a Dummy head to the
                              * current block (L keys; the Sec. 4.2 proxies and the
                              * "exactly one block" of Sec. 4.4).  2: the App. B / App. C
                              * reading -- Sink to block 0 and the current block, Dummy
                              * to the previous and the current block (2L keys once a
                              * previous block exists; needs window_blocks >= 3 so that
                              * the previous block lies in the window, else
                              * HC_E_INVAL).  The classification proxies use one block
                              * either way.                                             */
} hc_config;

/* Fills the paper's defaults (Sec. 5.1) for a 30 x 12-head, head_dim 128,
 * 3-frame-block, 7-block-window model at a 30x52 latent grid, r = 4, r_p = 2.
 * Never fails. */
void hc_config_default(hc_config *cfg);

/* HC_OK if the configuration is usable, else HC_E_INVAL.  Pure host check.
 * Besides the ranges above: L = frames_per_block*grid_h*grid_w must be a
 * multiple of 8 and W*L must fit in int32. */
hc_status hc_validate_config(const hc_config *cfg);

/* Static strings, never NULL. */
const char *hc_status_string(hc_status s);
/* Message of the last failing call on ctx ("" if none); valid until the next call. */
const char *hc_last_error(const hc_ctx *ctx);

/* Physical ring slot that block `block` occupies in a Global or Spatial buffer
 * with `window_blocks` slots: slot 0 keeps block 0 for good; later blocks
 * rotate through slots 1..W-1, evicting the oldest rolling block (Sec. 4.3,
 * "sliding-window layout retaining the initial sink tokens").  Pure host
 * function; returns -1 for block < 0 or window_blocks < 2. */
int32_t hc_ring_slot(int64_t block, int32_t window_blocks);

/* Creates a context on HIP device `device`.  The context owns all per-layer
 * compact buffers, head tables and work lists; it allocates per-layer buffers
 * when head types are first set.  Returns HC_E_INVAL (bad config / null out),
 * HC_E_DEVICE (device not usable) or HC_E_NOMEM. */
hc_status hc_create(const hc_config *cfg, int device, hc_ctx **out);
void hc_destroy(hc_ctx *ctx);   /* NULL is allowed; synchronises the device first */

/* One-time online classification of one layer (Sec. 4.2, Eq. 2-5), followed by
 * the cache split (Sec. 4.3).
 *   q      : bf16 [H][L][d]   queries of the current block (device)
 *   k_win, v_win : bf16 [H][W*L][d] the full window in logical order (device)
 *   types_out : host uint8 [H]   decided archetype per head (required)
 *   stats_out : host double [H][HC_N_STATS] statistics, or NULL
 * The current block is `cur_block`; the window must be full, i.e.
 * cur_block >= W-1 (the paper fires classification when the window first
 * fills), else HC_E_STATE.  Computes O_ref and the three proxy outputs, the
 * per-token cosines and squared errors, and per head the means, P5 (exact
 * order statistics, linear interpolation at rank 0.05 (L-1)), MSE and score
 * on the GPU (statistics in float64), and the Eq. 5 decision on the host from
 * those six numbers.  Then sets the layer's head
 * table and splits k_win / v_win into the compact buffers, exactly as
 * hc_set_head_types would.  SYNCHRONISES `stream` (the labels are host
 * outputs).  Needs device memory of about 2 * H*W*L*d*2 bytes (the window in
 * Global layout) + the window in Spatial layout (rows padded to a multiple of 8
 * keys) unless grid_w is a multiple of 8 + 4 * H*L*d*4 bytes (the proxy
 * outputs) + the per-block partials (H*W*ceil(L/128) slots of 128*(d+2) floats)
 * + the token statistics (about H*L doubles): the first call allocates it, the
 * context keeps it for
 * later calls (every layer of a generation) and releases it in hc_destroy;
 * hc_memory_bytes counts it. */
hc_status hc_classify_heads(hc_ctx *ctx, int layer, int64_t cur_block, const void *q,
                            const void *k_win, const void *v_win, uint8_t *types_out,
                            double *stats_out, hc_stream stream);

/* The classification outputs of the last hc_classify_heads call on this
 * context that returned HC_OK (Sec. 4.2: Eq. 2 and the three proxies), for
 * inspection of a decision and for checking the classification attention on
 * its own.  which: HC_CLS_O_REF (attention over the full window),
 * HC_CLS_O_SINK (block 0 alone), HC_CLS_O_DUMMY (the current block alone),
 * HC_CLS_O_SPATIAL (centred window of radius proxy_radius in every window
 * frame).  dst: device float32 [H][L][d], written by a copy enqueued on
 * `stream`.  The outputs are those of the layer classified last (each call
 * overwrites them).  HC_E_STATE before a successful classification,
 * HC_E_INVAL for another `which` or a NULL or misaligned dst. */
enum {
  HC_CLS_O_REF = 0,
  HC_CLS_O_SINK = 1,
  HC_CLS_O_DUMMY = 2,
  HC_CLS_O_SPATIAL = 3
};
hc_status hc_classify_outputs(hc_ctx *ctx, int which, float *dst, hc_stream stream);

/* Sets a layer's head table without classifying (restored labels, fixed
 * tables, the all-Global full-window baseline) and splits the given window
 * (bf16 [H][n*L][d], n = min(cur_block+1, W), logical order, device) into
 * compact buffers (Sec. 4.3): Sink heads keep block 0, Dummy heads the current
 * block, Global and Spatial heads the whole window in ring slots.
 * types: host uint8 [H] with values HC_SINK..HC_GLOBAL (else HC_E_INVAL).
 * Re-setting a layer replaces its buffers.  Async on `stream` apart from
 * allocation. */
hc_status hc_set_head_types(hc_ctx *ctx, int layer, const uint8_t *types, int64_t cur_block,
                            const void *k_win, const void *v_win, hc_stream stream);

/* Layout integers of a layer (host outputs):
 *   head_slot [H] : index of each head inside its buffer; Sink and Dummy heads
 *                   share the Sink-Dummy buffer; heads keep head-id order.
 *   ring_slot_of_logical [W] : physical slot of each logical window position
 *                   (sink block first, current block last), -1 while empty.
 * Either pointer may be NULL.  HC_E_STATE if the layer has no head table. */
hc_status hc_get_layout(const hc_ctx *ctx, int layer, int32_t *head_slot,
                        int32_t *ring_slot_of_logical);

/* Writes one block's K and V (bf16 [H][L][d], device) into the layer's
 * buffers (Sec. 4.3): Global and Spatial heads into the block's ring slot,
 * Dummy heads over their single block (rolling overwrite), Sink heads only for
 * block 0.  `block` equal to the current block overwrites it (the next
 * denoising step of the same block); current + 1 advances the window and
 * evicts the oldest rolling block.  Anything else: HC_E_ORDER.  HC_E_STATE if
 * the layer has no head table.  Async. */
hc_status hc_append_block(hc_ctx *ctx, int layer, int64_t block, const void *k_blk,
                          const void *v_blk, hc_stream stream);

/* Head-specific attention of one layer over all heads (Sec. 4.4):
 *   q : bf16 [H][L][d] queries of the current block (device)
 *   head_types : host uint8 [H]; must equal the layer's table (else HC_E_STATE)
 *   o : float32 [H][L][d] (device), every head written in place.
 * Launches the grouped work of the layer: every Global head is cut into one
 * work unit per window block (small windows stay whole) and every Sink/Dummy head
 * into one unit (per block), each unit 128 queries wide, and the last units of the
 * list into pieces where that ends the launch earlier; partial results of cut
 * heads are merged by a further launch.  Spatial heads run on the windowed kernel
 * (when they give too few work groups to fill the GPU, their key frames are cut
 * into ranges whose partial results the same launch merges).  Async. */
hc_status hc_attention(hc_ctx *ctx, int layer, const void *q, const uint8_t *head_types,
                       float *o, hc_stream stream);

/* Bytes of the fixed device scratch that hc_attention_static works in. */
#define HC_STATIC_SCRATCH_BYTES (64u << 20)

/* hc_attention for callers that cannot allocate device memory: code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation.  Same
 * arguments, head table check and outputs as hc_attention (within its
 * floating-point tolerance: the work is not tail-balanced, so partial results
 * may be merged in another order).  It allocates nothing, copies nothing from
 * the host and does not synchronise: the layer's work list, the per-block
 * partial results of Global (and two-block Sink/Dummy) heads and the split
 * partials of Spatial heads live in one fixed array of HC_STATIC_SCRATCH_BYTES
 * per GPU, held by the library until the process ends (Spatial and other
 * partials take turns in the same place where not both fit); the work list is
 * written by a kernel on `stream` at every call.  The key ranges of that list are
 * chosen on the host by the first call at a window fill (some microseconds, up to
 * about 50 for layers that run 150 and more; layers with as many heads of each kind
 * share the choice).  Every call on a GPU uses
 * that GPU's array and leaves its contents behind, so calls that overlap on
 * one GPU (other streams, other contexts, other threads) race and must be
 * ordered by the caller.  A layer whose work needs more than the array holds
 * (the Spatial split is reduced to what fits first) is HC_E_INVAL with the size in
 * hc_last_error, before anything is enqueued; so is a context with the cell
 * variant (spatial_cell > 0).  The layer's buffers are the context's, set up
 * beforehand by hc_set_head_types / hc_classify_heads. */
hc_status hc_attention_static(hc_ctx *ctx, int layer, const void *q, const uint8_t *head_types,
                              float *o, hc_stream stream);

/* Device bytes held by the context's buffers (all layers, partial-result
 * slots, and the classification memory once hc_classify_heads has run). */
hc_status hc_memory_bytes(const hc_ctx *ctx, int64_t *bytes);

/* ---------------------------------------------------------------------------
 * Operators beside the routed attention: what a model runs before it (rotary
 * positions), the attention over whole prompts and clips, and a cache held in 4
 * bits with its attention.  They take a context for its device, its message
 * (hc_last_error) and its kernel timing only: sizes and heads are arguments of
 * the call, not the context's.  They allocate nothing, copy nothing and do not
 * synchronise, so they may be captured into a HIP graph; a call that needs room for
 * partial results takes it from the caller, and two graphs (or two calls at once)
 * need a workspace each.  The calling thread's current device is left as it was.
 * Pointers are 16-byte aligned unless said otherwise, strides are in elements and
 * multiples of 8 (neighbouring dims of a head are always 1 apart; the stride of an axis of
 * length 1 is not looked at).  Lengths and
 * offsets in device memory are read when the call runs: they cannot be checked
 * by the host, and values out of range are clamped, so that nothing outside the
 * given tensors is read or written.
 * ------------------------------------------------------------------------- */
enum { HC_BF16 = 0, HC_F32 = 1 };

/* Rotary positions over several axes.  The first rot = sum(axis_dims) dims of
 * every head form rot / 2 pairs: dims (2i, 2i + 1), or (i, i + rot / 2) with
 * `halves`.  axis_dims[0] / 2 pairs turn with the position on axis 0, the next
 * axis_dims[1] / 2 with that on axis 1, and so on, by the angle
 * position * theta^(-2 j / m): j counts the pairs of the axis and m = axis_dims, or
 * with `joint` j counts all pairs and m = rot.  (a, b) becomes
 * (a cos - b sin, a sin + b cos); with `inverse` the angle's sign changes, which
 * also is the gradient of the rotation.  Dims behind rot are copied.  Angles are
 * computed in 64 bits; their sines and cosines, by the hardware's instructions on a fraction of a
 * turn rounded to 32 bits, are off by at most 2.8e-7; the rotation is in 32 bits, rounded once to the
 * output's type.
 *
 * Positions: int32 [n_axes][n_tokens] in device memory (4-byte aligned), or NULL for the
 * tokens of consecutive frames (n_axes = 3: frame, row, column): token t is at frame
 * frame0 + t / (grid_h grid_w), row t / grid_w % grid_h, column t % grid_w. */
typedef struct {
  const void *x;             /* [n_tokens][n_heads][head_dim] by the strides below       */
  void *out;                 /* may be x itself with equal strides and types, and may
                              * not overlap it otherwise; of two tensors, neither's output
                              * overlaps the other's input or output                     */
  int64_t x_token, x_head, out_token, out_head;
  int32_t n_heads;           /* >= 1                                                     */
} hc_rotate_tensor;

typedef struct {
  int32_t n_tokens;          /* 0 does nothing                                           */
  int32_t head_dim;          /* a multiple of 8, at most 256                             */
  int32_t x_type, out_type;  /* HC_BF16 or HC_F32, for all tensors of the call           */
  int32_t n_axes;            /* 1..4                                                     */
  int32_t axis_dims[4];      /* even; their sum is a multiple of 16, at most head_dim     */
  int32_t halves, joint, inverse;
  int32_t grid_h, grid_w, frame0;
  double theta;              /* > 0, finite; angles of positions up to 2^31 finite too   */
  const int32_t *positions;
} hc_rotate_args;

/* Rotates one or two tensors (a block's queries and keys) of the same tokens in one
 * launch.  Async. */
hc_status hc_rotate(hc_ctx *ctx, const hc_rotate_args *args, const hc_rotate_tensor *tensors,
                    int n_tensors, hc_stream stream);

/* Attention over packed sequences: prompts, clips, or blocks over their own text.
 * The queries of sequence s are rows cu_q[s] .. cu_q[s+1] - 1 of q, its keys rows
 * cu_k[s] .. cu_k[s+1] - 1 of k and v (bfloat16).  Query head h reads key head
 * h / (n_heads / n_kv_heads).  With n queries and m keys, query i of a sequence sits at
 * position p = m - n + i and sees, of the m keys,
 *   causal_block = 0      all,
 *   causal_block = c > 0  those before (p / c + 1) c, none if p < 0: c = 1 is the
 *                         causal mask, c = block_tokens lets a block see itself and
 *                         every earlier block.
 * A query that sees nothing gets zeros.  Output rows outside every sequence are
 * left as they were.  Probabilities are rounded to bfloat16 for the product with the values, as in
 * hc_attention; logits, the softmax's maxima and sums (of the rounded probabilities) and the outputs'
 * sums are float32, rounded once to the output.  Logits may be up to 2^28 in magnitude (times log2 e):
 * a running maximum is rounded by 2^-24 of itself, and beyond that its rounding nears the range of exp2.
 * A NaN or infinity in a sequence's own keys or values may reach any of that sequence's queries, and no
 * other sequence's. */
typedef struct {
  const void *q, *k, *v;     /* bf16 [tokens][heads][head_dim] by the strides below       */
  void *out;                 /* bf16 [n_tokens][n_heads][head_dim]; may be q itself with
                              * the same strides, and overlaps no input otherwise        */
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;
  int32_t n_tokens;          /* rows of q and out; 0 does nothing                        */
  int32_t n_keys;            /* rows of k and v, at most 2^31 - 65                        */
  int32_t n_seqs;            /* >= 1                                                     */
  int32_t n_heads, n_kv_heads;   /* n_heads a multiple of n_kv_heads                      */
  int32_t head_dim;          /* 64 or 128                                                */
  int32_t causal_block;      /* >= 0                                                     */
  float softmax_scale;       /* 0 => 1/sqrt(head_dim)                                    */
  const int32_t *cu_q;       /* device [n_seqs + 1] (4-byte aligned); NULL: n_seqs equal
                              * parts (n_tokens a multiple of n_seqs)                    */
  const int32_t *cu_k;       /* NULL: the queries' offsets (n_keys = n_tokens then)       */
  void *workspace;           /* hc_packed_workspace bytes, NULL if that is 0              */
  int64_t workspace_bytes;
} hc_packed_args;

/* Bytes of workspace that hc_packed_attention needs for these arguments (its device
 * pointers are not read).  Pure host. */
hc_status hc_packed_workspace(hc_ctx *ctx, const hc_packed_args *args, int64_t *bytes);
hc_status hc_packed_attention(hc_ctx *ctx, const hc_packed_args *args, hc_stream stream);

/* A cache of keys and values in 4 bits, in memory of the caller: n_seqs sequences of
 * up to `capacity` tokens, hc_qcache_bytes bytes at `data`.  Every 32 neighbouring dims
 * of a token share a power of two 2^e, and each is stored as the nearest of
 * 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e with its sign (ties to an even code).  For the
 * largest magnitude a of the 32, 2^k <= a < 2^(k+1): e = k - 2, or k - 1 if a > 7/4 2^k,
 * so that no value is off by more than half a step; e stays in [-125, 125].  If one
 * of the 32 is infinite or NaN, all of them read back as NaN.  The layout inside is the
 * library's own.  Slots that were never written hold nothing that is read, as long as
 * lengths say so: memory need not be cleared. */
typedef struct {
  void *data;
  int32_t n_seqs;            /* >= 1                                                     */
  int32_t n_heads;           /* key heads, >= 1                                          */
  int32_t head_dim;          /* 64 or 128                                                */
  int32_t capacity;          /* tokens per sequence, >= 1                                */
} hc_qcache;

hc_status hc_qcache_bytes(const hc_qcache *cache, int64_t *bytes);   /* `data` is not read */

/* Tokens for (append) or from (read) the cache: rows cu_seqlens[s] .. cu_seqlens[s+1] - 1
 * of k and v are slots start[s], start[s] + 1, ... of sequence s (NULL cu_seqlens: n_seqs
 * equal parts).  Rows whose slot lies outside [0, capacity), or that belong to no sequence,
 * are neither stored nor written.  A slot may be written again (a block's next denoising
 * step, a ring of blocks).  Async. */
typedef struct {
  void *k, *v;               /* bf16 [n_tokens][n_heads][head_dim] by the strides below; hc_qcache_append
                              * only reads them, hc_qcache_read writes both: then they do not
                              * overlap                                                  */
  int64_t k_token, k_head, v_token, v_head;
  int32_t n_tokens;          /* 0 does nothing                                           */
  const int32_t *start;      /* device [n_seqs] (4-byte aligned)                          */
  const int32_t *cu_seqlens; /* device [n_seqs + 1], or NULL                              */
} hc_qcache_rows;

hc_status hc_qcache_append(hc_ctx *ctx, const hc_qcache *cache, const hc_qcache_rows *rows,
                           hc_stream stream);
hc_status hc_qcache_read(hc_ctx *ctx, const hc_qcache *cache, const hc_qcache_rows *rows,
                         hc_stream stream);

/* Attention of new queries over the first kv_len[s] slots of each sequence, with the
 * position and mask rules of hc_packed_attention (m = kv_len[s]).  The keys and values
 * are the stored 4-bit ones; roundings and the range of logits are those of hc_packed_attention too.
 * With a ring of blocks (slots not in the order of positions) use causal_block = 0.
 * kv_len is clamped to [0, capacity]. */
typedef struct {
  const void *q;             /* bf16 [n_tokens][n_heads][head_dim]                        */
  void *out;                 /* bf16, the same shape; may be q itself with the same strides,
                              * and does not overlap it otherwise                        */
  int64_t q_token, q_head, out_token, out_head;
  int32_t n_tokens;          /* 0 does nothing                                           */
  int32_t n_heads;           /* a multiple of the cache's heads                           */
  int32_t causal_block;
  int32_t max_kv;            /* about the longest kv_len, 0 if unknown: the key range of a
                              * query is split by it; the result does not depend on it
                              * beyond rounding                                          */
  float softmax_scale;       /* 0 => 1/sqrt(head_dim)                                    */
  const int32_t *kv_len;     /* device [n_seqs] (4-byte aligned)                          */
  const int32_t *cu_seqlens; /* device [n_seqs + 1]; NULL: n_seqs equal parts             */
  void *workspace;           /* hc_qcache_workspace bytes, NULL if that is 0              */
  int64_t workspace_bytes;
} hc_qcache_attention_args;

hc_status hc_qcache_workspace(hc_ctx *ctx, const hc_qcache *cache,
                              const hc_qcache_attention_args *args, int64_t *bytes);
hc_status hc_qcache_attention(hc_ctx *ctx, const hc_qcache *cache,
                              const hc_qcache_attention_args *args, hc_stream stream);

/* Kernel timing: when enabled, every launch the context makes records a pair
 * of HIP events on the stream it is launched on.  hc_profile_read synchronises
 * those events and returns the summed duration (ms) and the launch count of
 * one kernel kind since the last reset, then resets it.  A merge of partials
 * counts as HC_K_COMBINE; one of Spatial ranges alone is timed with its
 * HC_K_SPATIAL launch.  HC_K_SEQUENCE is hc_packed_attention and
 * hc_qcache_attention (the merge of their key ranges included), HC_K_CACHE hc_qcache_append and
 * hc_qcache_read. */
enum { HC_K_DENSE = 0, HC_K_SPATIAL = 1, HC_K_SCATTER = 2, HC_K_STATS = 3, HC_K_COMBINE = 4,
       HC_K_ROTATE = 5, HC_K_SEQUENCE = 6, HC_K_CACHE = 7, HC_K_COUNT = 8 };
hc_status hc_profile_enable(hc_ctx *ctx, int on);
hc_status hc_profile_read(hc_ctx *ctx, int kernel_kind, double *total_ms, int64_t *launches);

#ifdef __cplusplus
}
#endif
#endif /* HEADCAST_H */
