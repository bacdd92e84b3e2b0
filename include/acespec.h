/*
 * acespec.h -- C ABI of the MI355X (gfx950) tree-verification library.
 *
 * The library implements the cloud side of AceSpec's edge-cloud speculative decoding
 * (Section III-B, "Verify Loop"): one forward pass of a decoder-only target model over a
 * batch of drafted token trees, each node attending to its session's KV prefix and to its
 * own ancestors (Section III-C, tree attention mask), followed by the per-node reduction
 * of the target distribution to what the downlink carries (Algorithm 1, RECEIVE_WAIT
 * returns the rejection index and a sparse target distribution): the min(1, p/q)
 * acceptance test against the draft distribution, the residual max(0, p - q) resample,
 * a bonus sample, and a top-k sparse distribution; then the per-session path walk with
 * the sibling-hit rule of Algorithm 1 (the resampled token looked up among the drafted
 * alternatives).
 *
 * Conventions for every entry point:
 *  - All tensor pointers are DEVICE pointers, owned by the caller; the library never
 *    frees them.  Layouts are dense row-major with the shapes given in the comments.
 *  - Work is enqueued on `stream`; the call returns without synchronising and the
 *    outputs are valid once the stream has completed.
 *  - Argument and shape errors are reported synchronously, before anything is
 *    launched, by a negative return code; acespec_last_error() then holds a message.
 *  - Malformed per-session data found on the device sets status[b] for that session
 *    only; its other outputs are then unspecified but every access stays in bounds:
 *      ACESPEC_EBADTREE    a parent index that is not an earlier row, a token id outside
 *                          the vocabulary, a prefix length that does not fit the cache;
 *      ACESPEC_EBADDRAFT   a draft distribution the step reads holds a NaN, infinite or
 *                          negative entry (dense draft_q rows with children), or a scalar
 *                          q_hat outside [0, 1];
 *      ACESPEC_ENONFINITE  a target logit of the session is not finite: an activation
 *                          left the range of the 16-bit type it is handed on in (fp16
 *                          between the kernels of a bf16 model, max 65504), or the
 *                          weights, KV cache or hidden states hold NaN/inf.
 *    When several apply the first in this list that the step detects is reported
 *    (tree checks run before the forward pass; of the two data errors the
 *    non-finite logits win).
 *  - No C++ exception crosses this interface.
 *  - A context must not be used by two calls that overlap in time (its workspace is
 *    shared by all calls on it).
 */
#ifndef ACESPEC_H
#define ACESPEC_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ACESPEC_OK = 0,
  ACESPEC_EINVAL = -1,        /* bad argument (null pointer, size out of range, ...)   */
  ACESPEC_EUNSUPPORTED = -2,  /* valid but not supported by these kernels            */
  ACESPEC_ENOMEM = -3,        /* workspace allocation failed in acespec_create        */
  ACESPEC_EHIP = -4,          /* a HIP runtime call failed                            */
  ACESPEC_EBADTREE = -5,      /* per-session status only: malformed tree or prefix    */
  ACESPEC_EBADDRAFT = -6,     /* per-session status only: NaN/inf/negative draft data  */
  ACESPEC_ENONFINITE = -7     /* per-session status only: non-finite target logits     */
} acespec_status;

typedef enum { ACESPEC_F32 = 0, ACESPEC_BF16 = 1 } acespec_dtype;

/* Decoder shape.  The paper names only the model families (Qwen, LLaMA; Section V-A);
 * the reading implemented is a Llama-style pre-norm decoder: RMSNorm with gains,
 * rotate-half RoPE (theta_i = rope_base^(-2i/head_dim)), grouped-query attention with
 * scale 1/sqrt(head_dim), SwiGLU MLP, no biases, untied LM head.
 * Supported: head_dim in {64, 128}; n_heads % n_kv_heads == 0;
 * d_model, n_heads*head_dim and d_ff multiples of 64; vocab a multiple of 4. */
typedef struct {
  int n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff, vocab;
  float rope_base;   /* e.g. 10000 */
  float rms_eps;     /* e.g. 1e-5  */
  acespec_dtype dtype;  /* weights, activations between kernels and KV cache */
} acespec_model_desc;

/* Per-layer weights, all in the model dtype, row-major [out, in] (K contiguous). */
typedef struct {
  const void *attn_norm;   /* [d_model]                                              */
  const void *wqkv;        /* [(n_heads + 2 n_kv_heads) head_dim, d_model]: q, k, v rows */
  const void *wo;          /* [d_model, n_heads head_dim]                             */
  const void *mlp_norm;    /* [d_model]                                               */
  const void *w_gate_up;   /* [2 d_ff, d_model]: gate rows then up rows                */
  const void *w_down;      /* [d_model, d_ff]                                         */
} acespec_layer_weights;

/* Storage of the dense matrices of a bf16 model (wqkv, wo, w_gate_up, w_down, lm_head).
 * The embedding and the RMSNorm gains are always row-major in the model dtype. */
typedef enum {
  ACESPEC_LAYOUT_ROWS = 0,    /* bf16, row-major [out, in] as above                       */
  ACESPEC_LAYOUT_PACKED = 1   /* fp16 in the fragment order of acespec_pack_weight (same
                                 size); bf16 models only, vocab a multiple of 16           */
} acespec_layout;

typedef struct {
  const void *embed;                     /* [vocab, d_model]                           */
  const acespec_layer_weights *layers;   /* HOST array of n_layers entries              */
  const void *final_norm;                /* [d_model]                                  */
  const void *lm_head;                   /* [vocab, d_model]                           */
  acespec_layout layout;                 /* of the dense matrices; 0 = row-major        */
} acespec_weights;

/* KV cache, in the model dtype.  Keys: k [n_layers][B][n_kv_heads][capacity][head_dim],
 * stored after RoPE.  Values are head-dim-major: v [n_layers][B][n_kv_heads][head_dim]
 * [capacity] (slot s of a head is column s), so that the attention's contraction over
 * slots reads contiguous memory.  Slots [0, prefix_len[b]) hold session b's verified
 * context and are only read.  The verify call writes the tree's keys and values into
 * slots prefix_len[b] + r for tree rows r = 0..N (nothing is committed: calling again
 * with the same inputs gives the same result). */
typedef struct {
  void *k, *v;
  int capacity;                 /* slots per (layer, session, kv head); multiple of 64 */
  const int32_t *prefix_len;    /* [B] DEVICE; needs prefix_len[b] + N + 1 <= capacity */
} acespec_kv_cache;

/* Target sampling parameters (Section III-B: nucleus sampling on the target side). */
typedef struct {
  float temperature;   /* > 0: logits are divided by it                               */
  float top_p;         /* (0, 1]: smallest most-probable set reaching this mass        */
  int top_k;           /* 1..256 and <= vocab: size of the sparse downlink payload     */
} acespec_params;

/* Caller-allocated device outputs.  Row counts: B*(N+1) rows for verify_tree (row 0 of
 * each session is the root), R rows for verify_tail. */
typedef struct {
  uint8_t *accept;          /* [rows] 1 if the row's token is accepted by its parent's
                               distribution (root rows: 1)                             */
  int32_t *acc_prefix_len;  /* [rows] leading accepted nodes on the root-to-row path  */
  int32_t *resample_token;  /* [rows] residual inverse-CDF sample (root rows: -1)     */
  int32_t *bonus_token;     /* [rows] sample from the row's own target distribution   */
  int32_t *topk_ids;        /* [rows, top_k] most probable first                      */
  float   *topk_probs;      /* [rows, top_k] renormalised over the k ids (0 outside
                               the top-p nucleus)                                     */
  int32_t *path;            /* [B, N+1] kept drafted rows root-first, -1 padded       */
  int32_t *path_len;        /* [B] drafted tokens kept                                */
  int32_t *next_token;      /* [B] token emitted after the kept path                  */
  uint8_t *sibling_hit;     /* [B] 1 if the walk continued through a drafted sibling */
  int32_t *status;          /* [B] ACESPEC_OK, or EBADTREE / EBADDRAFT / ENONFINITE   */
  float   *logits_out;      /* optional [rows, vocab] fp32 logits; NULL = not kept    */
} acespec_outputs;

typedef struct acespec_ctx acespec_ctx;

/* Creates a context on the current HIP device and allocates its workspace for up to
 * max_batch sessions of up to max_nodes drafted nodes (max_nodes <= 64), i.e.
 * max_batch*(max_nodes+1) rows.  The same bound limits verify_tail's row count.
 * Returns ACESPEC_OK and *out, or an error (ENOMEM if the workspace does not fit). */
int acespec_create(const acespec_model_desc *desc, int max_batch, int max_nodes,
                   acespec_ctx **out);

/* Frees the workspace (synchronises the device first).  NULL is accepted. */
void acespec_destroy(acespec_ctx *ctx);

/* One verify step over B drafted trees of N drafted nodes each.
 *  tree_tokens [B, N+1] int32: row 0 is the root (the last committed token, not yet in
 *                the cache), rows 1..N the drafted tokens.
 *  parent_idx  [B, N+1] int32: parent_idx[b,0] = -1 and 0 <= parent_idx[b,r] < r.
 *                The lowest-index child of a row is its main-chain child.
 *  draft_q     [B, N+1, vocab] fp32: row r holds the draft distribution that proposed
 *                r's children; only rows with children are read.
 *  uniforms    [B, N+1, 3] fp32 in (0, 1): per row (accept, residual, bonus).
 * Writes every field of *outs (logits_out only if non-NULL). */
int acespec_verify_tree(acespec_ctx *ctx, const acespec_weights *weights,
                        const acespec_kv_cache *kv, const int32_t *tree_tokens,
                        const int32_t *parent_idx, const float *draft_q,
                        const float *uniforms, int B, int N, const acespec_params *params,
                        const acespec_outputs *outs, hipStream_t stream);

/* The same step for the paper's own uplink (Section III-B, Algorithm 1: the edge sends
 * the drafted tokens and a compressed draft distribution; the cloud does no resampling of
 * its own and returns the rejection index with a sparse target distribution):
 *  q_hat [B, N+1] fp32: q_hat[b, r] = the draft probability of row r's own token under
 *                its parent's draft distribution (row 0 unused) -- one float per node
 *                instead of a vocabulary-sized row.
 * Per row: accept (u[.., 0] * q_hat < p), acc_prefix_len, topk_ids / topk_probs as in
 * acespec_verify_tree; resample_token = bonus_token = -1 (no cloud-side sampling).
 * Per session: path / path_len along accepted main children (no sibling hits: they need
 * the resample token), next_token = -1, sibling_hit = 0.  The edge resamples from the
 * top-k payload of row path_len (acc. position) against its own draft distribution;
 * that is exact only where the payload covers the target's nucleus. */
int acespec_verify_tree_scalar_q(acespec_ctx *ctx, const acespec_weights *weights,
                                 const acespec_kv_cache *kv, const int32_t *tree_tokens,
                                 const int32_t *parent_idx, const float *q_hat,
                                 const float *uniforms, int B, int N,
                                 const acespec_params *params, const acespec_outputs *outs,
                                 hipStream_t stream);

/* LM head and verification only, over R given hidden states (the last stage of
 * verify_tree on its own).  Each row r is the parent of one drafted token
 * draft_tokens[r]; rows form chains of chain_len consecutive rows (R % chain_len == 0).
 *  lm_head [vocab, d_model] in the layout lm_head_layout (ACESPEC_LAYOUT_PACKED: as
 *          written by acespec_pack_weight, for bf16 models with vocab a multiple of 16;
 *          another value: ACESPEC_EINVAL, a packed head otherwise ACESPEC_EUNSUPPORTED),
 *  final_norm [d_model] or NULL (no normalisation),
 *  hidden [R, d_model] in the model dtype, draft_q [R, vocab], uniforms [R, 3].
 * Per row: accept, resample_token, bonus_token, topk_*, acc_prefix_len (leading accepts
 * within its chain, counting the row).  Per chain c: path_len[c] = leading accepts,
 * path[c, 0..chain_len) = kept row indices within the chain (-1 padded),
 * next_token[c] = resample at the first rejected row, or -1 when the whole chain is
 * accepted (the bonus then needs the row after the chain); sibling_hit[c] = 0;
 * status[c] = OK, EBADTREE (a draft token outside the vocabulary), or EBADDRAFT /
 * ENONFINITE for a row of the chain (without final_norm, hidden values beyond the fp16
 * range of a bf16 model overflow and give ENONFINITE).  path is [R/chain_len, chain_len]. */
int acespec_verify_tail(acespec_ctx *ctx, const void *lm_head, acespec_layout lm_head_layout,
                        const void *final_norm, const void *hidden, const int32_t *draft_tokens,
                        const float *draft_q, const float *uniforms, int R, int chain_len,
                        const acespec_params *params, const acespec_outputs *outs,
                        hipStream_t stream);

/* acespec_verify_tail without a context, for callers that cannot allocate device memory
 * at all (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same kernels and results as acespec_verify_tail, the intermediate data
 * in a fixed device array of the library (48 MiB per device, held from the first call on
 * that device until the process ends).  Nothing is allocated, by this call or at set-up.
 *  desc: the model (only dtype, d_model, vocab and rms_eps are read).
 *  outs->logits_out is REQUIRED: the fp32 logits [R, vocab] are written there.
 * R is limited by the array: R * (4 + 4 ceil(vocab / 128) + d_model * 2) bytes (d_model * 4
 * for an fp32 model with a final norm; no d_model term for an fp32 model without one) must
 * fit in 48 MiB, else ACESPEC_EINVAL before anything is launched (e.g. R <= 4096 at
 * d_model 4096, vocab 128256).  The LM head is never sliced along K here (where
 * acespec_verify_tail slices it, the logits differ in the order of their fp32 sums).
 * All calls on one device share the array: two calls that overlap in time on the same
 * device race (serialise them, e.g. on one stream).  Every byte a call reads from the
 * array it has written first, so no clearing is needed between calls. */
int acespec_verify_tail_noalloc(const acespec_model_desc *desc, const void *lm_head,
                                acespec_layout lm_head_layout, const void *final_norm,
                                const void *hidden,
                                const int32_t *draft_tokens, const float *draft_q,
                                const float *uniforms, int R, int chain_len,
                                const acespec_params *params, const acespec_outputs *outs,
                                hipStream_t stream);

/* Commits the accepted path of every session into its KV cache (Algorithm 1, the
 * cloud's COMPACT_KV after RECEIVE_WAIT: only the state of the kept prefix survives a
 * verify round).  Inputs are a verify_tree call's outputs over the same cache:
 *  path [B, N+1], path_len [B]: the kept drafted rows root-first (outs->path, path_len);
 *  status [B] or NULL: sessions whose status is not ACESPEC_OK are not committed.
 * For every layer and kv head, the keys and values of row 0 (the root) and of the kept
 * rows path[b, 0 .. path_len[b]) move from slots prefix_len[b] + row to the contiguous
 * slots prefix_len[b] + 0 .. prefix_len[b] + path_len[b] -- the slots a causal decode of
 * the accepted tokens fills, since a kept node at depth i sits at RoPE position
 * prefix_len[b] + i.  Slots below prefix_len[b] are not touched; the tree slots past the
 * new end keep stale entries.
 *  new_prefix_len [B] DEVICE output: prefix_len[b] + 1 + path_len[b], or -1 for a session
 *  that was not committed (bad status, prefix_len + N + 1 > capacity, path_len outside
 *  [0, N] or a kept row outside [1, N]); nothing of such a session is moved.  It must not
 *  overlap kv->prefix_len (every workgroup of a session reads prefix_len[b] while one of
 *  them writes new_prefix_len[b]): an overlapping pair returns ACESPEC_EINVAL before
 *  anything is launched.  Copy new_prefix_len into prefix_len after the call instead.
 * The next round's root is the verify step's next_token (not yet in the cache). */
int acespec_commit_kv(acespec_ctx *ctx, const acespec_kv_cache *kv, const int32_t *path,
                      const int32_t *path_len, const int32_t *status, int B, int N,
                      int32_t *new_prefix_len, hipStream_t stream);

/* Re-lays one row-major bf16 weight matrix [rows, cols] (rows % 16 == 0, cols % 32 == 0)
 * out into the packed layout (ACESPEC_LAYOUT_PACKED): for every 16-row block and 32-column
 * step, the 1 KB operand of one 16x16x32 matrix-core instruction, contiguous, its values
 * widened to fp16.  The packed matrix holds the operands the verify pass multiplies by
 * anyway (the row-major path widens each bf16 weight to fp16 the same way before its
 * products, so the two layouts differ at most in how a product's k-slices are summed in
 * fp32); packed, each wave of the GEMMs loads its weight operands straight into
 * registers, and only the activations pass through LDS.  Weights
 * beyond the fp16 range (|w| > 65504) become +-inf, as they do on the row-major path.
 * Not part of the verify step: a caller packs its weights once (e.g. at load time).
 *  src [rows, cols] bf16, dst rows*cols*2 bytes; both DEVICE, caller-owned, no overlap.
 * Enqueued on stream; ACESPEC_EINVAL for a NULL pointer or a shape outside the above. */
int acespec_pack_weight(const void *src, void *dst, int rows, int cols, hipStream_t stream);

/* Value-cache layout conversion, for callers that keep values slot-major like the keys
 * (v[planes][capacity][head_dim], slot s of a head is row s): the verify step reads the
 * head-dim-major layout of acespec_kv_cache (v[planes][head_dim][capacity]), in which the
 * attention's sum over slots (Section III-C) streams contiguous memory.  Not part of the
 * verify step: a caller converts a session's prefix once when it loads it, and converts
 * back when it needs slot-major values again.
 *  planes     = n_layers * B * n_kv_heads (the leading dimensions, same order in both),
 *  capacity   slots per plane, a positive multiple of 64 (as in acespec_kv_cache),
 *  head_dim   >= 1,  dtype: ACESPEC_BF16 or ACESPEC_F32 (element size 2 or 4 bytes),
 *  direction  ACESPEC_V_TO_HEAD_DIM_MAJOR (src slot-major) or ACESPEC_V_TO_SLOT_MAJOR
 *             (src head-dim-major, the inverse),
 *  src, dst   DEVICE, caller-owned, planes*capacity*head_dim elements each, no overlap.
 * Values are copied bit for bit.  Enqueued on stream; ACESPEC_EINVAL (nothing launched)
 * for a NULL pointer, overlap, an unknown dtype or direction, a size outside the above,
 * or more than 2^31 - 1 tiles of 32 x 32 (convert in parts). */
typedef enum { ACESPEC_V_TO_HEAD_DIM_MAJOR = 0, ACESPEC_V_TO_SLOT_MAJOR = 1 } acespec_v_direction;
int acespec_convert_v_cache(const void *src, void *dst, int planes, int capacity, int head_dim,
                            acespec_dtype dtype, acespec_v_direction direction,
                            hipStream_t stream);

/* ---- The KV cache in 4 bits -------------------------------------------------------------
 * Slots are held in blocks of 32.  A group is 32 consecutive head dims of one key, or the 32
 * slots of a block for one head dim of the values; its elements are e2m1 values (0, 1/2, 1,
 * 3/2, 2, 3, 4, 6 and their negatives) times one power of two 2^e.  With top the group's
 * largest magnitude, e = floor(log2 top) - 2, one more if top >= 1.75 * 2^floor(log2 top), and
 * at least -13; an element is held as the nearest such value (ties to the even code), so it is
 * off by at most 2^e.  A group with a NaN, an infinity or a magnitude of 57344 or more (fp16
 * could not hold it) is marked instead, and all 32 elements read as NaN.
 *  blocks  [n_layers][B][n_kv_heads][capacity / 32] records of 34 * head_dim bytes (17/32
 *          byte an element).  A record's inner order is that of the attention's matrix
 *          operands; acespec_quantize_kv and acespec_commit_kv_quant write it,
 *          acespec_dequantize_kv reads it back.
 *  tail_k, tail_v  the slots of the last, incomplete block and behind them the tree's rows,
 *          in the model dtype: [n_layers][B][n_kv_heads][tail_capacity][head_dim] and
 *          [..][head_dim][tail_capacity], as in acespec_kv_cache.
 * A session of P = prefix_len[b] slots holds slots [0, P / 32 * 32) in blocks, slot
 * P / 32 * 32 + i in tail slot i (i < P % 32), and tree row r in tail slot P % 32 + r.
 * P % 32 = 0 leaves no slot in the tail, and P may be 0.  blocks, tail_k and tail_v do not
 * overlap (ACESPEC_EINVAL from every call below). */
typedef struct {
  void *blocks;
  void *tail_k, *tail_v;
  int capacity;                 /* slots in blocks; a positive multiple of 32.  Launches are
                                   chosen by it: one far above the prefixes costs time    */
  int tail_capacity;            /* a multiple of 64; at least 31 + N + 1 where a tree of N
                                   drafted nodes is verified or committed               */
  const int32_t *prefix_len;    /* [B] DEVICE; at most capacity + 31                     */
} acespec_kv_quant;

/* Which positions a row at position p attends to, besides the tree mask: with window > 0
 * those in (p - window, p] and those below sinks (the first tokens, which stay visible);
 * window 0: all, whatever sinks is.  Positions are not renumbered: keys keep the rotation of
 * their own position.  A row always sees itself.  A NULL span is {0, 0}. */
typedef struct {
  int window;   /* >= 0 */
  int sinks;    /* >= 0 */
} acespec_attn_span;

/* Brings a cache to 4 bits (the model's dtype, shapes of ctx): of every session the complete
 * blocks of slots [0, prefix_len[b]), and the prefix_len[b] % 32 slots behind them copied into
 * the tail.  prefix_len is kv's; qc's is not read (it may be NULL).
 *  first [B] DEVICE or NULL: slots below first[b] are taken to be held already, and blocks
 *          that lie wholly below it are left alone (for prefixes that grew: quantise what was
 *          appended).
 *  status [B] DEVICE or NULL: ACESPEC_OK, or ACESPEC_EBADTREE for a session with
 *          prefix_len[b] outside [0, kv->capacity], beyond qc->capacity + 31, or first[b]
 *          outside [0, prefix_len[b]]; nothing of such a session is written.
 * kv->capacity is a multiple of 64; k, v, blocks and the tails are 16-byte aligned.  They do not
 * overlap, and what the call writes overlaps nothing else that it reads or writes.  Enqueued on
 * stream; ACESPEC_EINVAL before anything is launched for arguments outside the above. */
int acespec_quantize_kv(acespec_ctx *ctx, const acespec_kv_cache *kv, const acespec_kv_quant *qc,
                        const int32_t *first, int B, int32_t *status, hipStream_t stream);

/* Reads a cache in 4 bits back into one of the model's dtype: slots [first[b] / 32 * 32,
 * prefix_len[b]) of every session (prefix_len: qc's; kv's is not read).  The elements' values
 * are exact in bf16 and fp32.  Slots from prefix_len[b] on are left as they were.  first,
 * status and the rest as above. */
int acespec_dequantize_kv(acespec_ctx *ctx, const acespec_kv_quant *qc, const acespec_kv_cache *kv,
                          const int32_t *first, int B, int32_t *status, hipStream_t stream);

/* Tree attention of one layer over a cache in 4 bits: row r of session b, at position
 * prefix_len[b] + depth(r), attends to the prefix, its ancestors and itself, as far as span
 * shows them, with scale 1/sqrt(head_dim).
 *  layer   in [0, n_layers) of ctx's model,
 *  q, out  [B, N+1, n_heads, head_dim] in the model dtype, q rotated; 16-byte aligned.  out and
 *          status overlap nothing else that is given (ACESPEC_EINVAL).  Tail slots
 *          prefix_len[b] % 32 + r hold the keys (rotated) and values of the tree's rows.  A
 *          decode of single tokens is N = 0.
 *  parent_idx [B, N+1] as in acespec_verify_tree,
 *  status [B]: ACESPEC_OK or ACESPEC_EBADTREE (parents, or prefix_len outside
 *          [0, capacity + 31]).
 * A bf16 model multiplies in fp16 with fp32 sums: queries, and keys and values of the tail,
 * beyond its range (65504) count as infinite, and softmax weights below 2^-25 of a row's largest
 * may count as 0.  A NaN or an infinity among the keys and values
 * reaches the rows that attend to its slot and no others. */
int acespec_attention_quant(acespec_ctx *ctx, const acespec_kv_quant *qc, int layer,
                            const acespec_attn_span *span, const void *q,
                            const int32_t *parent_idx, int B, int N, void *out, int32_t *status,
                            hipStream_t stream);

/* acespec_verify_tree, or with q_hat in draft_q's place acespec_verify_tree_scalar_q, over a
 * cache in 4 bits (exactly one of draft_q and q_hat is given).  The tree's keys and values are
 * written to its tail in the model dtype and attended to unrounded; nothing is committed.  A
 * bf16 model's rotated queries are fp16, as in acespec_verify_tree; against blocks each is held
 * exactly, or, below 1/64 of the largest in its 32 head dims, to 2^-17 of that. */
int acespec_verify_tree_quant(acespec_ctx *ctx, const acespec_weights *weights,
                              const acespec_kv_quant *qc, const acespec_attn_span *span,
                              const int32_t *tree_tokens, const int32_t *parent_idx,
                              const float *draft_q, const float *q_hat, const float *uniforms,
                              int B, int N, const acespec_params *params,
                              const acespec_outputs *outs, hipStream_t stream);

/* acespec_commit_kv over a cache in 4 bits: the root and the kept rows join the tail's
 * committed slots, every 32 of which become a block; the rest move to the tail's front.  Tail
 * slots past them keep stale entries.  Arguments and new_prefix_len as in acespec_commit_kv, none
 * of them inside blocks or the tails (ACESPEC_EINVAL); a session is not committed (-1, nothing
 * moved) also where its new blocks do not fit capacity. */
int acespec_commit_kv_quant(acespec_ctx *ctx, const acespec_kv_quant *qc, const int32_t *path,
                            const int32_t *path_len, const int32_t *status, int B, int N,
                            int32_t *new_prefix_len, hipStream_t stream);

/* ---- Sessions behind shared prefixes ----------------------------------------------------
 * Prefixes that several sessions of a batch have in common (a system prompt, a document, the
 * prompt of several samples) are held once, apart from the sessions' own caches.  A bf16 model's
 * larger batches attend to them once for all rows of the sessions behind them; where that takes
 * longer (few rows or few slots, by the capacities of store and cache), and in an fp32 model, each
 * session reads its prefix for itself.  Caches in 4 bits (above) stand behind no shared prefix and
 * take no norms.  A session behind a prefix of n slots that has P
 * own slots in its acespec_kv_cache (prefix_len[b] = P) is at position n + P; own slot i is
 * position n + i, and tree row r writes slot P + r.  acespec_commit_kv serves the own cache as it
 * is.
 *  blocks  [n_layers][prefixes][n_kv_heads][capacity / 64] records of 128 * head_dim elements, in
 *          fp16 for a bf16 model (as in the verify step a value beyond its range counts as
 *          infinite, and one below 2^-14 keeps multiples of 2^-24 only) and in fp32 for an fp32 model.  A record holds 64 slots' keys and values in the
 *          order of the attention's matrix operands; acespec_share_prefix writes it.
 *  len     [prefixes] slots held, in [0, capacity]; what lies behind them is not read as numbers.
 * One prefix and kv head takes less than 2 GiB (ACESPEC_EUNSUPPORTED otherwise). */
typedef struct {
  void *blocks;
  int prefixes;                 /* >= 1                                                  */
  int capacity;                 /* slots of each; a positive multiple of 64              */
  const int32_t *len;           /* [prefixes] DEVICE                                     */
} acespec_kv_shared;

/* Gains [head_dim] in the model dtype, 16-byte aligned, of the RMSNorm (eps: the model's rms_eps)
 * that each query head and each key head passes before its rotation; NULL: no norm there. */
typedef struct {
  const void *q_gain, *k_gain;
} acespec_qk_norm;

/* The calls of this section take arrays that are 16-byte aligned (the caches, blocks, q, qkv, out)
 * and, for what one of them writes, apart from everything else that it is given (ACESPEC_EINVAL;
 * weights aside), for at most 65535 sessions with trees.
 * prefix_of [B] DEVICE: the prefix that session b stands behind, or -1.  Any number of sessions may
 * stand behind one, in any order.  status[b] is ACESPEC_EBADTREE for a malformed tree, a prefix_of
 * outside [-1, prefixes), a len outside [0, capacity] or a prefix_len that leaves no room. */

/* Takes sessions' first slots over into the store.  from [prefixes] DEVICE: the session of kv (of
 * B) whose slots [0, count[p]) become prefix p, or -1: p is left as it is; count DEVICE, NULL: all
 * prefix_len of them.  Behind the last slot its record is zeroed; later records are left as they
 * were.  new_len [prefixes] DEVICE output: the slots of each prefix now (for -1 len[p]), or -1 for
 * one that was refused (from outside [-1, B), count outside [0, prefix_len] or beyond capacity),
 * of which nothing is written.  Copy it into len after the call. */
int acespec_share_prefix(acespec_ctx *ctx, const acespec_kv_cache *kv, int B,
                         const acespec_kv_shared *sh, const int32_t *from, const int32_t *count,
                         int32_t *new_len, hipStream_t stream);

/* Tree attention of one layer: row r of session b attends to its shared prefix, its own slots, its
 * ancestors and itself, with scale 1/sqrt(head_dim).  q (rotated), out [B, N+1, n_heads, head_dim]
 * in the model dtype; own slots prefix_len[b] + r hold the tree rows' keys and values.  A decode of
 * single tokens is N = 0.  A bf16 model multiplies in fp16 with fp32 sums.  A NaN or an infinity
 * among the keys and values reaches the rows that attend to its slot and no others. */
int acespec_attention_shared(acespec_ctx *ctx, const acespec_kv_shared *sh, const int32_t *prefix_of,
                             const acespec_kv_cache *kv, int layer, const void *q,
                             const int32_t *parent_idx, int B, int N, void *out, int32_t *status,
                             hipStream_t stream);

/* From one layer's projection qkv [B, N+1, (n_heads + 2 n_kv_heads) head_dim] (model dtype; heads
 * of q, k, v) in one pass: every query and key head normalised as norm says and rotated to its
 * row's position (prefix, own slots and depth in the tree), q [B, N+1, n_heads, head_dim] written,
 * and the keys and values into slots prefix_len[b] + r of kv's layer.  Sines and cosines are
 * evaluated in 32 bits of an angle that is reduced in 64 (off by 2^-23; the verify step's are
 * rounded from 64 bits, so that the two may differ in a last bit).  sh and prefix_of may be NULL
 * (both): no session stands behind a prefix.  Nothing of a session with a bad status is written. */
int acespec_qk_norm_rope(acespec_ctx *ctx, const acespec_qk_norm *norm, const acespec_kv_shared *sh,
                         const int32_t *prefix_of, const acespec_kv_cache *kv, int layer,
                         const void *qkv, const int32_t *parent_idx, int B, int N, void *q,
                         int32_t *status, hipStream_t stream);

/* acespec_verify_tree, or with q_hat in draft_q's place acespec_verify_tree_scalar_q, for sessions
 * behind shared prefixes, for a decoder whose query and key heads are normalised, or for both.
 *  norms  HOST array of n_layers entries, or NULL: no norms,
 *  sh, prefix_of  both, or both NULL: no shared prefixes. */
int acespec_verify_tree_shared(acespec_ctx *ctx, const acespec_weights *weights,
                               const acespec_qk_norm *norms, const acespec_kv_shared *sh,
                               const int32_t *prefix_of, const acespec_kv_cache *kv,
                               const int32_t *tree_tokens, const int32_t *parent_idx,
                               const float *draft_q, const float *q_hat, const float *uniforms,
                               int B, int N, const acespec_params *params,
                               const acespec_outputs *outs, hipStream_t stream);

/* Sessions take over others' slots (a beam that goes on twice, samples of one session, a batch that
 * closes its gaps, the rest of sessions whose front became a shared prefix): session b of dst gets
 * slots [first[b], prefix_len) of session from[b] of src, as its slots from 0 on, in all layers;
 * what lies behind them is left as it was.  from[b] = -1: session b stays as it is.  first NULL: 0.
 *  src, dst  caches of src_batch and dst_batch sessions (each at most max_batch) that lie apart,
 *          or one and the same (k, v, capacity and batch equal), where a session that receives
 *          another's slots is no session's source, and one that is its own source (from[b] = b)
 *          stays as it is.
 *  new_prefix_len [dst_batch] DEVICE output: the session's slots now (for -1 dst's prefix_len), or
 *          -1 for one that was refused (from, first or the lengths out of range, no room, or a
 *          source that itself receives), of which nothing is written. */
int acespec_fork_kv(acespec_ctx *ctx, const acespec_kv_cache *src, int src_batch,
                    const acespec_kv_cache *dst, int dst_batch, const int32_t *from,
                    const int32_t *first, int32_t *new_prefix_len, hipStream_t stream);

/* Message for the last non-OK return on this thread ("" if none). */
const char *acespec_last_error(void);

/* Per-kernel timing with HIP events recorded on the launch stream around every
 * kernel.  enable != 0 turns it on for subsequent calls.  acespec_timing_read waits
 * for the recorded events, returns per-kernel-kind totals accumulated since the last
 * read (names[i], total_ms[i], launches[i] for i < returned count, at most max
 * entries) and clears them.  names point to static strings. */
int acespec_timing_enable(acespec_ctx *ctx, int enable);
int acespec_timing_read(acespec_ctx *ctx, const char **names, double *total_ms,
                        int *launches, int max);
/* Restricts the timing events to the kernels of one kind (a name acespec_timing_read
 * reports, e.g. "gemm_gate_up"); NULL restores every kind.  Each timed launch adds two
 * event records to the stream, so timing one kind keeps the cost to the measured step
 * small.  Unknown names return ACESPEC_EINVAL and leave the selection unchanged. */
int acespec_timing_only(acespec_ctx *ctx, const char *kind);

#ifdef __cplusplus
}
#endif
#endif /* ACESPEC_H */
