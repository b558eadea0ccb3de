/*
 * gm.h -- C ABI of the batched speculative-decoding step (MI355X / gfx950).
 *
 * One step of speculative rollout generation for a batch of B sequences
 * (GrowMTP, Sec. 2.2): the target verifies a block of k+1 positions per
 * sequence in one forward (gm_verify_forward, gm_verify_attention), accepts a
 * prefix of the k drafts and draws one more token (gm_spec_accept), commits
 * the accepted KV entries and rolls back the rest (gm_kv_commit), and the MTP
 * draft head proposes the next block (gm_mtp_draft).  Beside the chain stand
 * the operators of draft trees (gm_kv_append, gm_tree_*) and of token
 * log-probabilities (gm_token_logprobs and its gradient).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Pointers are DEVICE pointers unless a comment says "host".  Every buffer
 *   is owned by the caller; no call keeps a pointer after it returns and no
 *   call allocates or frees device memory.  Scratch memory is passed in as a
 *   workspace whose size gm_workspace_size() reports.
 * - Every call enqueues its kernels on `stream` (a hipStream_t; NULL is the
 *   null stream) and returns without waiting for them.
 * - Shapes and arguments are validated on the host before anything is
 *   launched; a failed check returns a negative gm_status, launches nothing
 *   and leaves a message for gm_last_error().  Faults that only the device
 *   can see (a token id outside the vocabulary, a block-table entry outside
 *   the page pool) are reported through the optional `dev_err` word: the
 *   kernel ORs a GM_DEVERR_* bit into it and skips the offending access.
 * - Outputs are bit-deterministic for fixed inputs (no reduction depends on
 *   the order of atomics).
 * - Token ids are int32.  Logits, uniforms and hidden states are float32.
 *   Weights and KV entries use the model dtype: GM_F32 (float) or GM_BF16
 *   (bfloat16 stored as uint16).  Norm weights use the model dtype too.
 * - Block layout: block position i of sequence b (0 <= i <= k) is absolute
 *   position m_b + i, where m_b = seq_lens[b] is the committed length; the
 *   block is [t_m, d_1 .. d_k]: the pending token (drawn by the last cycle,
 *   not yet in the cache) followed by the k drafts.
 */
#ifndef GM_H
#define GM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GM_OK = 0,
  GM_ERR_INVALID_ARG = -1,   /* null pointer, bad size or shape */
  GM_ERR_UNSUPPORTED = -2,   /* a valid configuration this build does not implement */
  GM_ERR_CAPACITY = -3,      /* the KV page table cannot hold the positions the call writes */
  GM_ERR_WORKSPACE = -4,     /* workspace missing or smaller than gm_workspace_size() */
  GM_ERR_DEVICE = -5         /* a HIP runtime call failed */
} gm_status;

enum { GM_DEVERR_TOKEN = 1, GM_DEVERR_PAGE = 2, GM_DEVERR_TREE = 4 };

typedef enum { GM_F32 = 0, GM_BF16 = 1 } gm_dtype;
typedef enum { GM_GREEDY = 0, GM_SAMPLE = 1 } gm_accept_mode;
typedef enum {
  GM_OP_VERIFY_FORWARD = 0,
  GM_OP_VERIFY_ATTENTION = 1,
  GM_OP_SPEC_ACCEPT = 2,
  GM_OP_MTP_DRAFT = 3,
  GM_OP_DCA_LOSS = 4,    /* B = cycles N, k = draft length K, cfg->vocab = V */
  GM_OP_MTP_RECONSTRUCT = 5,  /* B = cycles R, k = depth K, max_ctx = the cache's max_ctx */
  GM_OP_TREE_ATTENTION = 6,   /* k = nodes N of a tree, 1..64 */
  GM_OP_TOKEN_LOGPROBS = 7    /* B = rows M, k = topk, cfg->vocab = V */
} gm_op;

/* Decoder shape: pre-norm RMSNorm / RoPE (rotate-half, angle pos * base^(-2i/d))
 * / grouped-query attention / SwiGLU, the layer of the paper's backbones
 * (App. "Models and Draft Heads").  Limits of this build: head_dim 128 for
 * GM_BF16 (64 or 128 for GM_F32), n_heads a multiple of n_kv_heads with
 * (n_heads / n_kv_heads) * (k + 1) <= 64, hidden and ffn multiples of 64,
 * hidden and (n_heads + 2 n_kv_heads) * head_dim at most 16384, vocab at
 * most 524288 (also the limit of gm_spec_accept's V);
 * GM_BF16 needs vocab a multiple of 128 and hidden, ffn and
 * n_heads * head_dim multiples of 256. */
typedef struct {
  int n_layers, hidden, n_heads, n_kv_heads, head_dim, ffn, vocab;
  float rope_base;       /* 10000 */
  float rms_eps;         /* 1e-6 */
  int dtype;             /* gm_dtype */
  int qk_norm;           /* 1: per-head RMSNorm of q and k before RoPE (Qwen3) */
  int tie_embed;         /* informational: lm_head may alias embed */
} gm_model_config;

/* One decoder layer.  A linear weight W[out][in] (y = W x) is stored
 *  - GM_F32: row-major;
 *  - GM_BF16: tiled, in tiles of 16 rows x 32 columns (out a multiple of 128):
 *    element (n, c) at
 *      (((n / 128) * (in / 32) + c / 32) * 8 + (n / 16) % 8) * 512
 *        + ((c % 32) / 8) * 128 + (n % 16) * 8 + c % 8,
 *    so that each 1 KiB tile is read by one 16-byte-per-lane load of a
 *    64-lane wave in the operand order of the matrix cores, and the tiles of
 *    8 consecutive 16-row strips at one 32-column step are consecutive (the
 *    strips streamed together are one contiguous run per step).  (Row-major W
 *    converts to this layout by viewing it as [out/128][8][16][in/32][4][8]
 *    and permuting to [out/128][in/32][8][4][16][8].)
 * The tiled layout applies to w_qkv, w_o, w_gate_up, w_down, the MTP w_proj
 * and lm_head; embeddings and norm weights are plain vectors / row-major. */
typedef struct {
  const void *attn_norm;  /* [H] */
  const void *w_qkv;      /* [(n_heads + 2 n_kv_heads) head_dim, H]: the rows of W_q, then W_k, then W_v */
  const void *q_norm;     /* [head_dim], or NULL when qk_norm == 0 */
  const void *k_norm;     /* [head_dim], or NULL when qk_norm == 0 */
  const void *w_o;        /* [H, n_heads head_dim] */
  const void *ffn_norm;   /* [H] */
  const void *w_gate_up;  /* [2 ffn, H]: the rows of W_gate, then W_up */
  const void *w_down;     /* [H, ffn] */
} gm_layer_weights;

typedef struct {
  const void *embed;                /* [vocab, H] */
  const void *final_norm;           /* [H] */
  const void *lm_head;              /* [vocab, H] */
  const gm_layer_weights *layers;   /* host array [n_layers] */
} gm_model_weights;

/* The recurrent MTP draft head (App. "Models and Draft Heads"): RMSNorm_h of
 * the conditioning hidden and RMSNorm_e of the token embedding, concatenated
 * hidden first, a bias-free projection 2H -> H, one decoder layer with a KV
 * cache of its own, a final RMSNorm and the backbone's LM head. */
typedef struct {
  const void *norm_h;      /* [H] */
  const void *norm_e;      /* [H] */
  const void *w_proj;      /* [H, 2H]: columns 0..H-1 act on RMSNorm_h(h), H..2H-1 on RMSNorm_e(E[t]) */
  const void *final_norm;  /* [H] */
  gm_layer_weights layer;
} gm_mtp_weights;

/* Paged KV cache.  Each layer owns two page pools, K and V, each
 * [num_pages][n_kv_heads][page_size * head_dim] elements of the model dtype.
 * Position t of sequence b lives in page block_table[b][t / page_size] at
 * offset t % page_size.  Inside the block of one (page, kv head) the tokens
 * come in tiles of 16 (tile j holds offsets 16j .. 16j+15) of 16 * head_dim
 * elements, and inside a tile (token s = 0..15, channel c = 0..head_dim-1):
 *   K element at  (c / 32) * 512 + ((c % 32) / 8) * 128 + s * 8 + c % 8
 *   V element at  (c / 32) * 512 + (s / 4) * 128 + (c % 16) * 8 + ((c / 16) % 2) * 4 + s % 4
 * so that one 64-lane load of 16 bytes per lane reads 1 KiB of the tile in
 * the order the matrix-core operands take it.  page_size is a multiple of 16. */
typedef struct {
  void *const *k_pages;        /* host array [n_layers] of device bases */
  void *const *v_pages;        /* host array [n_layers] of device bases */
  int n_layers;
  int page_size;
  int num_pages;
  int max_pages_per_seq;
  const int32_t *block_table;  /* [B][max_pages_per_seq] */
  int32_t *seq_lens;           /* [B] committed lengths m_b */
  int max_ctx;                 /* host: an upper bound on every seq_lens[b] */
} gm_kv_cache;

/* Softmax statistics of one logits row z at temperature T: the max of z / T,
 * the lowest id attaining it, and sum over ids of exp(z / T - max).
 * gm_mtp_draft can emit them for its draft logits; gm_spec_accept can take them
 * in place of its own pass over those rows (q's normaliser, Sec. 2.2). */
typedef struct {
  float max;
  int32_t argmax;
  double sum;
} gm_row_stats;

/* Top-p: the nucleus of one logits row (see gm_spec_accept's top_p): the kept ids are
 * those whose logit's order key exceeds `key`, and those with that key up to id
 * `last_id`; `mass` is sum over them of exp(z / T - m).  (The order key of a float32
 * x: its bits with the sign bit set if x >= 0, all bits inverted if x < 0; -0 as +0.)
 * gm_mtp_draft can emit them for its draft rows under top-p; gm_spec_accept can take
 * them in place of its own passes over those rows. */
typedef struct {
  double m;
  double mass;
  uint32_t key;
  int32_t last_id;
} gm_nucleus;

/* The cycle record's verification distributions (App. "Implementing Draft-Path
 * Reconstruction in verl", recording in rollout): for every sequence b and draft
 * position i < k, the `topk` largest entries of p_i = softmax(target_logits[b][i] / T),
 * as log p_i (normalised over the whole vocabulary, not over the kept entries)
 * rounded to bf16, and their ids; in decreasing probability, equal probabilities
 * in increasing id.  (The record's other items -- the drafts, the accepted
 * length, the start position and the hidden at the cycle's start -- are inputs
 * or outputs of the step already.) */
typedef struct {
  int topk;           /* 1..64, at most V */
  uint16_t *logp;     /* [B][k][topk] bf16 */
  int32_t *ids;       /* [B][k][topk] */
} gm_record;

/* Bytes of workspace the given call needs (0 on invalid arguments).
 * `max_ctx` is the bound that the call's gm_kv_cache carries. */
size_t gm_workspace_size(int op, const gm_model_config *cfg, int B, int k, int max_ctx);

/* Verification forward (Sec. 3.1, Eq. verification-context; App.
 * "Draft-Path Reconstruction": one target forward over the draft path).
 * tokens [B][k+1] is the block [t_m, d_1..d_k].  Writes the K/V entries of
 * the block at positions m_b .. m_b+k of every layer (seq_lens is not
 * changed: gm_kv_commit decides what stays), logits [B][k+1][vocab] float32
 * (row i is the target's distribution for the token after block position i)
 * and hidden [B][k+1][H] float32, the last layer's output before the final
 * RMSNorm (the feature the MTP head consumes).
 * target_stats [B][k+1] (may be NULL): also the softmax statistics of every
 * logits row at `temperature` (gm_row_stats), taken in the LM head's epilogue;
 * gm_spec_accept takes them for the same rows and temperature in place of its
 * pass over the target rows (Sec. 2.2, Eq. accept-rule: p's normaliser and
 * arg-max).  temperature is read only when target_stats is given (> 0).
 * Errors: GM_ERR_CAPACITY if max_ctx + k + 1 > max_pages_per_seq * page_size;
 * GM_ERR_INVALID_ARG for target_stats with temperature <= 0. */
gm_status gm_verify_forward(const gm_model_config *cfg, const gm_model_weights *w,
                            const gm_kv_cache *cache, int B, int k, const int32_t *tokens,
                            float *logits, float *hidden, float temperature, gm_row_stats *target_stats,
                            void *ws, size_t ws_bytes, int32_t *dev_err, void *stream);

/* Verify attention of one layer: the query at block position i of sequence b
 * attends causally to cache positions 0 .. m_b + i (the committed prefix and
 * block positions 0..i, which must already be in the cache), scale
 * 1/sqrt(head_dim), query head h reading KV head h / (n_heads / n_kv_heads).
 * q and out are [B][k+1][n_heads][head_dim] in the model dtype; q is after
 * RoPE. */
gm_status gm_verify_attention(const gm_model_config *cfg, const gm_kv_cache *cache, int layer,
                              int B, int k, const void *q, void *out, void *ws, size_t ws_bytes,
                              int32_t *dev_err, void *stream);

/* Accept rule (Sec. 2.2, Eq. accept-rule).  p_i = softmax(target_logits[b][i] / T),
 * q_i = softmax(draft_logits[b][i] / T).
 * GM_SAMPLE: scanning i = 0..k-1, draft d_i is accepted iff u_accept[b][i] <
 *   p_i(d_i) / q_i(d_i) (ratio rounded to float32); the scan stops at the
 *   first rejection.  With n accepted, the final token is an inverse-CDF draw
 *   with u_final[b] (smallest id x with sum_{y<=x} w(y) > u * sum w) from
 *   w = max(0, p_n - q_n) if n < k (from p_n if that mass is 0), or from
 *   w = p_k (bonus token) if n = k.
 * GM_GREEDY: d_i is accepted iff it is the argmax of target_logits[b][i]
 *   (lowest id on ties); the final token is the argmax of row n.
 *   draft_logits, draft_stats, u_accept and u_final may be NULL.
 * top_p in (0, 1] (GM_SAMPLE; the evaluation setting of App. "Evaluation
 *   Configuration" decodes at T = 1, top-p 0.7): below 1, every p_i and q_i is
 *   replaced by its nucleus before the rule -- the ids ranked by logit (larger
 *   first, the lower id first among equal logits) up to the first at which the
 *   running probability reaches top_p, renormalised -- so the drafts must be
 *   samples of the head's nucleus (gm_mtp_draft with the same top_p).  The
 *   running masses are exact sums of float64 exponentials rounded to 2^-44 of
 *   the row maximum's term.  GM_GREEDY ignores top_p; 1 keeps every id.
 *   GM_ERR_INVALID_ARG outside (0, 1].
 * draft_nucleus [B][k] (may be NULL; read in GM_SAMPLE mode with top_p < 1 only): the
 *   nuclei of the draft_logits rows at this T and top_p, as gm_mtp_draft writes them.
 *   Given, they stand in for the passes over the draft rows (their statistics and
 *   their nucleus); the caller guarantees that they describe these draft_logits.
 * draft_stats [B][k] (may be NULL; read in GM_SAMPLE mode only): the statistics
 *   of softmax(draft_logits[b][i] / T) at this temperature, as gm_mtp_draft
 *   writes them.  Given, they stand in for a pass over the draft rows; the
 *   caller guarantees that they describe these draft_logits.
 * target_stats [B][k+1] (may be NULL): the statistics of softmax(target_logits[b][i] / T)
 *   at this temperature, as gm_verify_forward writes them.  Given, they stand in for
 *   the pass over the target rows (that pass still runs when a record is requested,
 *   whose selection needs it); the caller guarantees that they describe these
 *   target_logits.
 * Outputs: n_accept [B] in [0, k]; out_tokens [B][k+1] = d_0..d_{n-1}, final, -1 pad.
 * record (host struct, may be NULL): also writes the cycle record's top-k
 *   log-probabilities of the target rows 0..k-1 (see gm_record), taken in the same
 *   pass over the target logits.  GM_ERR_INVALID_ARG if topk is outside 1..min(64, V)
 *   or a record buffer is NULL.
 * The logits rows are read in place; no probability matrix is written. */
gm_status gm_spec_accept(int B, int k, int V, int mode, float temperature, float top_p,
                         const float *target_logits, const float *draft_logits,
                         const gm_row_stats *target_stats, const gm_row_stats *draft_stats,
                         const gm_nucleus *draft_nucleus,
                         const int32_t *draft_tokens, const float *u_accept, const float *u_final,
                         int32_t *n_accept, int32_t *out_tokens, const gm_record *record, void *ws,
                         size_t ws_bytes, void *stream);

/* gm_spec_accept for callers that cannot allocate (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same arguments and
 * results, without the workspace.  Its scratch is a fixed 16 MiB device array that
 * each GPU the library runs on holds until the process ends; the call allocates and
 * frees nothing.  Limit: calls whose gm_workspace_size(GM_OP_SPEC_ACCEPT, ...) exceeds
 * 16 MiB return GM_ERR_CAPACITY before touching the device (B = 256 sequences at
 * k = 7, V = 151936 fit, top-p included).  Every call on one GPU shares that GPU's
 * scratch: calls that overlap in time on one GPU (other streams, other threads) race
 * and must be serialised by the caller.  GM_ERR_DEVICE if the scratch's device
 * address cannot be obtained on the current device. */
gm_status gm_spec_accept_noalloc(int B, int k, int V, int mode, float temperature, float top_p,
                                 const float *target_logits, const float *draft_logits,
                                 const gm_row_stats *target_stats, const gm_row_stats *draft_stats,
                                 const gm_nucleus *draft_nucleus, const int32_t *draft_tokens,
                                 const float *u_accept, const float *u_final, int32_t *n_accept,
                                 int32_t *out_tokens, const gm_record *record, void *stream);

/* Commit / rollback (Sec. 2.2; App. "Train--Inference Inconsistency under
 * Teacher Forcing", Eq. tf-restart-kv): block positions 0..n_b stay, the rest
 * are rolled back by index only (no KV bytes move): seq_lens[b] += n_b + 1.
 * committed_slots [B][k+1] (may be NULL) receives the physical slot
 * (page * page_size + offset) of each committed block position, -1 for rolled
 * back ones. */
gm_status gm_kv_commit(const gm_kv_cache *cache, int B, int k, const int32_t *n_accept,
                       int32_t *committed_slots, void *stream);

/* MTP draft of the next block (Sec. 2.2; App. "Models and Draft Heads";
 * Eqs. tf-restart, tf-restart-kv).  mtp_cache is a one-layer cache whose
 * seq_lens hold the head's committed length, equal to the target's committed
 * length before the last verification.  Slot s of the head's cache holds the
 * entry of the pair (h_s, x_{s+1}) rotated at position s+1, where h_s is the
 * target hidden at position s.  Extend: the n_b+1 rows (verify_hidden[b][i],
 * out_tokens[b][i]), i = 0..n_b, are written at slots m_b..m_b+n_b and the
 * head's length becomes m_b+n_b+1 (the entries behind the boundary come from
 * target features).  The output of row n_b gives q_1; chain step j feeds
 * (layer output of step j-1, draft j-1) at slot m_b+n_b+j; those entries lie
 * past the committed length and are overwritten by the next extend.
 * Drafts are argmax (GM_GREEDY) or inverse-CDF draws with u_draft[b][j]
 * (GM_SAMPLE) from softmax(z / T).  Outputs: drafts [B][k],
 * draft_logits [B][k][vocab] float32, and (if draft_stats is not NULL)
 * draft_stats [B][k], the softmax statistics of each draft_logits row at T
 * (the draw's own; gm_spec_accept takes them for the same rows and T).
 * top_p in (0, 1] (GM_SAMPLE): below 1, each draft is the inverse-CDF draw with
 * u_draft[b][j] from the nucleus of softmax(z / T) (as in gm_spec_accept);
 * draft_stats must then be NULL (GM_ERR_UNSUPPORTED otherwise); draft_nucleus [B][k]
 * (may be NULL) receives the nucleus of every draft_logits row (gm_spec_accept takes
 * them for the same rows, T and top_p).  With top_p = 1 or GM_GREEDY it is not written.
 * Errors: GM_ERR_CAPACITY if max_ctx + 2k + 1 > max_pages_per_seq * page_size
 * of the head's cache; GM_ERR_INVALID_ARG for top_p outside (0, 1]. */
gm_status gm_mtp_draft(const gm_model_config *cfg, const gm_mtp_weights *mtp,
                       const gm_model_weights *shared, const gm_kv_cache *mtp_cache, int B, int k,
                       int mode, float temperature, float top_p, const float *verify_hidden,
                       const int32_t *n_accept, const int32_t *out_tokens, const float *u_draft,
                       int32_t *drafts, float *draft_logits, gm_row_stats *draft_stats,
                       gm_nucleus *draft_nucleus, void *ws,
                       size_t ws_bytes, int32_t *dev_err, void *stream);

/* Draft-path reconstruction (App. "Draft-Path Reconstruction"; App. "Parallelizing
 * GrowMTP Training"): the head's chain of each of R recorded cycles re-run under the
 * current head weights with the recorded drafts as inputs and nothing sampled, as K
 * batched single-row steps (one per depth, all cycles together).  mtp_cache is a
 * one-layer cache with one block table row per cycle; seq_lens[r] = s_r, the number of
 * committed head entries the cycle sees (slot s holds the pair (h_s, x_{s+1}) rotated
 * at position s+1, as gm_mtp_draft writes them).  Depth 1 feeds (start_hidden[r],
 * start_tokens[r]) -- the boundary hidden and the last committed token the cycle
 * started from -- at slot s_r; depth j >= 2 feeds (its layer output at depth j-1,
 * drafts[r][j-2]) at slot s_r + j - 1.  Depth j attends to slots 0 .. s_r + j - 1 of the
 * cycle's own table: causal over the committed prefix, its own chain's entries (the
 * diagonal mask of the batched form).  The entries at slots s_r .. s_r + K - 1 are
 * written, so those pages must be the cycle's own (cycles may share the pages of their
 * prefix).  seq_lens is not changed.
 * start_hidden [R][H] float32; start_tokens [R]; drafts [R][K] (d_1..d_{K-1} are read;
 * may be NULL when K = 1); head_logits [R][K][vocab] float32: row j is the head's
 * logits at depth j+1 (q_{r,j+1} = softmax of it), the input of gm_dca_loss.
 * Errors: GM_ERR_CAPACITY if max_ctx + K > max_pages_per_seq * page_size. */
gm_status gm_mtp_reconstruct(const gm_model_config *cfg, const gm_mtp_weights *mtp,
                             const gm_model_weights *shared, const gm_kv_cache *mtp_cache, int R, int K,
                             const float *start_hidden, const int32_t *start_tokens, const int32_t *drafts,
                             float *head_logits, void *ws, size_t ws_bytes, int32_t *dev_err, void *stream);

/* Depth-coupled acceptance loss with verify-gated masking, and its gradient in
 * the head logits (Sec. "The Depth-Coupled Acceptance Loss" and "Learning up to
 * the First Rejection", Eqs. alpha, chain, dca, vgm; App. "DCA"), over the cycle
 * record's sparse support (App. "Implementing Draft-Path Reconstruction in
 * verl").  For cycle n and draft position k: q = softmax(head_logits[n][k]) over
 * the whole vocabulary, gathered at the record's ids S; p = exp(rec_logp); one
 * residual bin holds the mass outside S, p_R = max(0, 1 - sum_S p), q_R = 1 - sum_S q.
 *   alpha[n][k] = sum_S min(p, q) + min(p_R, q_R)
 *   loss[n]     = -log sum_{l=1}^{L} prod_{i<=l} alpha[n][i],
 *                 L = min(n_accept[n] + 1, K) if vgm, else K
 * grad (may be NULL) [N][K][V]: d loss[n] / d head_logits[n][k][x] (positions past
 * L get 0; the subgradient of min is 0 where its arguments are equal).
 * head_logits [N][K][V] float32; rec_logp [N][K][topk] bf16; rec_ids [N][K][topk]
 * (distinct ids in 0..V-1; an id outside gets q = 0 and is never read); n_accept [N] in 0..K.
 * loss [N] and alpha [N][K] are float32 (computed in float64); grad is float32.
 * Limits: 1 <= K <= 15, 1 <= topk <= min(64, V), V <= 524288. */
gm_status gm_dca_loss(int N, int K, int V, int topk, const float *head_logits, const uint16_t *rec_logp,
                      const int32_t *rec_ids, const int32_t *n_accept, int vgm, float *loss, float *alpha,
                      float *grad, void *ws, size_t ws_bytes, void *stream);

/* ---- Draft trees.
 * A tree of up to 64 nodes per sequence takes the place of the draft chain (the
 * method drafts a chain, Sec. 2.2; a tree verifies several continuations at once):
 * node 0 is the pending token t_m, node i > 0 continues node parents[b][i] < i.
 * Node i's K/V entry is written at slot m_b + i, rotated at position m_b + depth_i
 * (gm_kv_append), node i attends to the committed positions, to its ancestors and
 * to itself (gm_tree_attention), the target's tokens select one path from the root
 * (gm_tree_accept), and the path's entries move to the slots behind the committed
 * length (gm_tree_commit).  n_nodes [B] (may be NULL: all N) are the nodes each
 * sequence has, 0..N (values outside are clamped); the rest is padding. */

/* Append: keys and values of T new positions, rotated and written into one layer of
 * the cache, and (optionally) their queries rotated.  Sequence b owns the rows
 * row_start[b] .. row_start[b+1] - 1 (row_start [B+1], increasing; NULL: T / B rows
 * each, T a multiple of B); its i-th row goes to slot seq_lens[b] + i and is rotated
 * at position seq_lens[b] + offsets[row] (offsets [T]; NULL: seq_lens[b] + i), so a
 * prompt is appended in one call and a draft tree with its nodes' depths as offsets
 * (plus 1 in the MTP head's cache, whose slots are rotated one position on).
 * Rows outside every sequence's range are left alone.  seq_lens is not changed.
 * k and v are [T][n_kv_heads][head_dim], q [T][n_heads][head_dim] in the model dtype;
 * a row's heads are consecutive and rows are *_stride elements apart (the column
 * blocks of one projection can be given in place).  q_out [T][n_heads][head_dim] is
 * contiguous; it may be q itself if q is contiguous, and must not overlap q otherwise.
 * q and q_out may both be NULL.  With cfg->qk_norm, k (and q) pass a per-head RMSNorm
 * with weights k_norm and q_norm [head_dim] before the rotation.  Rotation: pairs
 * (c, c + head_dim / 2) by position * rope_base^(-2 c / head_dim), angles in float64.
 * max_rows (host): an upper bound on every sequence's rows.
 * Errors: GM_ERR_CAPACITY if max_ctx + max_rows > max_pages_per_seq * page_size;
 * dev_err GM_DEVERR_PAGE for a block-table entry outside the pool (its rows' K/V are
 * not written; q_out is). */
gm_status gm_kv_append(const gm_model_config *cfg, const gm_kv_cache *cache, int layer, int B, int T, int max_rows,
                       const int32_t *row_start, const int32_t *offsets, const void *q, int64_t q_stride,
                       const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *q_norm,
                       const void *k_norm, void *q_out, int32_t *dev_err, void *stream);

/* The plan of a batch of trees, made once per step and read by every layer: masks
 * [B][N], bit j of masks[b][i] set iff node j is i or an ancestor of i, and depths
 * [B][N] (0 for node 0).  A node whose parent is outside -1 .. i-1, or not a node of
 * the tree, has no ancestors (dev_err GM_DEVERR_TREE); parent -1 is allowed for any
 * node (such a node continues the committed tokens, as node 0 does).  Nodes past
 * n_nodes[b] get mask 0 and depth 0. */
gm_status gm_tree_masks(int B, int N, const int32_t *parents, const int32_t *n_nodes, uint64_t *masks,
                        int32_t *depths, int32_t *dev_err, void *stream);

/* Attention of one layer over the cache for the nodes of a tree: node i of sequence b
 * attends to positions 0 .. m_b - 1 and to m_b + j for every bit j < n_nodes[b] of
 * masks[b][i] (any set of nodes: gm_tree_masks makes those of a tree; the entries must
 * already be in the cache).  q and out are [B][N][n_heads][head_dim] in the model
 * dtype, q after the rotation; scale 1 / sqrt(head_dim), query head h reads KV head
 * h / (n_heads / n_kv_heads).  Rows of padding nodes, and of nodes that see nothing,
 * are 0.  A node's row does not depend on entries it does not attend to, whatever
 * they hold.
 * Limits: 1 <= N <= 64, n_heads / n_kv_heads <= 64.
 * Errors: GM_ERR_CAPACITY if max_ctx + N > max_pages_per_seq * page_size; dev_err
 * GM_DEVERR_PAGE for a block-table entry outside the pool (its positions are not
 * attended to; which of those behind them are is not specified). */
gm_status gm_tree_attention(const gm_model_config *cfg, const gm_kv_cache *cache, int layer, int B, int N,
                            const void *q, const uint64_t *masks, const int32_t *n_nodes, void *out, void *ws,
                            size_t ws_bytes, int32_t *dev_err, void *stream);

/* The accept of a tree.  next_ids [B][N] holds the target's own token after each node:
 * its arg-max (greedy), or a draw from its distribution at that node (each node's
 * draw an independent one: the committed tokens are then distributed as the target's,
 * whatever the tree holds).  From node 0 the walk goes on to the child whose token is
 * next_ids of the node it stands on (the lowest index if several), until there is none.
 * Outputs: n_accept [B], the accepted nodes without node 0; path [B][N] = 0, the
 * accepted nodes in order, -1 pad; out_tokens [B][N] = the accepted nodes' tokens, then
 * next_ids of the last node, -1 pad.  A sequence with n_nodes[b] = 0 gets n_accept -1
 * and -1 throughout. */
gm_status gm_tree_accept(int B, int N, const int32_t *parents, const int32_t *tokens, const int32_t *next_ids,
                         const int32_t *n_nodes, int32_t *path, int32_t *n_accept, int32_t *out_tokens, void *stream);

/* Commit of a tree's path: in every layer of the cache the K and V entries of slot
 * m_b + path[b][i] move to slot m_b + i, i = 0 .. n_accept[b], and seq_lens[b] grows by
 * n_accept[b] + 1; the rest is rolled back by index only.  path is increasing with
 * path[b][i] >= i, as gm_tree_accept writes it (a sequence's entries that are not are
 * left where they are: dev_err GM_DEVERR_TREE); n_accept is clamped to -1 .. N-1.  The
 * cache's page pools are those of cfg's dtype, n_kv_heads and head_dim; every layer of
 * the cache is committed (n_layers need not be cfg's: the MTP head's cache has one).
 * committed_slots [B][N] (may be NULL): the physical slot (page * page_size + offset)
 * of each committed position, -1 for the others.  dev_err GM_DEVERR_PAGE for a
 * block-table entry outside the pool (that entry does not move). */
gm_status gm_tree_commit(const gm_model_config *cfg, const gm_kv_cache *cache, int B, int N, const int32_t *path,
                         const int32_t *n_accept, int32_t *committed_slots, int32_t *dev_err, void *stream);

/* Softmax statistics that gm_token_logprobs leaves for its gradient: the row's largest
 * logit and sum over ids of exp((z - max) / T).  (log-sum-exp of z / T = max / T + log sum.) */
typedef struct {
  float max;
  float sum;
} gm_token_stats;

/* Log-probabilities of given tokens under softmax(z / T), with the entropy and the most
 * likely alternatives: the policy's side of an RL update, the target's choice at a
 * tree's nodes, and the candidates a tree is grown from.
 * logits [M][V], dtype GM_F32 or GM_BF16, rows ld elements apart (ld >= V).  Each output
 * may be NULL:
 *   logp [M]: log p(ids[m]), 0 where ids[m] < 0 (no token); needs ids [M].  An id >= V
 *     counts as no token (dev_err GM_DEVERR_TOKEN).
 *   entropy [M]: -sum p log p (ids of probability 0 add 0).
 *   top_logp, top_ids [M][topk] (both or neither): the topk largest logits' log p and
 *     ids, in decreasing logit, equal logits in increasing id; 1 <= topk <= min(64, V).
 *   stats [M]: for gm_token_logprobs_grad.
 * Sums are float32 over at most 4096 ids, added pairwise in part, and float64 beyond.
 * Logits of -inf have probability 0; a log p below float32's range is -inf.  A row
 * without any other logit: log p -inf, entropy 0, stats (-inf, 0), alternatives
 * 0 .. topk-1.  A row that holds NaN or +inf gives NaN log p and entropy, and
 * alternatives -1.
 * Limits: V <= 524288, M <= 2^23, temperature >= 1e-37. */
gm_status gm_token_logprobs(int M, int V, int dtype, const void *logits, int64_t ld, float temperature,
                            const int32_t *ids, float *logp, float *entropy, int topk, float *top_logp,
                            int32_t *top_ids, gm_token_stats *stats, void *ws, size_t ws_bytes, int32_t *dev_err,
                            void *stream);

/* Its gradient in the logits: grad[m][x] = g_logp[m] d logp[m] / d z_x
 * + g_entropy[m] d entropy[m] / d z_x
 *   = ([x = ids[m]] g_logp - p_x (g_logp + g_entropy (log p_x + entropy))) / T,
 * with g_logp taken as 0 where ids[m] is no token.  logits, ld, ids and temperature as
 * in the call that wrote stats (and entropy); g_entropy may be NULL (0), else entropy is
 * needed; ids and g_logp may both be NULL.  grad [M][V] has the logits' dtype (rounded
 * once, from float32) and rows ld_grad elements apart; it may be the logits themselves
 * (with the same ld), and must not overlap them otherwise.  A row whose statistics are
 * (-inf, 0) gets 0.  The alternatives have no gradient. */
gm_status gm_token_logprobs_grad(int M, int V, int dtype, const void *logits, int64_t ld, float temperature,
                                 const int32_t *ids, const gm_token_stats *stats, const float *entropy,
                                 const float *g_logp, const float *g_entropy, void *grad, int64_t ld_grad,
                                 void *stream);

/* Thread-local message describing the last non-OK status of this thread. */
const char *gm_last_error(void);

/* Kernel timing.  While tracing is on, every kernel the library launches
 * whose name matches `filter` (all kernels when NULL) is bracketed by a pair
 * of HIP events on its stream.  gm_trace_stop() waits for the recorded events
 * and sums their durations per kernel name.  The events record timestamps
 * only (no system-scope fence); each still leaves the stream idle for a few
 * microseconds.  gm_trace_every(n) (n >= 1, else GM_ERR_INVALID_ARG; default
 * 1) brackets only every n-th matching launch, counted from gm_trace_start, so
 * that a timing sample perturbs fewer launches. */
gm_status gm_trace_every(int n);
gm_status gm_trace_start(const char *filter);
gm_status gm_trace_stop(void);
int gm_trace_count(void);
gm_status gm_trace_get(int i, const char **name, int *launches, double *total_ms);

#ifdef __cplusplus
}
#endif
#endif /* GM_H */
