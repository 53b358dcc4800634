/*
 * adore.h - C ABI of the ADORE decode-step library for MI355X (gfx950).
 *
 * One context holds the state of one decode job of B sequences: per layer a
 * fixed-size, slot-addressed K/V cache of K rows per (sequence, head), the
 * per-token keep probabilities sigma_i, and the controller's GRU state.
 * One decode step = the four stages of the paper's method (arXiv 2407.02328):
 *
 *   attend    single-query attention over the occupied slots, the current
 *             token's k, v included                       (Sec. 2.1, Eq. 1 and
 *                                                          the "target" equation)
 *   schedule  controller score of the arriving token       (Sec. 2.2, Eq. 2;
 *             App. "Implementation Details", controller module),
 *             release of the lowest-scored rows            (Sec. 2.2, third
 *                                                          design strategy),
 *             choice of the top-R released tokens          (Sec. 2.3)
 *   rebuild   K/V of the chosen tokens re-projected from their hidden states
 *             with W_k / W_v and written into the freed slots (Sec. 2.3)
 *
 * Symbols: L layers, B sequences, H heads, d head_dim, D hidden size, K cache
 * slots per (sequence, head), R rebuild budget per step and sequence,
 * m = K - R - 1 persistent rows, d' controller hidden size, n = 0-based
 * position of the current token, S prompt length.
 *
 * Conventions
 *   - Every pointer is a DEVICE pointer unless its comment says HOST.  The two
 *     structs below are read on the host.
 *   - All arrays are contiguous, row-major, last index fastest, bases 16-byte
 *     aligned.  "storage type" is adore_config.dtype (bf16 or fp32).
 *   - The caller owns all memory.  The library allocates no device memory; the
 *     workspace passed to adore_create holds all of its state.
 *   - attend / schedule / rebuild / decode_step only enqueue work on the
 *     context's stream and never synchronise it: outputs are valid once the
 *     caller has synchronised that stream.  Input buffers must stay unchanged
 *     until then.  Inputs may be produced by work enqueued on that stream before
 *     the call (see adore_set_input_order for the one exception a caller can
 *     ask for).
 *   - The return value is the only error channel.  Arguments and the order of
 *     calls are validated on the host before anything is enqueued: a call that
 *     returns E_INVALID, E_STATE, E_UNSUPPORTED or E_WORKSPACE has had no effect.
 *     E_HIP means the HIP runtime refused something in the middle of a call;
 *     part of the step may have been enqueued, and the context has to be
 *     restarted with adore_init_cache (or adore_set_state) before its next step.
 *   - A context is bound to one stream and is not thread-safe.  Contexts are
 *     independent of each other.
 *   - Ties between equal sigma are broken in favour of the lower position, so
 *     every selection has exactly one result.  A NaN sigma is treated as 0.
 */
#ifndef ADORE_H
#define ADORE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ADORE_ABI_VERSION 10

typedef struct adore_ctx adore_ctx; /* opaque */

enum { ADORE_F32 = 0, ADORE_BF16 = 1 };

/* When the controller's score of a token is taken (the two readings of Sec. 2.2):
 * STATIC:  sigma_i once, when token i arrives, with the position feature i * pos_scale (Eq. 2 as printed).
 * RESCORE: at every step n, sigma_i for every token i <= n from its stored GRU state z_i with the
 *          position feature (n - i) * pos_scale (the controller rates the cached tokens "for the current
 *          token", Sec. 2.2 and the caption of Fig. 2); both selections of the step use the new values,
 *          so a rebuilt token can be kept.  score_override must be NULL in every call, set_state is
 *          not available, and d' must be a multiple of 4. */
/* H2O:     the H2O(Rebuilt) baseline of Sec. 3.1 (baselines 6 and 7): no controller; the score of a token is the
 *          attention it has received so far, kept per head: score[b][h][i] = sum over the steps at which head h
 *          held a row of token i of the probability the step's query gave that row (fp32, added in step order; an
 *          evicted token keeps its score and collects again once rebuilt).  Every head releases on its own scores
 *          and has its own slot map.  The rebuild is per sequence (one row of the re-projection serves all heads):
 *          candidates are the tokens at least one head is missing, ranked by the fp32 sum of their scores over the
 *          heads (head 0 first), equal sums to the lower position; a head that still holds a chosen token keeps its
 *          row, the others put it into their lowest free slots in rank order.  (The paper gives the baseline two
 *          sentences; the rest is this reading.)  One layer per context, no rotary embedding, heads <= 255,
 *          max_positions <= about 7000 (the keys of a sequence live in 64 KB of LDS; fewer with a large R); x_n and the controller weights are not read (x_n may be NULL, the weight
 *          pointers must still be non-null); score_override of adore_init_cache is [B][H][S], the attention the
 *          prompt tokens collected during the prompt (NULL: zeros), and must be NULL in the step calls; the scores
 *          of get_state are [B][H][N_max]; no set_state, no adore_forward_step. */
enum { ADORE_SCORE_STATIC = 0, ADORE_SCORE_RESCORE = 1, ADORE_SCORE_H2O = 2 };

enum {
  ADORE_OK = 0,
  ADORE_E_INVALID = -1,     /* null pointer, bad shape or value */
  ADORE_E_STATE = -2,       /* call out of order, or step past max_positions */
  ADORE_E_UNSUPPORTED = -3, /* valid in principle, no kernel for it */
  ADORE_E_WORKSPACE = -4,   /* workspace too small or misaligned */
  ADORE_E_HIP = -5          /* a HIP runtime call failed */
};

typedef struct {
  int32_t layers, batch, heads, head_dim, hidden;     /* L, B, H, d, D */
  int32_t cache_slots, rebuild_budget, max_positions; /* K, R (0 <= R <= K-2), N_max */
  int32_t ctrl_hidden;                                /* d' */
  int32_t dtype;                                      /* ADORE_F32 | ADORE_BF16 */
  float pos_scale;                                    /* position feature of token i = (float)i * pos_scale */
  int32_t score_mode;                                 /* ADORE_SCORE_STATIC | ADORE_SCORE_RESCORE | ADORE_SCORE_H2O */
  float rope_base;                                    /* 0: off.  > 0: rotary position embedding (the one the paper's
                                                         backbones apply to q and k; the paper names it in its related
                                                         work on length extrapolation) on every key the library makes
                                                         from a hidden state, and on the queries of the rebuild forward:
                                                         the projection is rounded to the storage type, elements j and
                                                         j + d/2 of each head are turned by pos * rope_base^(-2j/d), and
                                                         the result is rounded again.  Keys and queries the caller
                                                         supplies (prompt_k, k_new, q) are taken as they are. */
} adore_config;

/* Device pointers, caller-owned, read-only, must outlive the context. */
typedef struct {
  const void *w_kv;      /* [L][2*H*d][D] storage type; rows 0..H*d-1 = W_k, the rest = W_v;
                            within each half, rows h*d..h*d+d-1 belong to head h */
  const void *gru_w_ih;  /* [3*d'][D]  storage type, gate order r, z, n */
  const void *gru_w_hh;  /* [3*d'][d'] storage type, gate order r, z, n */
  const float *gru_b_ih; /* [3*d'] */
  const float *gru_b_hh; /* [3*d'] */
  const float *pos_w;    /* [d']      position layer, 1 -> d' */
  const float *pos_b;    /* [d'] */
  const float *mlp_w1;   /* [d'][d']  interaction layer (tanh) */
  const float *mlp_b1;   /* [d'] */
  const float *out_w;    /* [d']      output layer (sigmoid) */
  const float *out_b;    /* [1] */
} adore_weights;

/* Bytes of device workspace adore_create needs for this configuration (0 if the
 * configuration is invalid).  HOST call, no GPU work.  For prompts beyond 512 tokens over a small cache (less than
 * 6 KB * ctrl_hidden of keys per sequence) this includes room that earlier versions did not ask for; adore_create still takes their
 * amounts, and such prompts are then loaded 5 to 12 % slower. */
size_t adore_workspace_bytes(const adore_config *cfg);

/* Creates a context over `workspace` (device memory, 256-byte aligned, at least
 * adore_workspace_bytes(cfg) bytes, owned by the caller and kept alive until
 * adore_destroy).  `hip_stream` is a hipStream_t (NULL = the default stream).
 * cfg and weights are HOST structs and are copied.  The cache starts empty;
 * call adore_init_cache before the first step.
 * Errors: E_INVALID (null, R > K-2, sizes <= 0, or sizes beyond what 32-bit counts hold with a wide
 * margin: L > 4096, B*H > 2^20, H*d or D > 2^20, K > 2^20, N_max > 2^24), E_UNSUPPORTED (head_dim not in
 * {64,128}, K > 1024 unless K - R - 1 >= N_max, i.e. a cache that holds every
 * token and is the full attention of Eq. 1 ... see adore_strerror), E_WORKSPACE. */
int adore_create(const adore_config *cfg, const adore_weights *weights, void *workspace,
                 size_t workspace_bytes, void *hip_stream, adore_ctx **out);

/* Frees the host-side context.  Does not touch device memory. */
int adore_destroy(adore_ctx *ctx);

/* Loads a prompt of S >= 1 tokens (the paper's user input t_1..t_s, Sec. 2.1) by
 * applying the step rules once: the controller scores tokens 0..S-1 in order
 * (Eq. 2); the residents are token S-1 plus the best min(S,m)-1 older tokens,
 * placed from slot 0 in ascending position with the given K/V; the best
 * min(R, rest) of the remaining tokens are rebuilt from hidden_store into the
 * next slots by rank.
 *   prompt_k, prompt_v  [L][B][H][S][d]  storage type
 *   hidden_store        [L][B][N_max][D] storage type, rows < S valid
 *   ctrl_input          [B][S][D]        storage type (token embeddings x_i)
 *   score_override      [B][S] fp32 or NULL: if given, replaces the controller's sigma
 * hidden_store == NULL prepares the context for adore_forward_step instead: the best min(R, rest)
 * tokens are chosen and given their slots, but their K/V are computed by the first forward step.
 * Enqueues work; does not synchronise.  May be called again to restart.
 * Errors: E_INVALID (null, S < 1, S >= N_max), E_UNSUPPORTED (hidden_store == NULL and K > 8192 or
 * H2O scores: see adore_forward_step). */
int adore_init_cache(adore_ctx *ctx, const void *prompt_k, const void *prompt_v,
                     const void *hidden_store, const void *ctrl_input,
                     const float *score_override, int32_t S);

/* Stage 1 for one layer (Sec. 2.1): writes k_new, v_new into the slot reserved
 * for the current token and computes
 *   out[b][h][:] = sum_k softmax_k(q . Kc[k] / sqrt(d)) Vc[k]  over occupied slots.
 *   q, k_new, v_new  [B][H][d] storage type;  out [B][H][d] fp32.
 * Each layer must be attended exactly once per step, before adore_schedule.
 * Errors: E_INVALID, E_STATE (no init, layer already attended, step past N_max). */
int adore_attend(adore_ctx *ctx, int32_t layer, const void *q, const void *k_new,
                 const void *v_new, float *out);

/* Stages 2 and 3, once per step for all layers (uniform policy, Sec. 2.2):
 * sigma_n from the controller (Eq. 2) or from score_override; release of the
 * x = max(0, occupied - m) lowest-ranked rows of every (b,h), never the current
 * token; choice of the best min(R, pool) released tokens per sequence
 * (Sec. 2.3); assignment of rebuilt rank rho to the rho-th lowest free slot.
 *   x_n             [B][D] storage type (embedding of the current token)
 *   score_override  [B] fp32 or NULL
 *   slot_map        [B][H][K] i32 or NULL: position held by each slot after the
 *                   step, -1 = free
 *   released_pos    [B][H][R+1] i32 or NULL: released positions in ascending slot
 *                   order, -1 padded
 *   rebuilt_pos     [B][max(R,1)] i32 or NULL: chosen positions best first, -1 padded
 * Errors: E_INVALID, E_STATE (a layer not yet attended, schedule already done). */
int adore_schedule(adore_ctx *ctx, const void *x_n, const float *score_override,
                   int32_t *slot_map, int32_t *released_pos, int32_t *rebuilt_pos);

/* Stage 4 for one layer (Sec. 2.3): for each chosen token, one rounding to the
 * storage type of W_kv[layer] . hidden_store_layer[b][pos] (fp32 accumulation),
 * head slices scattered into the slots assigned by adore_schedule.
 *   hidden_store_layer  [B][N_max][D] storage type; rows of all positions <= n valid
 * Each layer must be rebuilt exactly once per step, after adore_schedule; the
 * step completes (n advances) when the last layer is rebuilt.
 * Errors: E_INVALID, E_STATE. */
int adore_rebuild(adore_ctx *ctx, int32_t layer, const void *hidden_store_layer);

/* The whole step for L == 1: attend(0); schedule; rebuild(0).
 *   q, k_new, v_new [B][H][d]; hidden_store [B][N_max][D]; x_n [B][D];
 *   score_override [B] or NULL; out [B][H][d] fp32; slot_map [B][H][K] or NULL.
 * Errors: as the three calls; E_INVALID if L != 1. */
int adore_decode_step(adore_ctx *ctx, const void *q, const void *k_new, const void *v_new,
                      const void *hidden_store, const void *x_n, const float *score_override,
                      float *out, int32_t *slot_map);

/* Rebuild forward through the layer stack (Sec. 2.3 in full: "the embeddings of the top-R released tokens
 * are concatenated with the current token" and go through every layer as R+1 query rows, whose
 * outputs are the next layer's inputs).  One call is one whole step for all L layers; it replaces
 * attend / schedule / rebuild, which need the caller to supply per-layer hidden states.
 * Rows of a sequence: the r tokens chosen by the previous step (or by adore_init_cache), by rank, then the
 * current token n.  Per layer l, with x the rows entering the layer (layer 0: their embeddings):
 *   q = round(W_q[l] x), [k; v] = round(W_kv[l] x)      k, v go to the rows' cache slots
 *   o[j] = softmax over the slots whose position is <= position(j) of q[j] . Kc / sqrt(d), times Vc
 *          (the paper prints no mask for these rows; a decoder's causal rule is used, so a rebuilt
 *           state equals the state the token had when all earlier tokens are present)
 *   x'   = round(x + W_o[l] round(o))                   a layer is attention + residual only: norms and
 *                                                        feed-forward belong to the backbone model
 * then the controller, the release and the choice of the next r tokens as in adore_schedule.
 *   fw->w_q   [L][H*d][D]  storage type, rows grouped by head like W_k
 *   fw->w_o   [L][D][H*d]  storage type
 *   embed     [B][N_max][D] storage type: token embeddings, rows of all positions <= n valid
 *   score_override, slot_map, released_pos, rebuilt_pos: as adore_schedule
 *   rows_out  [B][R+1][D] storage type: the last layer's rows; rank j at [b][j], the current token
 *             at [b][R]; rows of unused ranks are left untouched
 *   layer_rows [L][B][R+1][D] storage type or NULL: the rows leaving every layer (the hidden states of the
 *             rebuilt tokens and of the current one, layer by layer), laid out like rows_out; [L-1] equals rows_out
 * Requires a context initialised with hidden_store == NULL and K <= 8192.  bf16 storage with H*d and D
 * multiples of 128 runs the projections on the matrix cores, and with R + 1 <= 64 the attention too; any
 * other configuration (fp32 storage, other widths, more rows) takes plain kernels for that part, one wave
 * per output element: the same arithmetic in fp32, a reference path rather than a fast one.
 * Enqueues work; does not synchronise.
 * Errors: E_INVALID, E_STATE (not initialised for the forward, step past N_max). */
typedef struct {
  const void *w_q;
  const void *w_o;
} adore_forward_weights;
int adore_forward_step(adore_ctx *ctx, const adore_forward_weights *fw, const void *embed,
                       const float *score_override, void *rows_out, void *layer_rows, int32_t *slot_map,
                       int32_t *released_pos, int32_t *rebuilt_pos);

/* Snapshot / restore between steps.  Any pointer may be NULL (skipped).
 *   slot_pos [B][H][K] i32; scores [B][N_max] fp32; z [B][d'] fp32;
 *   cache_k, cache_v [L][B][H][K][d] storage type; step: HOST pointer, the
 *   position n of the next token.
 * get enqueues device-to-device copies (no synchronisation; *step is written at
 * once).  set copies, then SYNCHRONISES the stream to recount the occupied
 * slots; slot_pos must be given and must leave at least one free slot per (b,h).
 * Errors: E_INVALID, E_STATE (in the middle of a step). */
int adore_get_state(adore_ctx *ctx, int32_t *slot_pos, float *scores, float *z,
                    void *cache_k, void *cache_v, int32_t *step);
int adore_set_state(adore_ctx *ctx, const int32_t *slot_pos, const float *scores,
                    const float *z, const void *cache_k, const void *cache_v, int32_t step);

/* Input order.  The controller and the selections of a step run on a stream of the
 * context's own, next to the attention and the rebuild (where a step is too short for
 * that to pay, on the context's stream like everything else); they read x_n / embed and
 * score_override.  ordered != 0 (the default): they start behind everything that was
 * enqueued on the context's stream before the call, so those inputs may come from
 * kernels enqueued there, at the price of one more cross-stream event per step.
 * ordered == 0: the caller guarantees that x_n (embed) and score_override of a step
 * are complete in memory when the step's call is made (say, the token's embedding
 * was gathered before the stream was last synchronised); that event is dropped and
 * the side work of later steps may start early.  All other inputs are read on the
 * context's stream in either mode.  Outputs with ordered == 0: slot_map, released_pos
 * and rebuilt_pos of a step may then be written as soon as its call is made, ahead of
 * work queued on the context's stream; a caller whose earlier work on that stream
 * still reads the previous step's values gives each step buffers of its own (or
 * synchronises first).  `out` and rows_out are written on the context's stream.
 * The first step after adore_init_cache starts behind the init in either mode.
 * HOST call between steps.
 * Errors: E_INVALID, E_STATE (in the middle of a step). */
int adore_set_input_order(adore_ctx *ctx, int32_t ordered);

/* Per-kernel timing with HIP events on the context's stream (for benchmarks).
 * While enabled, every kernel launch is bracketed by two events.
 * adore_read_timing SYNCHRONISES the stream, adds up the elapsed milliseconds
 * per kernel since the last read into ms[ADORE_N_KERNELS] and the launch counts
 * into launches[ADORE_N_KERNELS] (both HOST arrays), and clears the record. */
enum {
  ADORE_KERNEL_ATTEND = 0,      /* insert + attention (partials when a row is split) */
  ADORE_KERNEL_ATTEND_COMBINE,  /* merge of the split partials; not launched for one split */
  ADORE_KERNEL_CTRL_INPUT,      /* GRU input projection */
  ADORE_KERNEL_CTRL_CELL,       /* GRU cell + MLP + sigmoid */
  ADORE_KERNEL_RELEASE,         /* per-(b,h) release select */
  ADORE_KERNEL_REBUILD_SELECT,  /* per-sequence top-R select + slot assignment */
  ADORE_KERNEL_REBUILD_GEMM,    /* re-projection + scatter */
  ADORE_KERNEL_RESCORE,         /* RESCORE mode: sigma of every token for the current step */
  ADORE_KERNEL_FWD_QKV,         /* rebuild forward: q, k, v projection of the rebuilt tokens' rows + scatter */
  ADORE_KERNEL_FWD_QKV_CUR,     /* rebuild forward: the same for the current tokens' rows (one per sequence) */
  ADORE_KERNEL_FWD_ATTEND,      /* rebuild forward: attention of the R+1 rows */
  ADORE_KERNEL_FWD_OPROJ,       /* rebuild forward: output projection + residual, rebuilt tokens' rows */
  ADORE_KERNEL_FWD_OPROJ_CUR,   /* rebuild forward: the same for the current tokens' rows */
  ADORE_KERNEL_ROPE,            /* rotary embedding of the rows a projection just wrote (rope_base > 0) */
  ADORE_KERNEL_H2O_RELEASE,     /* H2O mode: the step's attention added to the scores, then the per-head release */
  ADORE_KERNEL_H2O_CHOICE,      /* H2O mode: per-sequence choice of the tokens to rebuild on the sum over heads */
  ADORE_KERNEL_H2O_PLACE,       /* H2O mode: per head, the slots of the chosen tokens it is missing */
  ADORE_N_KERNELS
};
int adore_set_timing(adore_ctx *ctx, int32_t enable);
int adore_read_timing(adore_ctx *ctx, float *ms, int32_t *launches);
const char *adore_kernel_name(int32_t kernel);

/* Top-K attention over a whole sequence (Sec. 2.1: keeping the highest of a query's full weights is the ideal
 * sparsity; Sec. 2.2, first strategy, and App. "Implementation Details": the attention the backbone is fine-tuned
 * with, the weights outside the top K masked out).  Stateless: no context.  Causal, per row (= sequence x head):
 *   w[i][j] = q_i . k_j for j <= i;  query i keeps its top_k largest weights (all while i + 1 <= top_k; equal
 *   weights go to the lower j);  out_i = sum over the kept j of softmax_j(w[i][j] / sqrt(head_dim)) v_j.
 * q, k, v, out: DEVICE [rows][seq][head_dim] bf16, dense; out may not alias the inputs.  workspace: DEVICE,
 * 256-byte aligned, at least adore_topk_attention_workspace_bytes(rows, seq, head_dim) bytes, caller-owned, free to reuse
 * after the work enqueued here has run (reserved: the kernel keeps everything on chip and does not touch it).  The call only enqueues work on
 * hip_stream (a hipStream_t, NULL = the default stream).  The selection is exact on the weights as the kernel
 * computes them (bf16 products accumulated in fp32); inputs must be finite.
 * Errors: E_INVALID (null, sizes <= 0, top_k < 1), E_UNSUPPORTED (head_dim not in {64,128}, seq > 32768,
 * rows > 65535), E_WORKSPACE, E_HIP.  adore_topk_attention_workspace_bytes is a HOST call and returns 0 for
 * sizes the entry point would not take. */
size_t adore_topk_attention_workspace_bytes(int32_t rows, int32_t seq, int32_t head_dim);
int adore_topk_attention(const void *q, const void *k, const void *v, void *out, void *workspace,
                         size_t workspace_bytes, int32_t rows, int32_t seq, int32_t head_dim, int32_t top_k,
                         void *hip_stream);

/* adore_topk_attention for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid it): the same kernel and the same result, bit for bit, without a workspace.  The call allocates
 * and frees nothing.  Limits: seq <= 2048 and rows * head_dim * ceil(seq / 32) * 64 <= ADORE_TOPK_STATIC_SCRATCH_BYTES, else
 * E_WORKSPACE (e.g. 256 rows of 1024 tokens at head_dim 128).  Calls share nothing: they may overlap on any streams and threads.
 * Errors: as adore_topk_attention; E_WORKSPACE when the shape exceeds those limits. */
#define ADORE_TOPK_STATIC_SCRATCH_BYTES (64u << 20)
int adore_topk_attention_static(const void *q, const void *k, const void *v, void *out, int32_t rows, int32_t seq,
                                int32_t head_dim, int32_t top_k, void *hip_stream);

/* ---- Attention over whole prompts (Sec. 2.1, Eq. 1 for every token of the prompt) ----
 * The pass that makes what adore_init_cache and the 4-bit cache below are loaded with, its gradients, and the attention
 * every token received in it (what H2O goes by, Sec. 3.1).  Stateless: no context.  Causal, with grouped heads: query head
 * h reads kv head h / (heads / kv_heads).
 *   w_ij = scale q_i . k_j for j <= i + nk - nq (a sequence's last query sees its last key; with nq < nk the keys before
 *   its first query are a prefix that is there already, with nq > nk the first queries see nothing)
 *   lse_i = ln sum_j exp w_ij;   out_i = sum_j exp(w_ij - lse_i) v_j   (no key: out_i = 0, lse_i = -inf)
 *   received_j = the sum of exp(w_ij - lse_i) over the queries of all heads of j's group
 * Sequences: with q_start and k_start (both [batch + 1] i32, DEVICE) packed ones, of any lengths from 0 on: the tokens
 * of sequence b are rows q_start[b] .. q_start[b + 1] - 1 of the q_tokens rows of q, d_out, out, dq (k_start: of the k_tokens
 * rows of k, v, dk, dv); starts that do not rise or leave the tensor are cut off at its ends.  Outputs at rows in front of the first
 * sequence and behind the last one are set to zero (lse to -inf), so that a buffer may be longer than its sequences together.  Without
 * starts (both NULL): `batch` sequences of q_tokens queries and k_tokens keys each.
 * lse: fp32 [heads][q_tokens] packed, [batch][heads][q_tokens] without starts; scores alike with kv_heads and k_tokens,
 * which for a dense batch is the layout that adore_init_cache takes as score_override in H2O mode.
 * Products are accumulated in fp32, softmax statistics are fp32, weights and their gradients are rounded to the storage
 * type where they enter a product; outputs are rounded once.  A row reaches what sees it and nothing else, infinities and NaN too
 * (later keys and values no earlier query, earlier queries no later key's gradients or scores); what the definition makes infinite
 * may come out as NaN.  A product of minus infinity has weight 0 (a row that has no other: out 0, lse -inf), one of plus infinity makes
 * its row NaN, lse too.  No atomics: equal inputs give equal bits.
 * Calls only enqueue work on hip_stream (a hipStream_t, NULL = the default stream), on the current device, which has to be the
 * buffers' (here and in the calls on a 4-bit cache).
 * Errors of all: E_INVALID (null, sizes, kv_heads that do not divide heads, a scale that is negative or not finite, one of
 * the two starts alone, rows not on 16-byte boundaries, a negative stride or a token stride beyond 2^22 elements),
 * E_UNSUPPORTED (head_dim not in {64,128}, more than 2^24 tokens, 4096 heads or 65536 sequences, 2^24 blocks of 32
 * tokens x heads or more), E_HIP. */
typedef struct {
  int32_t batch, heads, kv_heads, head_dim;
  int32_t q_tokens, k_tokens; /* rows of the packed tensors, or tokens of every sequence */
  int32_t dtype;              /* ADORE_F32 | ADORE_BF16: q, k, v, out and the gradients */
  float scale;                /* 0: 1 / sqrt(head_dim) */
} adore_prompt_config;

/* Where rows are: token t of sequence b, head h at data + b * seq + (start[b] + t) * token + h * head (elements; start[b] = 0
 * without starts), head_dim elements one behind the other. */
typedef struct {
  void *data; /* DEVICE, 16-byte aligned like every row */
  int64_t seq, token, head;
} adore_rows;

/* lse may be NULL.  rest, bf16 only, may be NULL: what rounding out to bf16 left, rounded to bf16 itself; the weights then
 * enter their product as two bf16 terms instead of one.  Handed to the backward pass it makes the gradients of rows with
 * few or sharp weights up to 1.6 times as exact. */
int adore_prompt_attention(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start,
                           const adore_rows *q, const adore_rows *k, const adore_rows *v, const adore_rows *out,
                           float *lse, const adore_rows *rest, void *hip_stream);

/* Gradients of sum(d_out . out) by q, k and v; dk and dv are summed over the heads of a group.  out, rest and lse as
 * adore_prompt_attention wrote them (rest may be NULL).  workspace: DEVICE, 256-byte aligned, at least
 * adore_prompt_backward_workspace_bytes(cfg, packed) bytes (packed != 0: with starts; 0 for a configuration that is not
 * taken), free to reuse after the work enqueued here has run.  dq, dk, dv may not alias the inputs.
 * Errors also: E_WORKSPACE. */
size_t adore_prompt_backward_workspace_bytes(const adore_prompt_config *cfg, int32_t packed);
int adore_prompt_attention_backward(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start,
                                    const adore_rows *d_out, const adore_rows *q, const adore_rows *k,
                                    const adore_rows *v, const adore_rows *out, const adore_rows *rest, const float *lse,
                                    const adore_rows *dq, const adore_rows *dk, const adore_rows *dv, void *workspace,
                                    size_t workspace_bytes, void *hip_stream);

/* scores (fp32): received_j.  lse as adore_prompt_attention wrote it for the same q and k. */
int adore_prompt_scores(const adore_prompt_config *cfg, const int32_t *q_start, const int32_t *k_start,
                        const adore_rows *q, const adore_rows *k, const float *lse, float *scores, void *hip_stream);

/* ---- A cache held in 4 bits, evicted by the attention its rows received (Sec. 3.1, baseline 6: H2O) ----
 * For prompts and answers whose cache should be small: 17/32 of a byte per element instead of 2 or 4, and `slots` rows per
 * (sequence, kv head), of which each holds its own tokens.  Stateless calls over four buffers of the caller's (DEVICE):
 *   cache     adore_q4_cache_bytes, 256-byte aligned: blocks of 64 slots, [batch][kv_heads][ceil(slots / 64)][68 * head_dim]
 *             bytes, laid out as csrc/q4_cache.hip says
 *   slot_pos  [batch][kv_heads][slots] i32: position of the token in the slot, -1 = free
 *   score     [batch][kv_heads][slots] fp32: the attention the slot's token has received, from all query heads of the group
 *   cursor    [batch][kv_heads][2] i32: the slot that the next token takes, its position
 * slot_pos, score 16-byte aligned, cursor 8.  An empty cache: slot_pos -1, score 0, cursor 0.
 * Values: 32 neighbouring elements of a row share a power of two, such that the largest of them is in (3.5, 7] of its
 * units (exponents from -100 to 125); an element is the nearest of 0, +-0.5, 1, 1.5, 2, 3, 4, 6 units, ties to the one with the even
 * code, larger ones to 6.  A NaN is held as 0.
 * Eviction: the next token takes the lowest free slot; a full row's next one to go is the token with the lowest score,
 * equal scores the lowest slot (in adore_q4_fill: position), never one of the `recent` last tokens.  (Elsewhere in this library equal
 * scores keep the older token; here tokens that received nothing make room for newer ones.)  A NaN score counts as 0.
 * Errors of all: E_INVALID (null, sizes, slots < 2, recent outside 1 .. slots - 1, a negative or infinite scale, misaligned
 * buffers), E_UNSUPPORTED (head_dim not in {64,128}, slots > 2^20, batch > 2^16, heads > 2^12, batch * kv_heads * blocks > 2^23,
 * batch * heads > 2^20), E_HIP. */
typedef struct {
  int32_t batch, heads, kv_heads, head_dim;
  int32_t slots, recent;
  int32_t dtype; /* ADORE_F32 | ADORE_BF16: q, k, v and outputs */
  float scale;   /* 0: 1 / sqrt(head_dim) */
} adore_q4_config;
size_t adore_q4_cache_bytes(const adore_q4_config *cfg);     /* HOST calls; 0 for a configuration that is not taken */
size_t adore_q4_workspace_bytes(const adore_q4_config *cfg); /* of adore_q4_step */

/* Loads prompts, by the eviction rule at once: of a sequence's n tokens the last `recent` and the best slots - recent of the
 * others stay (all if n <= slots), in slots of ascending position.  k, v as in adore_prompt_attention: packed with k_start
 * (k_tokens rows in all), or k_tokens per sequence.  scores (may be NULL: all 0): as adore_prompt_scores wrote them. */
int adore_q4_fill(const adore_q4_config *cfg, const int32_t *k_start, int32_t k_tokens, const adore_rows *k,
                  const adore_rows *v, const float *scores, void *cache, int32_t *slot_pos, float *score, int32_t *cursor,
                  void *hip_stream);

/* One token: k_new, v_new [batch][kv_heads][head_dim] go into the cursor's slots (score 0), then
 *   out[b][h][:] = sum_s softmax_s(scale q[b][h] . K[s]) V[s]   over the occupied slots, the new one as it is held,
 * q, out [batch][heads][head_dim] storage type; every slot's score grows by the weights its group's heads gave it (fp32), and the
 * cursor moves to the next token.  k_held, v_held [batch][kv_heads][head_dim] or NULL: the new row as it is held.
 * bf16: products are exact, a weight times its power of two is within 2^-16; fp32: 2^-23.
 * workspace: 256-byte aligned, at least adore_q4_workspace_bytes(cfg) bytes, free to reuse after the work enqueued here has run.
 * Errors also: E_WORKSPACE. */
int adore_q4_step(const adore_q4_config *cfg, const void *q, const void *k_new, const void *v_new, void *cache,
                  int32_t *slot_pos, float *score, int32_t *cursor, void *out, void *k_held, void *v_held, void *workspace,
                  size_t workspace_bytes, void *hip_stream);

/* What the cache holds: k, v [batch][kv_heads][slots][head_dim] storage type, zeros in free slots. */
int adore_q4_read(const adore_q4_config *cfg, const void *cache, const int32_t *slot_pos, void *k, void *v, void *hip_stream);

const char *adore_strerror(int code);
/* Debug aid for callers and tests, not a step of the method (no passage of the paper): with ADORE_GUARD_WORDS=1
 * in the environment of the process, adore_workspace_bytes and adore_create lay the workspace out with 256 bytes of
 * a fixed pattern behind each of its regions (cache, slot maps, scores, lists, scratch).  No kernel has a reason to
 * touch them; a kernel that writes past the end of a region does.  adore_check_guards waits for the context's
 * streams and writes to *damaged (host) the number of 4-byte guard words that no longer hold the pattern: 0 after
 * any sequence of calls, -1 if the context has no guard words (the variable was not set at create, or no call has
 * touched the GPU yet).  Errors: E_INVALID (null), E_HIP. */
int adore_check_guards(adore_ctx *ctx, int32_t *damaged);

int adore_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ADORE_H */
