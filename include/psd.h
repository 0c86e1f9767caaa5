/*
 * psd.h -- C ABI of the MI355X (gfx950) library for the Parallel Speculative Decoding
 * (PSD) denoising step of masked-diffusion language models.
 *
 * One loop iteration of the paper's Alg. 1 is
 *     stage 1  forward -> (x_hat, c) on the masked positions of the active block  (Sec. 3.1)
 *              T = pi(x, c); commit x_hat on T                                      (Eq. 1)
 *     stage 2  sigma = residual masks by step-t confidence; K drafts               (Eq. 2)
 *     stage 3  one batched forward over the K drafts; hierarchical acceptance over
 *              the draft DAG; advance to the deepest accepted draft                 (Sec. 3.2)
 * and every step runs in hand-written HIP kernels behind the calls below.
 *
 * Conventions
 *   - Every function returns an int32 status: PSD_OK (0) or a negative PSD_ERR_*.
 *     Arguments are validated on the host before anything is enqueued; on error nothing
 *     is launched and no output is written.  psd_last_error() gives a message.
 *   - "device" pointers are HIP device memory owned by the caller (any allocator).
 *     "host" pointers are ordinary host memory.  The library allocates device memory only
 *     inside psd_create (for bf16 models a second copy of the LM-head matrix in MFMA-fragment
 *     order, vocab*d_model*2 bytes) and frees it in psd_destroy.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls
 *     enqueue asynchronously and do not synchronise, except psd_decode_block, which
 *     returns host statistics and reads small counters back once per iteration.
 *   - Layouts are row-major.  tokens int32 [B, N]; the active block is positions
 *     block_start .. block_start+L-1 of every sequence (1 <= L <= 64; the step calls take one block_start for
 *     the batch, psd_decode_block and psd_decode one per sequence).  Per-block tables
 *     are top1 int32 [B, L] and conf float [B, L]: a masked position carries the
 *     prediction, any other position the sentinel (its own token, -1.0f).
 *   - Sequences of a batch are independent.  In the whole-sequence calls batching never changes a sequence's
 *     logits or top-1 tokens; the confidence normaliser is summed in an order that depends on the number of rows
 *     in the call, so confidences can differ in the last fp32 bit between batch shapes.  The block-row calls
 *     (psd_*_cached, psd_*_approx) cut the output and down projections along K when a call has at most 128 rows,
 *     so there a sequence's fp32 sums, and with near-tied confidences its decisions, can depend on how many
 *     sequences or drafts share the call; results agree to fp32 rounding of those sums.
 *   - Token ids outside [0, vocab) are invalid input: they read a zero embedding row (no fault).  A block row
 *     whose logits are all non-finite has no prediction: it yields (token 0, confidence 0).
 */
#ifndef PSD_H
#define PSD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PSD_OK               0
#define PSD_ERR_INVALID_ARG -1
#define PSD_ERR_SHAPE       -2
#define PSD_ERR_WORKSPACE   -3
#define PSD_ERR_DEVICE      -4
#define PSD_ERR_UNSUPPORTED -5

#define PSD_MAX_NODES 32   /* K, root included */
#define PSD_MAX_BLOCK 64   /* L */

#define PSD_DTYPE_FP32 0   /* debug path: fp32 storage and arithmetic, plain kernels */
#define PSD_DTYPE_BF16 1   /* bf16 storage, MFMA contractions with fp32 accumulation */
#define PSD_ATTN_BIDIRECTIONAL 0
#define PSD_ATTN_BLOCK_CAUSAL 1

typedef struct psd_handle psd_handle;

/* Model layout.  The paper only requires a bidirectional transformer that yields a
 * distribution per position (Sec. 3.1); this is the pre-norm RMSNorm / rotary / SwiGLU
 * decoder stack of the benchmarked 7-8B models, run without a causal mask. */
typedef struct {
    int32_t n_layers, d_model, n_heads, n_kv_heads, d_head, d_ffn, vocab;
    int32_t mask_id;       /* id of [M]; it has an embedding row but is never predicted */
    float   rms_eps;
    int32_t qkv_bias;      /* 1: bq/bk/bv present */
    int32_t dtype;         /* PSD_DTYPE_*: type of every weight matrix */
    float   logit_scale;   /* logits = logit_scale * (y W_lm^T); 1.0 normally */
    int32_t max_seq;       /* rows of the rotary tables */
    int32_t attention;     /* PSD_ATTN_*: bidirectional (default 0), or context-causal blocks (App. A: full
                            * attention inside a block of the decoding block length, causal across blocks) */
} psd_model_config;

/* Device pointers, borrowed for the life of the handle.  Matrices are [out, in] in the
 * model dtype; norm gains, biases and rotary tables are fp32.  The per-layer members are
 * host arrays of n_layers device pointers (copied by psd_create). */
typedef struct {
    const void  *tok_emb;      /* [vocab, d_model] */
    const float *final_norm;   /* [d_model] */
    const void  *lm_head;      /* [vocab, d_model] */
    const float *rope_cos;     /* [max_seq, d_head/2], cos(pos * theta^(-2j/d_head)) */
    const float *rope_sin;     /* [max_seq, d_head/2]; pairs are (j, j + d_head/2) */
    const float *const *attn_norm;   /* [d_model] */
    const void  *const *wq;          /* [n_heads*d_head, d_model] */
    const void  *const *wk;          /* [n_kv_heads*d_head, d_model] */
    const void  *const *wv;          /* [n_kv_heads*d_head, d_model] */
    const float *const *bq, *const *bk, *const *bv;   /* NULL arrays when qkv_bias == 0 */
    const void  *const *wo;          /* [d_model, n_heads*d_head] */
    const float *const *ffn_norm;    /* [d_model] */
    const void  *const *w_gate;      /* [d_ffn, d_model] */
    const void  *const *w_up;        /* [d_ffn, d_model] */
    const void  *const *w_down;      /* [d_model, d_ffn], row stride w_down_stride */
    int32_t w_down_stride;           /* elements between rows of w_down; 0 = d_ffn (dense).  A multiple of 8.
                                      * Rows padded by 64 elements avoid cache-channel conflicts on MI355X
                                      * when a dense row is a multiple of 8 KB (d_ffn = 12288). */
} psd_weights;

/* Transfer policy pi (Sec. 3.2 stage 1; App. B.2): over the masked positions of the block,
 * ordered by confidence descending (ties: lower position first), commit every position
 * with c > tau plus the k_min most confident; if k_max > 0 at most the k_max most
 * confident of those.  Greedy decoding: tau = +inf, k_min = 1.  Confidence Parallel
 * Decoding: tau = 0.9, k_min = 1.  The same rule is the acceptance criterion A_pi. */
typedef struct {
    float   tau;
    int32_t k_min;
    int32_t k_max;   /* 0 = unbounded */
    /* EOS early stopping of psd_decode_block / psd_decode_block_cached (evaluation protocol of
     * App. B.1; the other calls ignore both fields).  eos_stop = 0: off.  eos_stop = 1: a sequence
     * stops as soon as an EOS token has been produced: after every update of its state (the stage-1
     * commit; the advance with its post-verification commit) its block is searched for eos_id, and
     * if it is there the sequence takes part in no further model call, whatever is still masked. */
    int32_t eos_stop;
    int32_t eos_id;  /* 0 <= eos_id < vocab, not the mask token (checked when eos_stop = 1) */
    /* Block loops only (psd_decode, psd_decode_block, psd_decode_block_cached); 0 = the literal Alg. 1.
     * 1 = a variant that is NOT the literal Alg. 1 and gives different results in general: the last line
     * of stage 3 commits, by pi, predictions of the accepted draft k* -- the literal loop then calls the
     * model again on the committed state (stage 1 of the next iteration).  The variant takes that
     * post-verification commit as the next iteration's stage-1 commit and draws the next speculative
     * ordering and drafts from k*'s verifier output (x_hat_k*, c_k*), the model's exact prediction on the
     * state just before that commit.  An iteration then costs one model call, the batched verification;
     * only the call that enters a block is a stage-1 call.  Every committed token still comes from an
     * exact forward of an exact state.  The tables live for one library call: each call starts with a
     * stage-1 call for every sequence (so max_iterations = 1 gains nothing). */
    int32_t single_forward;
} psd_policy;

/* Draft DAG (Sec. 3.2 stage 2).  Node k speculates on the ranks of the speculative
 * ordering sigma whose bits are set in rank_set[k] (bit r <-> sigma_{r+1}); node 0 is the
 * root with rank_set[0] = 0.  Edges are implied: (p, k) is an edge iff S_p is a strict
 * subset of S_k.  Ranks >= m (the number of residual masks) are ignored. */
typedef struct {
    int32_t  K;
    uint64_t rank_set[PSD_MAX_NODES];
} psd_graph;

/* Per-sequence counters of psd_decode_block.  TPF = tokens / invocations with
 * tokens = tokens_policy + tokens_draft + tokens_postverify; a batched verification
 * counts as one invocation (Sec. 4.1 "Metrics"). */
typedef struct {
    int64_t invocations;
    int64_t tokens_policy;       /* committed by pi in stage 1 */
    int64_t tokens_draft;        /* |S_k*| of the accepted drafts */
    int64_t tokens_postverify;   /* committed by pi on k*'s verifier output */
    int32_t depth_hist[PSD_MAX_NODES + PSD_MAX_BLOCK + 1];   /* histogram of |S_k*| */
    /* App. B.1: tokens up to and including the EOS position.  tokens_counted grows by the number of
     * block positions the call resolved at or before the first EOS token of the block (tokens
     * unmasked beyond it are discarded, whenever they were unmasked); by all it resolved when the
     * call did not stop on an EOS.  stopped is set to 1 and eos_pos to the sequence position of that
     * first EOS token when it did; both are left alone otherwise. */
    int64_t tokens_counted;
    int32_t stopped;
    int32_t eos_pos;
} psd_stats;

const char *psd_status_string(int32_t status);
/* sizeof of the structures above as this library was built, in the order psd_model_config, psd_weights,
 * psd_policy, psd_graph, psd_stats, psd_work, psd_graph_score, psd_debug_layout (the first n of them into out; returns how many
 * there are): lets a foreign-language binding check its own declarations. */
int32_t psd_struct_sizes(int32_t *out, int32_t n);
/* Message of the last error raised on the calling thread ("" if none). */
const char *psd_last_error(void);

/* Creates a handle on the current HIP device.  Fails with PSD_ERR_DEVICE when no gfx950
 * device is present, PSD_ERR_SHAPE / PSD_ERR_UNSUPPORTED on layouts the kernels do not
 * cover (bf16 needs d_head in {64, 128} and d_model, d_ffn multiples of 64; fp32 takes
 * any even d_head). */
int32_t psd_create(const psd_model_config *cfg, const psd_weights *w, psd_handle **out);
int32_t psd_destroy(psd_handle *h);

/* Bytes of device workspace that a forward over up to max_seqs sequences of length N with
 * block length L needs (psd_verify_accept and psd_decode_block run max_seqs = B*K).
 * Negative status on bad arguments. */
int64_t psd_workspace_bytes(const psd_model_config *cfg, int32_t max_seqs, int32_t N, int32_t L);

/* Prefix chain: node k speculates on the k*width most confident residual positions. */
int32_t psd_graph_chain(int32_t K, int32_t width, psd_graph *out);
/* Subset lattice: one node for every subset of the `depth` most confident residual positions
 * (2^depth nodes, ordered by size): the densest multi-parent DAG over those positions -- a
 * deeper draft can be reached through every order of unmasking (Sec. 3.2 stage 2).  depth 0..5. */
int32_t psd_graph_lattice(int32_t depth, psd_graph *out);

/* Model call (Sec. 3.1; Alg. 1 stage 1 and the batched pass of stage 3): forward S
 * sequences over all N positions with bidirectional attention, then on the L block rows of
 * each the top-1 token x_hat = argmax_v p(v) and confidence c = max_v p(v), p the softmax
 * of the logits over the vocabulary without [M].  Ties go to the lowest token id.  The
 * logits are reduced on the fly and never stored.
 *   tokens device int32 [S, N] (read); top1 device int32 [S, L], conf device float [S, L]
 *   (written); ws device, ws_bytes >= psd_workspace_bytes(cfg, S, N, L). */
int32_t psd_forward_confidence(psd_handle *h, const int32_t *tokens, int32_t S, int32_t N,
                               int32_t block_start, int32_t L, int32_t *top1, float *conf,
                               void *ws, int64_t ws_bytes, void *stream);

/* Debug companion of psd_forward_confidence: writes the raw block logits
 * logit_scale * (y W_lm^T), [M] column included, as float [S*L, vocab] (device).  Only for
 * numeric parity checks; the decode path never materialises logits. */
int32_t psd_forward_logits(psd_handle *h, const int32_t *tokens, int32_t S, int32_t N,
                           int32_t block_start, int32_t L, float *logits,
                           void *ws, int64_t ws_bytes, void *stream);

/* Debug switch for numeric cross-checks: bit 0 runs the layer contractions, bit 1 the
 * attention, bit 2 the LM-head on the plain (non-MFMA) kernels; bit 3 keeps the rotary embedding and the
 * transpose of V in a kernel of their own instead of the QKV projection's epilogue (same bits either way); bit 4
 * takes the entries that a refresh stores in the approximate cache from the row-major values instead of the
 * transposed ones (same bits too).
 * 0 (default) = MFMA path. */
int32_t psd_debug_set_plain(psd_handle *h, int32_t mask);

/* Debug hook for parity checks of one layer at full width: runs layer `layer` of the model alone on a residual
 * stream supplied by the caller -- hidden, device float [S*N, d_model], updated in place as one layer of the forward
 * would (Sec. 3.1 only asks for a bidirectional transformer; the layer is RMSNorm, QKV, rotary, attention over the
 * sequence's N rows, output projection, RMSNorm, SwiGLU, down projection, with the kernels and tiles the forward picks
 * for S*N rows).  stop_after = 1 stops once the attention output is written and leaves hidden untouched.  The
 * intermediates stay in the workspace, where psd_debug_workspace_layout says (byte offsets; row strides in elements
 * of the model dtype): a = output of the last norm that ran [S*N, d_model]; qkv = projections with rotary applied
 * [S*N, ld_qkv]; vT = values transposed, [S, n_kv_heads*d_head, ld_vt] with the keys of every group of 16 in the
 * order 0-3, 8-11, 4-7, 12-15; o = attention output [S*N, n_heads*d_head]; act = SwiGLU output [S*N, ld_act].
 * ws as for psd_forward_confidence(S, N, L).  Honours psd_debug_set_plain. */
typedef struct {
    int64_t off_a, off_qkv, off_vt, off_o, off_act;
    int32_t ld_qkv, ld_act, ld_vt, reserved;
} psd_debug_layout;
int32_t psd_debug_workspace_layout(const psd_model_config *cfg, int32_t S, int32_t N, int32_t L, psd_debug_layout *out);
int32_t psd_debug_layer(psd_handle *h, int32_t layer, float *hidden, int32_t S, int32_t N, int32_t L, int32_t stop_after,
                        void *ws, int64_t ws_bytes, void *stream);

/* Debug / tuning: forces the workgroup tile of the layer contractions (see psd_probe_begin
 * and psd_kernel_gemm_tile_name for the numbering; -1 = pick per shape; a tile that cannot run the
 * epilogue asked for is ignored).  Process-wide. */
int32_t psd_debug_force_gemm_tile(int32_t tile);
/* Debug: what the dispatcher does with a contraction of this shape on aligned operands.  psd_debug_gemm_plan returns the kernel as
 * psd_probe_begin numbers it, and in *parts (may be NULL) the parts along K that a cached call cuts a residual contraction into;
 * psd_debug_qkv_cut the first column that the QKV projection of whole sequences leaves to a second launch (0: one launch).
 * psd_debug_gemm_cut: the other contractions over more than 128 rows; *rows / *cols of the first of two launches (both 0: one launch).
 * psd_debug_qkv_fused: 1 where the QKV projection of packed weights rotates and transposes in its epilogue (into a KV cache or not), 0 in two passes.
 * psd_debug_gemm_ahead: the workgroups that the last launch of such a contraction adds to read the next weights ahead.
 * psd_debug_head_plan: the LM-head pass of a bf16 model over `rows` hidden rows; *ids x *width the tile, returns 1 where the forward streams a
 * packed copy of the matrix instead, 0 otherwise. */
int32_t psd_debug_gemm_plan(int64_t M, int32_t Nout, int32_t Kin, int32_t epilogue, int32_t *parts);
int32_t psd_debug_gemm_cut(int64_t M, int32_t Nout, int32_t Kin, int32_t epilogue, int64_t *rows, int64_t *cols);
int32_t psd_debug_qkv_fused(int64_t M, int32_t Nout, int32_t Kin, int32_t d_head, int32_t v_start, int32_t rows_per_seq, int32_t into_cache);
int32_t psd_debug_gemm_ahead(int64_t M, int32_t Nout, int32_t Kin, int32_t epilogue);
int32_t psd_debug_head_plan(int32_t rows, int32_t vocab, int32_t d, int32_t *ids, int32_t *width);
int32_t psd_debug_qkv_cut(int64_t M, int32_t Nout, int32_t Kin, int32_t d_head, int32_t v_start, int32_t rows_per_seq);
/* Optional: the block loops (psd_decode, psd_decode_block) replay the whole-sequence model calls of a shape they have
 * seen twice as HIP graphs.  Results are bit-identical to eager launches.  Off by default: on the one workload where
 * a model call is ~75 kernels of 4-11 microseconds (8 layers, d_model 512) the queue already runs them back to back and
 * the graph changes nothing (119 ms per decode either way); the time goes to the kernels' own floor, not to launches.
 * enabled = 1 / 0 switches it on / off for the handle, a negative value leaves it; replays (may be NULL) receives the
 * number of graph launches so far.  A graph holds the addresses the call was captured with (tokens, tables, workspace):
 * up to 24 distinct calls are kept, least recently used replaced.  Calls that are being timed by psd_probe_begin and
 * the KV-cached calls always launch eagerly. */
int32_t psd_debug_set_graphs(psd_handle *h, int32_t enabled, int64_t *replays);

/* Stage 1 commit (Eq. 1): applies pi to every sequence in place.
 *   tokens device int32 [B, N] (updated); top1/conf device [B, L] (read);
 *   transfer_mask device uint8 [B, L] (1 where committed); n_selected device int32 [B]. */
int32_t psd_select_unmask(psd_handle *h, int32_t *tokens, int32_t B, int32_t N, int32_t block_start,
                          int32_t L, const int32_t *top1, const float *conf, const psd_policy *policy,
                          uint8_t *transfer_mask, int32_t *n_selected, void *stream);

/* Stage 2 (Eq. 2): from the post-commit tokens and the step-t (top1, conf): the
 * speculative ordering sigma (block-local positions, confidence descending, ties lower
 * position first, padded with -1), the residual count m, and the K drafts.
 *   tokens device int32 [B, N] (read); sigma device int32 [B, L]; m device int32 [B];
 *   drafts device int32 [B, K, N] (written). */
int32_t psd_build_drafts(psd_handle *h, const int32_t *tokens, int32_t B, int32_t N, int32_t block_start,
                         int32_t L, const int32_t *top1, const float *conf, const psd_graph *graph,
                         int32_t *sigma, int32_t *m, int32_t *drafts, void *stream);

/* Hierarchical acceptance and state advance on given verifier outputs (Alg. 1 stage 3
 * without the model call).  Node k is accepted iff some accepted p with S_p a strict
 * subset of S_k has, on every position i of S_k \ S_p, v_top1[p, i] equal to the drafted
 * token and i committed by pi applied to p's verifier output.  k* is the accepted node
 * with the largest S (ties: lowest index); tokens <- draft k*, then pi is applied once more
 * on k*'s verifier output.  Sequences with m == 0 are left untouched (k_star = 0).
 *   tokens device int32 [B, N] (written); drafts device int32 [B, K, N]; sigma device
 *   [B, L]; m device [B]; v_top1 / v_conf device [B, K, L]; k_star device int32 [B];
 *   accepted device uint8 [B, K]. */
int32_t psd_accept(psd_handle *h, int32_t *tokens, const int32_t *drafts, int32_t B, int32_t N,
                   int32_t block_start, int32_t L, const int32_t *sigma, const int32_t *m,
                   const psd_graph *graph, const psd_policy *policy, const int32_t *v_top1,
                   const float *v_conf, int32_t *k_star, uint8_t *accepted, void *stream);

/* Stage 3 whole (Sec. 3.2): one batched forward over the B*K drafts (one invocation),
 * then psd_accept on its outputs, which are also returned in v_top1 / v_conf [B, K, L].
 * ws_bytes >= psd_workspace_bytes(cfg, B*K, N, L). */
int32_t psd_verify_accept(psd_handle *h, int32_t *tokens, const int32_t *drafts, int32_t B, int32_t N,
                          int32_t block_start, int32_t L, const int32_t *sigma, const int32_t *m,
                          const psd_graph *graph, const psd_policy *policy, int32_t *k_star,
                          uint8_t *accepted, int32_t *v_top1, float *v_conf,
                          void *ws, int64_t ws_bytes, void *stream);

/* Alg. 1 on one block of each of B sequences: sequence b decodes the block [block_start[b], block_start[b]+L) until
 * it has no masked position left (block_start: host int32 [B]; the sequences need not be on the same block).  An
 * iteration is one stage-1 model call over the sequences still running and one batched verification call over the K
 * drafts of those that keep masks after the stage-1 commit; sequences that finish early drop out of the model calls.
 * Blocks until done.  tokens device int32 [B, N] (updated in place);
 * stats host psd_stats [B], counters are ADDED to what it holds (zero it first);
 * ws_bytes >= psd_workspace_bytes(cfg, B*K, N, L) + psd_decode_scratch_bytes(B, N, L, K). */
int32_t psd_decode_block(psd_handle *h, int32_t *tokens, int32_t B, int32_t N, const int32_t *block_start,
                         int32_t L, const psd_policy *policy, const psd_graph *graph, psd_stats *stats,
                         void *ws, int64_t ws_bytes, void *stream);
/* The whole semi-autoregressive generation (Alg. 1 per block; App. B.1: blocks left to right, the next block of a
 * sequence starts once its current one is fully resolved; with policy->eos_stop a sequence ends with the block in
 * which an EOS token was produced).  block_start: host int32 [B], in and out: the first position of every sequence's
 * current block on entry (N - block_start[b] a multiple of L; block_start[b] >= N: nothing left to do), and where
 * the sequence stands on return (>= N when it reached the end).  Every sequence advances through its own blocks: a
 * sequence that resolves its block moves on in the next iteration while the others continue, so the model calls
 * keep all running sequences in one batch.  max_iterations > 0 returns after that many iterations of the batch
 * (0: until every sequence is done); *iterations_done (host, may be NULL) receives the number run.  A later call
 * continues from tokens and block_start as they stand.  Workspace and stats as for psd_decode_block; with
 * max_iterations > 0 and EOS stopping, tokens_counted of a call counts what that call resolved at or before the
 * first EOS its block holds by the end of the call. */
int32_t psd_decode(psd_handle *h, int32_t *tokens, int32_t B, int32_t N, int32_t *block_start, int32_t L,
                   const psd_policy *policy, const psd_graph *graph, psd_stats *stats, int32_t max_iterations,
                   int32_t *iterations_done, void *ws, int64_t ws_bytes, void *stream);
int64_t psd_decode_scratch_bytes(int32_t B, int32_t N, int32_t L, int32_t K);

/* ---- Context-causal block attention with an exact prefix KV cache ------------------------------
 * One model family of the paper (App. A, the continually pretrained block-diffusion model) attends
 * fully inside a block and causally across blocks.  With config.attention = PSD_ATTN_BLOCK_CAUSAL
 * (blocks = the decoding blocks, from position 0; prompt length a multiple of the block length):
 *   - the calls above still work on whole sequences (masked attention on the plain kernels: the
 *     on-device reference for this mode);
 *   - the calls below run the model on the L rows of the active block only.  Everything before the
 *     block is finished, so its keys and values are exact in a cache, and nothing after it is
 *     visible.  The K drafts of a verification batch share their sequence's cache (the "KV-cache
 *     sharing" of Sec. 3.2 stage 3, lossless here).
 * The cache is caller-owned device memory, psd_kv_cache_bytes(cfg, capacity) bytes per sequence,
 * sequences back to back, 256-byte aligned; per layer it holds the rotated keys
 * [capacity, n_kv_heads*d_head] and the values transposed.  It must be zeroed (psd_kv_reset) before a
 * sequence starts.  Its length is not stored: a call's block_start says how many positions it holds,
 * and psd_kv_prefill / psd_decode_block_cached extend it block by block.  Block lengths must be
 * multiples of 16.  Workspace: psd_workspace_bytes(cfg, sequences, L, L) (+ the decode scratch).
 *   psd_kv_prefill: forwards positions [0, n_prompt) of tokens [B, N] and fills the caches, in as few passes over whole blocks as
 *     the workspace allows, cut evenly: psd_workspace_bytes(cfg, B, L, L) at least, psd_workspace_bytes(cfg, B, n_prompt, L) for
 *     one pass.
 *   psd_forward_confidence_cached: tokens device int32 [S, N], only positions block_start .. +L are
 *     read; sequence s uses cache s / seqs_per_cache; writes top1/conf [S, L] (both or neither) and,
 *     if logits != NULL, the raw block logits [S*L, vocab] (debug).
 *   psd_decode_block_cached: psd_decode_block with cached model calls; afterwards the finished block
 *     is appended to the caches (one more forward over the B blocks, not counted as an invocation:
 *     it decodes nothing). */
int64_t psd_kv_cache_bytes(const psd_model_config *cfg, int32_t capacity);
int32_t psd_kv_reset(psd_handle *h, void *cache, int32_t n_seqs, int32_t capacity, void *stream);
int32_t psd_kv_prefill(psd_handle *h, const int32_t *tokens, int32_t B, int32_t N, int32_t n_prompt, int32_t L,
                       void *cache, int32_t capacity, void *ws, int64_t ws_bytes, void *stream);
int32_t psd_forward_confidence_cached(psd_handle *h, const int32_t *tokens, int32_t S, int32_t N, int32_t block_start,
                                      int32_t L, int32_t seqs_per_cache, const void *cache, int32_t capacity,
                                      int32_t *top1, float *conf, float *logits, void *ws, int64_t ws_bytes,
                                      void *stream);
int32_t psd_decode_block_cached(psd_handle *h, int32_t *tokens, int32_t B, int32_t N, int32_t block_start, int32_t L,
                                const psd_policy *policy, const psd_graph *graph, psd_stats *stats, void *cache,
                                int32_t capacity, void *ws, int64_t ws_bytes, void *stream);

/* ---- Keys that a batch shares, the weights they draw, and eviction by those weights ------------
 * Requests that begin with the same text need its keys and values once.  Here the keys that a row attends to come in segments,
 * coarse to fine: a prefix of the whole batch, the cache of a request (shared by its drafts), the rows of a block.  A segment
 * has S / seqs_per_unit units; sequences u * seqs_per_unit .. + seqs_per_unit - 1 see unit u of it, all of its keys.
 * Unit u: keys k + u * stride_k, key j in row j (row stride ld_k), channels of KV head g from g * d_head on; values transposed,
 * vt + u * stride_vt, row g * d_head + c (row stride ld_vt) the values of channel c with the keys of every group of 16 in the order
 * 0-3, 8-11, 4-7, 12-15 -- one layer of a KV cache as psd_kv_cache_bytes lays it out is such a unit.  What lies behind the
 * last key is never used.  Strides are in elements.  Rows are 16-byte aligned, rows of values hold whole groups of 16 keys. */
#define PSD_MAX_SEGMENTS 4
typedef struct {
    const void *k, *vt;          /* device, in the dtype of the call */
    const int32_t *lens;         /* device int32, keys of every unit (cut to 0 .. len), or NULL: each unit holds len */
    float *weights;              /* device: [units] stride_w apart, [n_kv_heads] ld_w apart, one per key; or NULL */
    int64_t stride_k, stride_vt, stride_w;
    int32_t ld_k, ld_vt, ld_w;
    int32_t len;                 /* keys of a unit, or the most that any unit holds (0: the segment is skipped); up to 2^30 */
    int32_t seqs_per_unit;       /* a multiple of the next segment's; that of the first divides S */
    int32_t reserved;            /* 0 */
} psd_kv_segment;
/* Rows of the attention: S sequences of L rows (1 .. 64), row i of sequence s at q + (s*L + i) * ld_q, n_heads heads of d_head.
 * dtype PSD_DTYPE_BF16: d_head 64 or 128; PSD_DTYPE_FP32: 16, 32, 64 or 128. */
typedef struct {
    int32_t S, L, n_heads, n_kv_heads, d_head, dtype;
    int64_t ld_q, ld_out;
} psd_attention_shape;
/* sizeof psd_kv_segment, psd_attention_shape and psd_kv_shared, as psd_struct_sizes gives those of the structures above. */
int32_t psd_shared_struct_sizes(int32_t *out, int32_t n);
/* psd_attention_shared: softmax(q k^T / sqrt(d_head)) v of every row over all keys of the units it sees.  out as q (row stride
 *   ld_out); lse device float [S*L, n_heads], ln of the sum of the exponentials of its scores, or NULL.  Neither may overlap an input or the
 *   other (q, keys and out may be columns of one buffer's rows).  A row without a key (all lengths 0), or without a score above -inf, gets
 *   zeros and lse -inf, and draws no weight.  ws: device, 256-byte aligned, psd_attention_shared_bytes of the same shape and segments (which
 *   looks at shapes and len only, not at device memory); calls that overlap need one each.  Sums and statistics are fp32; with bf16 the probabilities are rounded to bf16 before they meet the values.  How keys are cut follows shapes and lengths, so a row's
 *   bits depend on those of its batch, but not on what other sequences hold.
 * psd_attention_weights: what each key drew: weights[u][g][j] = sum over the rows of the unit's sequences and the query heads of KV head g
 *   of exp(score - lse), lse from psd_attention_shared over all segments (a float: a row's weights are off by a factor within |lse| 2^-21, and
 *   where that says nothing any more, beyond |lse| = 2^24, each is at least between 0 and 1).  Segments without `weights` are skipped, no two may share any; accumulate = 1
 *   adds to what is there, 0 overwrites.  Weights behind a unit's last key are left as they are.  ws likewise
 *   (psd_attention_weights_bytes; may be NULL where that is 0). */
int64_t psd_attention_shared_bytes(const psd_attention_shape *shape, const psd_kv_segment *segments, int32_t n_segments);
int32_t psd_attention_shared(const psd_attention_shape *shape, const void *q, const psd_kv_segment *segments, int32_t n_segments, void *out,
                             float *lse, void *ws, int64_t ws_bytes, void *stream);
/* Debug: how psd_attention_shared splits its work.  For the first n_jobs jobs 7 numbers each: first segment (of those with keys), segments,
 *   form (0: up to 32 rows a workgroup, 1: 128 rows, 2: a unit and KV head to a wavefront), units, tiles of rows of a unit and KV head, parts
 *   of the keys, and the rows of a unit and KV head.  Returns the number of jobs. */
int32_t psd_debug_attention_plan(const psd_attention_shape *shape, const psd_kv_segment *segments, int32_t n_segments, int32_t *jobs, int32_t n_jobs);
int64_t psd_attention_weights_bytes(const psd_attention_shape *shape, const psd_kv_segment *segments, int32_t n_segments);
int32_t psd_attention_weights(const psd_attention_shape *shape, const void *q, const psd_kv_segment *segments, int32_t n_segments,
                              const float *lse, int32_t accumulate, void *ws, int64_t ws_bytes, void *stream);
/* psd_kv_evict: of `units` units of src (seqs_per_unit is ignored) and every KV head the `keep` (1 .. 2^30) positions with the largest weights: the first n_first
 *   and the last n_last positions of a unit always (n_first + n_last <= keep), then by src->weights, descending, equal ones the
 *   lowest position first (both zeros are equal, NaN is below everything).  They go to dst in ascending order of their positions: keys, values and, where
 *   dst->weights is set, weights; a unit of at most `keep` positions is copied whole.  dst must hold min(keep, src->len) positions (its `len`), have
 *   lens NULL, and not overlap src; its units lie behind one another, or beside each other in rows that hold all of them; what lies behind
 *   the positions written is left as it is.  kept device int32 [units][n_kv_heads][keep]: the source position of each, -1 behind the last; kept_lens device int32 [units] (or NULL): positions of each unit now.
 *   Results share no memory with each other or with what is read, lens among it.
 *   The layers of the caches of n sequences are n * n_layers units in a row.  d_head * element size a multiple of 16 bytes. */
int32_t psd_kv_evict(const psd_kv_segment *src, const psd_kv_segment *dst, int32_t units, int32_t n_kv_heads, int32_t d_head, int32_t dtype,
                     int32_t keep, int32_t n_first, int32_t n_last, int32_t *kept, int32_t *kept_lens, void *stream);

/* Model calls whose block rows attend to a prefix that the whole batch shares, then to the cache of their sequence, then to their block.
 * All caches hold the same number of positions, all layers and heads of a cache too; caches that were cut to lengths of their own
 * (psd_kv_evict with lens) are for psd_attention_shared.
 * Both caches are laid out like the exact one (psd_kv_cache_bytes(cfg, capacity) per sequence; the prefix is one), and their positions
 * count as they lie: rotary positions are in the keys, so a cache may have gaps (psd_kv_evict), and the block's rows sit at positions block_start .. of
 * tokens whatever the caches hold.  A prefix is filled by psd_kv_prefill with B = 1, a sequence's cache behind it by psd_kv_extend_shared.
 * Block-causal models: exact while nothing is evicted.  Bidirectional models: the caches of psd_forward_confidence_approx, whole or evicted.
 *   psd_forward_confidence_shared: as psd_forward_confidence_cached; sequence s uses cache s / seqs_per_cache.  What every cached
 *     position drew from the block rows, layer by layer, is added to prefix_weights / cache_weights (zero them first; they may share none) where set.
 *   psd_kv_extend_shared: one forward over the block rows of B sequences (seqs_per_cache 1), whose keys and values go to positions len ..
 *     len + L - 1 of their caches.  Block-causal models only; adds no weights.
 *   psd_decode_block_shared: psd_decode_block with such model calls; afterwards the block is appended as by psd_kv_extend_shared.
 * L a multiple of 16.  Workspace: psd_shared_workspace_bytes(cfg, S, L, kv), 256-byte aligned; for psd_decode_block_shared with S = B*K and
 * kv->seqs_per_cache = K there (1 in the call), plus psd_decode_scratch_bytes(B, N, L, K). */
typedef struct {
    const void *prefix;          /* device, one cache, none of those that a block goes behind; may be NULL where prefix_len is 0 */
    void *cache;                 /* device, one per seqs_per_cache sequences; may be NULL where len is 0 and nothing is stored */
    float *prefix_weights;       /* device [n_layers][n_kv_heads][prefix_capacity], or NULL */
    float *cache_weights;        /* device [caches][n_layers][n_kv_heads][capacity], or NULL */
    int32_t prefix_capacity, prefix_len, capacity, len, seqs_per_cache;
    int32_t reserved;            /* 0 */
} psd_kv_shared;
int64_t psd_shared_workspace_bytes(const psd_model_config *cfg, int32_t S, int32_t L, const psd_kv_shared *kv);
int32_t psd_forward_confidence_shared(psd_handle *h, const int32_t *tokens, int32_t S, int32_t N, int32_t block_start, int32_t L,
                                      const psd_kv_shared *kv, int32_t *top1, float *conf, float *logits, void *ws, int64_t ws_bytes,
                                      void *stream);
int32_t psd_kv_extend_shared(psd_handle *h, const int32_t *tokens, int32_t B, int32_t N, int32_t block_start, int32_t L,
                             const psd_kv_shared *kv, void *ws, int64_t ws_bytes, void *stream);
int32_t psd_decode_block_shared(psd_handle *h, int32_t *tokens, int32_t B, int32_t N, int32_t block_start, int32_t L,
                                const psd_policy *policy, const psd_graph *graph, psd_stats *stats, const psd_kv_shared *kv, void *ws,
                                int64_t ws_bytes, void *stream);

/* ---- Head norms with rotary positions, and caches in 8 bits ---------------------------------------
 * What stands between the rows of a QKV projection and attention over a cache of half the size: psd_rotary turns queries and keys,
 * psd_kv8_store puts keys and values into the cache, psd_attention_kv8 attends to it and to the rows that are not in it yet, psd_kv8_load reads
 * it back.  These calls take no handle; they run on the current HIP device.
 *
 * psd_rotary: every head of the n_heads query heads and n_kv_heads key heads (0: no keys) of n_tokens rows,
 *     y = x / sqrt(mean x^2 + eps) * gain                                   (q_gain, k_gain: device float [d_head]; NULL: x as it is)
 *     (y_a, y_b) <- factor * (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * frequency of the pair,
 *   for the pairs a, b = j, j + rotated / 2 or, interleaved, 2j, 2j + 1 of its first `rotated` channels.  Heads of a row lie one behind the
 *   other, rows ld_* elements apart.  Everything is computed in fp32 and rounded once; an angle is position * frequency in 64 bits, with
 *   whole turns taken away before it is rounded.  frequencies: device double [rotated / 2], radians a position; positions: device int32 [n_tokens], or
 *   NULL: row i stands at first + i % rows_per_seq.  q_out / k_out may be q / k with the same row stride (in place); else no output may
 *   overlap an input or the other output (all may be columns of one buffer's rows).
 * psd_rotary_frequencies: theta^(-2j / rotated), host double [rotated / 2], plain or scaled for contexts `stretch` times as long as a model was
 *   trained for: PSD_ROTARY_LINEAR divides all by stretch; PSD_ROTARY_BASE uses theta * stretch^(rotated / (rotated - 2)), which keeps the
 *   fastest and divides the slowest by stretch; PSD_ROTARY_PARTS divides those that turn less than `slow` times over `trained` positions by stretch, keeps
 *   those that turn more than `fast` times, goes linearly between, and has a factor of 0.1 ln(stretch) + 1 (else *factor is 1; it may be NULL).  "Between" is in turns:
 *   a model whose ramp goes by the pair's index between two cut-offs needs frequencies of the caller's own. */
#define PSD_MAX_ROTARY_HEAD 256
#define PSD_ROTARY_PLAIN 0
#define PSD_ROTARY_LINEAR 1
#define PSD_ROTARY_BASE 2
#define PSD_ROTARY_PARTS 3
typedef struct {
    double theta, stretch, trained, slow, fast;   /* stretch >= 1; the last three: PSD_ROTARY_PARTS */
    int32_t kind;                                 /* PSD_ROTARY_* */
    int32_t reserved;                             /* 0 */
} psd_rotary_scaling;
typedef struct {
    int64_t n_tokens, ld_q, ld_k, ld_q_out, ld_k_out;   /* row strides in elements */
    int32_t n_heads, n_kv_heads, d_head;                /* d_head: even, up to PSD_MAX_ROTARY_HEAD */
    int32_t rotated, interleaved;                       /* channels that are turned (even); 0 / 1 */
    int32_t first, rows_per_seq;                        /* where positions is NULL */
    int32_t dtype;
    float   factor, eps;
    int32_t reserved;                                   /* 0 */
} psd_rotary_shape;
int32_t psd_rotary_frequencies(const psd_rotary_scaling *scaling, int32_t rotated, double *frequencies, double *factor);
int32_t psd_rotary(const psd_rotary_shape *shape, const void *q, const void *k, const double *frequencies, const int32_t *positions,
                   const float *q_gain, const float *k_gain, void *q_out, void *k_out, void *stream);

/* A cache in 8 bits: units (requests, or their layers) of `capacity` positions, a multiple of 32 and of `block`.  A unit has, for each KV head one
 * behind the other,
 *   codes   [capacity / 32] tiles of 32 * d_head bytes of keys, [d_head / 16][32 positions][16 channels], then as many of values,
 *           [d_head / w][2][w channels][16], w = min(32, d_head), part h of 2 with positions 8 b + 4 h + j at 4 b + j (b, j: 0 .. 3);
 *   scales  [capacity / block] pairs of floats: of the block's keys, of its values (not negative).
 * A code stands for code * scale: a whole number -127 .. 127 (PSD_KV8_INT8) or a float of 4 bits of exponent and 3 of mantissa, bias 7, up to 448
 * (PSD_KV8_E4M3).  What lies behind a unit's length is never used.  Nothing has to be zeroed.
 * psd_kv8_store: n rows of each unit (row i of unit u: k + (u * n + i) * ld_k, heads one behind the other; v likewise) go to positions first + i or, where
 *   starts is set (device int32 [units]), starts[u] + i; counts (device int32 [units], or NULL): only the first counts[u] (cut to 0 .. n).
 *   Rows that would lie outside the cache are left out.  A block's scale is the largest magnitude in its new rows over the largest code (127, 448),
 *   rounded to fp32, or what it was where positions in front of the new ones need more; codes are the nearest to x / scale, ties to even.  Where a
 *   block's scale grows, what it held in front of the new rows is rounded again to that.  What it held behind them stands for nothing any more.  A block with an
 *   infinity or NaN among its new rows reads as NaN until it is begun anew.  The lengths are the caller's (cache->lens is not written).
 *   Units may not overlap.  d_head 16, 32, 64 or 128 in either dtype; rows 16-byte aligned.
 * psd_kv8_load: positions first .. first + n - 1 of each unit to rows k, v (as in psd_kv8_store), code * scale rounded to dtype once; rows at or behind a
 *   unit's length are left as they are. */
#define PSD_KV8_INT8 0
#define PSD_KV8_E4M3 1
typedef struct {
    void *codes;                 /* device, 16-byte aligned */
    float *scales;               /* device, 8-byte aligned */
    const int32_t *lens;         /* device int32, positions of every unit (cut to 0 .. len), or NULL: each unit holds len */
    int64_t stride_codes;        /* from unit to unit: bytes, a multiple of 16 */
    int64_t stride_scales;       /* floats, even */
    int32_t capacity;            /* positions of a unit, up to 2^30 */
    int32_t len;                 /* positions that a unit holds, or the most that any does */
    int32_t block;               /* positions to a scale: 16, 32, 64 or 128 */
    int32_t format;              /* PSD_KV8_* */
    int32_t n_kv_heads, d_head;
    int32_t seqs_per_unit;       /* attention: sequences u * seqs_per_unit .. + seqs_per_unit - 1 see unit u */
    int32_t reserved;            /* 0 */
} psd_kv8_cache;
/* sizeof psd_rotary_shape, psd_rotary_scaling and psd_kv8_cache, as psd_struct_sizes gives those of the structures above. */
int32_t psd_kv8_struct_sizes(int32_t *out, int32_t n);
int32_t psd_kv8_store(const psd_kv8_cache *cache, int32_t units, const void *k, const void *v, int64_t ld_k, int64_t ld_v, int32_t dtype, int32_t n,
                      int32_t first, const int32_t *starts, const int32_t *counts, void *stream);
int32_t psd_kv8_load(const psd_kv8_cache *cache, int32_t units, int32_t first, int32_t n, void *k, void *v, int64_t ld_k, int64_t ld_v,
                     int32_t dtype, void *stream);
/* psd_attention_kv8: softmax(q k^T / sqrt(d_head)) v of every row over all positions of its sequence's unit and, where k and v are set, the L rows of its
 *   own sequence (row i of sequence s: k + (s*L + i) * ld_k, in the dtype of the call, 16-byte aligned rows), which are not in the cache: a block attends
 *   to all of itself.  Shape, out, lse and rows without a key as for psd_attention_shared (S a multiple of cache->seqs_per_unit; cache->len may be
 *   0, then codes and scales may be NULL with capacity 0).  Codes are used as they are: a key's scale multiplies its score, a value's its probability, which with
 *   bf16 is rounded after that.  Outputs are divided by the sum of the rounded ones (where a value scale is 0 or below the normal numbers, of the others); lse is of
 *   the others.  Sums and statistics are fp32.  ws: device, 256-byte aligned, psd_attention_kv8_bytes of the same shape and cache (own_rows: 1 where k is set; it
 *   does not look at device memory); calls that overlap need one each.
 * psd_debug_attention_kv8_plan: form (0: tiles of 32 rows, 1: of 128), tiles of rows of a unit and KV head, parts of the keys, keys of a part.
 * psd_debug_force_attention_kv8: the form (-1: by price; fp32 has form 0 only) and the parts (0: by price; cut to what there is) of the calls that
 *   follow, workspaces included.  Process-wide. */
int64_t psd_attention_kv8_bytes(const psd_attention_shape *shape, const psd_kv8_cache *cache, int32_t own_rows);
int32_t psd_attention_kv8(const psd_attention_shape *shape, const void *q, const psd_kv8_cache *cache, const void *k, const void *v, int64_t ld_k,
                          int64_t ld_v, void *out, float *lse, void *ws, int64_t ws_bytes, void *stream);
int32_t psd_debug_attention_kv8_plan(const psd_attention_shape *shape, const psd_kv8_cache *cache, int32_t own_rows, int32_t *plan);
int32_t psd_debug_force_attention_kv8(int32_t form, int32_t parts);

/* ---- Approximate KV cache for fully bidirectional models -----------------------------------------
 * Sec. 3.2 stage 3 notes that KV-cache sharing can cut redundant computation; with bidirectional
 * attention any cache is an approximation, and the paper fixes no scheme.  The one offered here is the
 * published prefix + suffix ("dual") cache of block-wise diffusion decoding: the model call that enters a
 * block runs over the whole sequences (exact) and freezes, per layer, the rotated keys and the values of the
 * N - L positions outside the block; every later call on that block runs on the L block rows alone and
 * attends to the frozen entries, which are stale by then.  Results differ from the exact calls above (they
 * are those of the same procedure under this approximation; the test oracle has the same mode).
 * config.attention must be PSD_ATTN_BIDIRECTIONAL, L a multiple of 16.  The cache is laid out like the exact
 * one (psd_kv_cache_bytes(cfg, capacity) per sequence, capacity >= N - L, zeroed once with psd_kv_reset).
 *   psd_forward_confidence_approx: refresh = 1: exact call over the S whole sequences, fills cache s for
 *     sequence s (seqs_per_cache must be 1); refresh = 0: block rows against the caches, sequence s using
 *     cache s / seqs_per_cache (the K drafts of a verification batch share their sequence's cache).
 *     Outputs as psd_forward_confidence_cached; ws as psd_workspace_bytes(cfg, S, refresh ? N : L, L).
 *   psd_decode_block_approx: Alg. 1 on the block; the first stage-1 call refreshes, all other calls use the
 *     caches.  cache for B sequences; ws_bytes >= max(psd_workspace_bytes(cfg, B, N, L),
 *     psd_workspace_bytes(cfg, B*K, L, L)) + psd_decode_scratch_bytes(B, N, L, K). */
int32_t psd_forward_confidence_approx(psd_handle *h, const int32_t *tokens, int32_t S, int32_t N, int32_t block_start,
                                      int32_t L, int32_t refresh, int32_t seqs_per_cache, void *cache, int32_t capacity,
                                      int32_t *top1, float *conf, float *logits, void *ws, int64_t ws_bytes,
                                      void *stream);
int32_t psd_decode_block_approx(psd_handle *h, int32_t *tokens, int32_t B, int32_t N, int32_t block_start, int32_t L,
                                const psd_policy *policy, const psd_graph *graph, psd_stats *stats, void *cache,
                                int32_t capacity, void *ws, int64_t ws_bytes, void *stream);

/* Offline calibration of the draft graph (Sec. 3.2 stage 2: the topology is fixed before inference so
 * as to maximise empirical throughput).  The calibration batch -- tokens device int32 [B, N], the first
 * n_prompt positions of every row resolved, the rest [M] -- is decoded block by block once per candidate
 * (on a copy in work_tokens, device int32 [B, N]; tokens itself is only read), timed with HIP events on
 * `stream`; scores[c] (host) receives the candidate's decode time, decoded tokens per second, TPF, tokens
 * and invocations summed over the batch, and *best the index with the highest tokens per second (lowest
 * index on ties).  cache = NULL: whole-sequence model calls; otherwise the block-causal cached path
 * (cache as for psd_decode_block_cached, for B sequences; it is reset and prefilled from the prompt before
 * every candidate, outside the timed region).  ws as for psd_decode_block with the largest K among the
 * candidates.  EOS early stopping is not applied (policy->eos_stop is ignored).  Blocks until done. */
typedef struct {
    double  seconds, tokens_per_s, tpf;
    int64_t tokens, invocations;
} psd_graph_score;
int32_t psd_calibrate_graph(psd_handle *h, const int32_t *tokens, int32_t *work_tokens, int32_t B, int32_t N,
                            int32_t n_prompt, int32_t L, const psd_policy *policy, const psd_graph *candidates,
                            int32_t n_candidates, psd_graph_score *scores, int32_t *best, void *cache,
                            int32_t capacity, void *ws, int64_t ws_bytes, void *stream);

/* Per-handle timing of the last psd_decode_block / forward calls is not kept; callers time
 * with HIP events on `stream`.  For roofline accounting the library reports the algorithmic
 * work of one forward: FLOPs of the layer contractions, of attention, and of the LM-head,
 * and the bytes the LM-head pass must move (weights once + hidden rows + outputs). */
typedef struct {
    double gemm_flops, attn_flops, head_flops, head_bytes, weight_bytes;
} psd_work;
int32_t psd_forward_work(const psd_model_config *cfg, int32_t S, int32_t N, int32_t L, psd_work *out);

/* Kernel-level hooks for parity tests and timing at full shapes without a model: the same
 * launchers the forward uses, on caller-provided device buffers (bf16 = raw 16-bit).
 *   gemm:  epilogue 0/1: out[m, n] = bf16(sum_k A[m,k] W[n,k] (+ bias[n]));
 *          2: resid[m, n] += sum (fp32);  3: out = bf16(silu(A W^T) * (A W2^T)).
 *          A [M, Kin] with row stride lda, W / W2 [Nout, Kin] with row stride ldw (elements, multiples
 *          of 8); Nout, Kin multiples of 64; ldo = row stride of out / resid.
 *   attention: qkv [S*N, (n_heads + 2 n_kv_heads) * d_head] with row stride ld_qkv (elements, multiple of 8),
 *          rotary already applied; vT is scratch of psd_kernel_attention_scratch_bytes; out
 *          [S*N, n_heads*d_head] dense.
 *   head:  y [rows, d], W [vocab, d] -> row_sum[r] = sum_v exp(z_v - max_v z), row_arg[r] =
 *          argmax_v z_v over v != mask_id, z = scale * y W^T; scratch from
 *          psd_kernel_head_scratch_bytes. */
int32_t psd_kernel_gemm_bf16(const void *A, const void *W, const void *W2, int64_t M, int32_t Nout, int32_t Kin,
                             int32_t lda, int32_t ldw, int32_t epilogue, const float *bias, void *out, float *resid,
                             int32_t ldo, void *stream);
/* The residual contraction (epilogue 2, dense A, W and resid) cut into k_splits parts along K (0 = the choice
 * the forward makes for this shape, possibly 1; otherwise 1..8 with Kin a multiple of 64*k_splits): part 0
 * adds into resid, the others go to `partial` (device, (k_splits-1)*M*Nout floats) and are then added
 * to resid in order by a second kernel, so that resid ends as resid + A W^T.  *used_splits (host, may be
 * NULL) receives the number of parts. */
int32_t psd_kernel_gemm_residual_splitk(const void *A, const void *W, int64_t M, int32_t Nout, int32_t Kin,
                                        float *resid, float *partial, int64_t partial_bytes, int32_t k_splits,
                                        int32_t *used_splits, void *stream);
int64_t psd_kernel_attention_scratch_bytes(int32_t S, int32_t N, int32_t n_kv_heads, int32_t d_head);
int32_t psd_kernel_attention_bf16(const void *qkv, int32_t ld_qkv, int32_t S, int32_t N, int32_t n_heads,
                                  int32_t n_kv_heads, int32_t d_head, void *vT, void *out, void *stream);
int64_t psd_kernel_head_scratch_bytes(int32_t rows, int32_t vocab);
/*   streaming head (at most 192 rows; the forward runs it up to 128, where a row of the matrix is 4 KB or over 8 KB): both operands in MFMA-fragment order,
 *          [ceil(R/32)][K/16][64 lanes][8 bf16]; psd_kernel_pack_rows builds that copy of a row-major
 *          [R, K] matrix into dst of psd_kernel_packed_bytes(R, K) bytes.  Same outputs and scratch as
 *          psd_kernel_head_confidence_bf16 (the tiled kernel, which the forward runs otherwise). */
int64_t psd_kernel_packed_bytes(int64_t R, int32_t K);
int32_t psd_kernel_pack_rows(const void *src, int64_t R, int32_t K, void *dst, void *stream);
int32_t psd_kernel_head_stream_bf16(const void *y_packed, const void *W_packed, int32_t rows, int32_t vocab, int32_t d,
                                    float scale, int32_t mask_id, void *scratch, float *row_sum, int32_t *row_arg,
                                    void *stream);
int32_t psd_kernel_head_confidence_bf16(const void *y, const void *W, int32_t rows, int32_t vocab, int32_t d, float scale,
                                        int32_t mask_id, void *scratch, float *row_sum, int32_t *row_arg, void *stream);
/* psd_kernel_head_stream_bf16 for callers that cannot allocate device memory or size a scratch buffer: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same inputs, outputs and kernels; the
 * per-slab partial results go to a static device array inside the library (11 796 480 bytes, held by every GPU the
 * library runs on until the process ends) instead of `scratch`.  Limits: rows <= 192, vocab <= 163 840
 * (PSD_ERR_WORKSPACE beyond them; nothing is launched).  Allocates nothing and frees nothing.  All calls on one GPU
 * share that array: calls that overlap on one GPU (different streams or threads) race; calls on one stream do not. */
int32_t psd_kernel_head_stream_static_bf16(const void *y_packed, const void *W_packed, int32_t rows, int32_t vocab,
                                           int32_t d, float scale, int32_t mask_id, float *row_sum, int32_t *row_arg,
                                           void *stream);

/* Calibration kernel: 256 workgroups of 4 wavefronts, each running `iters` rounds of 16 independent
 * v_mfma_f32_32x32x16_bf16 on operand data read from `operands` (device, bf16 values, >= 16 bytes)
 * and rotated between rounds; nothing else.  Returns in *flops the FLOPs of the launch; the
 * caller times it with events on `stream`.  The MFMA clock is power-managed, so the rate on real
 * data (not zeros) is the sustained ceiling for a contraction on this device.  sink: device, 4 MiB. */
int32_t psd_kernel_mfma_rate(const void *operands, int64_t operand_bytes, int32_t iters, void *sink, int64_t sink_bytes,
                             double *flops, void *stream);

/* Kernel timing for roofline accounting.  Between psd_probe_begin and psd_probe_end every
 * layer contraction with the given epilogue (0 store, 1 bias, 2 residual, 3 SwiGLU) that runs on the given kernel
 * is bracketed by HIP events on the stream it is launched on.  Kernels: an index below psd_kernel_gemm_tile_count, a
 * workgroup tile (psd_kernel_gemm_tile_name describes it: tile extent, depths of the two LDS rings);
 * psd_kernel_gemm_tile_count itself, the one that streams the weights past up to 128 rows; numbers behind it, two
 * tiles: the contraction runs as two launches, timed as one (up to
 * max_launches; later ones go untimed).  Kind 4 selects the LM-head confidence pass instead
 * (all its kernels, tile ignored), kind 5 every model call (forward + confidence pass) made by
 * psd_decode_block / psd_decode; both can be timed together with one contraction kernel.
 * psd_probe_end waits for those events and returns their summed duration, the number of timed
 * launches and their algorithmic work: FLOPs (2*M*N*K, twice that for SwiGLU) for a contraction,
 * bytes (vocab*d*2 + rows*d*2 + rows*8) for the LM-head pass, 0 for model calls (psd_forward_work gives it).
 * psd_probe_read (after psd_probe_end) copies the first max_n timed launches one by one: ms[i] their duration and
 * (a[i], b[i]) = (rows, output columns) of a contraction, (rows, 0) of an LM-head pass, (sequences, drafts per
 * sequence: 1 for a stage-1 call, K for a verification call) of a model call; returns how many it wrote.
 * psd_kernel_gemm_tile tells which of them the dispatcher picks for a shape at a K of 4096, psd_debug_gemm_plan at any K. */
int32_t psd_probe_begin(psd_handle *h, int32_t epilogue, int32_t tile, int32_t max_launches);
int32_t psd_probe_end(psd_handle *h, int32_t epilogue, double *total_ms, int64_t *launches, double *work);
int32_t psd_probe_read(psd_handle *h, int32_t epilogue, int32_t max_n, float *ms, int64_t *a, int64_t *b);
int32_t psd_kernel_gemm_tile(int64_t M, int32_t Nout, int32_t epilogue);
/* Number of tile configurations (valid tile ids are 0 .. count-1) and a static description of one, or of another kernel number. */
int32_t psd_kernel_gemm_tile_count(void);
const char *psd_kernel_gemm_tile_name(int32_t tile);

#ifdef __cplusplus
}
#endif
#endif /* PSD_H */
