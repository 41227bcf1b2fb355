/*
 * tabed.h -- C ABI of the TABED per-round hot path on one MI355X (gfx950).
 *
 * TABED (Test-time Adaptive Batched Ensemble Drafting) runs n drafting methods
 * as one batch through a shared draft model, mixes their next-token
 * distributions with test-time-adaptive weights, and has the target model
 * verify gamma drafted tokens by speculative sampling.  This library is the
 * part of one such round that sits behind the two models' transformer bodies:
 *
 *   tabed_update_weights   Alg. 1 (weight-selection step) with the many-draft policy of
 *                          App. B.2 (w = softmax(1/e; tau)), incl. the window.
 *   tabed_draft_step       Alg. 1 (loop body: draft forward, W-Avg, Sample) for one in-block position: LM head
 *                          of the n drafts as one batched GEMM, per-draft
 *                          softmax, weighted-average ensemble, next token.
 *   tabed_verify           Sec. 3 items 2-3: accept each drafted token with
 *                          probability min(1, p/q), resample the first rejected
 *                          one from norm(max(0, p - q)); plus the per-position
 *                          distances D(p, q^(j)) of Sec. 5.1 that feed the
 *                          next tabed_update_weights.
 *
 * Around that path:
 *
 *   tabed_draft_siblings,  Sec. 6.1 "Verification: Integrating Token Tree" (App. D): sibling candidates of a
 *   tabed_verify_tree      position and their verification by multi-round rejection sampling.
 *   tabed_draft_body_step, Sec. 5.1 "Ensemble learning via Batched Inference", Sec. 4.1 "Target and Draft
 *   tabed_draft_body_rollback   Models": one decode step of the shared LLaMA-style draft model for the n * B rows.
 *   tabed_draft_step_static     tabed_draft_step for callers that cannot allocate device memory.
 *   tabed_norm_q8, tabed_linear_q8,                The draft side in 8 bits: norm, product, key / value cache and
 *   tabed_cache_append_q8, tabed_attention_q8      the attention over it; a draft step and a body step of them:
 *   tabed_draft_step_q8, tabed_draft_body_step_q8
 *   tabed_cache_append_nodes, tabed_attention_nodes,   A tree of drafted tokens of any shape: its keys and values into a paged cache,
 *   tabed_verify_nodes, tabed_cache_keep_nodes         the attention over it, its verification, the accepted path kept.
 *
 * Notation: n = number of drafting methods (the paper's m), B independent
 * sequences, V vocabulary size, d draft hidden size, gamma block length,
 * h observation window (in verified positions).
 *
 * Conventions for every call
 *   - All data pointers are DEVICE pointers owned by the caller; `cfg` is a
 *     HOST pointer.  The library allocates, frees and synchronises nothing:
 *     kernels are enqueued on `stream` (a hipStream_t passed as void*; NULL is
 *     the default stream) and the call returns at once.
 *   - Row-major, innermost index last.  Base pointers 16-byte aligned.
 *   - Return value: TABED_OK or a negative TABED_E* code.  Argument errors are
 *     detected on the host before anything is enqueued.
 *   - `ws` is scratch memory of tabed_workspace_bytes(cfg) bytes.  It must be
 *     prepared once with tabed_workspace_init() and may then be reused by any
 *     number of calls with the same cfg on the same stream.  Calls that share
 *     a workspace must not overlap.
 *   - A temperature of 0 marks a greedy row: token decisions are arg-max
 *     (lowest index on ties) and its distributions are the untempered softmax.
 *   - Uniform random numbers come from Philox4x32-10 with key = cfg->seed and
 *     counter = (round, b, pos): word 0 at pos < gamma drives the draft sample,
 *     word 1 the accept test; word 0 at pos = gamma drives the corrected /
 *     bonus sample; u = (x >> 8) * 2^-24.  Each call also takes optional
 *     arrays of explicit uniforms that replace them (NULL = Philox).
 *   - flag bits: TABED_FLAG_* below.  A flagged decision had a margin below
 *     1e-6 relative and may legitimately differ from a higher-precision
 *     evaluation.
 */
#ifndef TABED_H
#define TABED_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TABED_MAX_N 16     /* drafting methods                      */
#define TABED_MAX_TREE_WIDTH 3 /* candidates per position of a token tree (1 = chain) */
#define TABED_MAX_GAMMA 32 /* block length                          */

#define TABED_OK 0
#define TABED_ENULL (-1)        /* a required pointer is NULL                         */
#define TABED_EINVAL (-2)       /* a cfg field is out of range                        */
#define TABED_ERANGE (-3)       /* pos >= gamma, n > TABED_MAX_N, ...                 */
#define TABED_EALIGN (-4)       /* a base pointer is not 16-byte aligned              */
#define TABED_EUNSUPPORTED (-5) /* valid request this build does not implement        */
#define TABED_EHIP (-6)         /* a kernel launch failed (see tabed_last_hip_error)  */
#define TABED_ETOOBIG (-7)      /* cfg needs more scratch than tabed_draft_step_static's built-in buffer */

#define TABED_FLAG_ACCEPT_MARGIN 1u /* accept test u*q < p closer than 1e-6 relative          */
#define TABED_FLAG_SAMPLE_MARGIN 2u /* CDF crossing / arg-max runner-up closer than 1e-6      */
#define TABED_FLAG_DEGENERATE 4u    /* empty residual, CDF never crossed, or token out of range */

typedef struct tabed_cfg {
    int32_t V;        /* vocabulary size, 1..262144                                        */
    int32_t d;        /* draft hidden size, >= 1 (multiple of 8 when w_dtype = 1)          */
    int32_t n;        /* drafting methods batched through the draft model, 1..TABED_MAX_N  */
    int32_t B;        /* independent sequences, 1..65535                                   */
    int32_t gamma;    /* draft block length, 1..TABED_MAX_GAMMA                            */
    int32_t h;        /* observation window length in verified positions, >= 1; 0 = ALL    */
                      /* positions since the start (the paper's default, App. B.1)         */
    int32_t w_dtype;  /* storage type of W and H: 0 = fp32, 1 = bf16                       */
    int32_t distance; /* D of Alg. 1: 0 = KL(p || q) (Sec. 5.1); 1 = total variation;      */
                      /* 2 = hard labels: 1 where the candidate's arg-max token differs    */
                      /*     from the token emitted at the position, else 0                */
    int32_t policy;   /* 0 = softmax(1/e; tau_w) (App. B.2); 1 = static equal weights;     */
                      /* 2 = two-draft grid (App. B.2): arg-min over w^c = [1-c/10, c/10], */
                      /*     c = 0..10, of the window sum of D(p, mixture); needs n = 2;   */
                      /* 3 = random weights, uniform on the simplex, fresh for every block */
                      /*     (the random-weights ablation of Sec. 6.2)                       */
    float tau_w;      /* temperature of the weight softmax, > 0 (paper default 1)          */
    float eps;        /* e is clamped to >= eps before 1/e, > 0                            */
    uint64_t seed;    /* Philox key                                                        */
} tabed_cfg;

#define TABED_GRID_CANDIDATES 11

/* Width DW of one distance vector (last dimension of `dev` and `ring`): n per-draft distances, or
 * TABED_GRID_CANDIDATES mixture distances when policy = 2; 0 if cfg is invalid. */
int32_t tabed_dev_width(const tabed_cfg* cfg);

/* Bytes of scratch the calls below need for this cfg; 0 if cfg is invalid. */
size_t tabed_workspace_bytes(const tabed_cfg* cfg);

/* Zeroes the arrival counters inside `ws` (a small fill kernel on `stream`).
 * Call once after allocating `ws`, before the first draft/verify call. */
int tabed_workspace_init(const tabed_cfg* cfg, void* ws, void* stream);

/* Static text for an error code. */
const char* tabed_strerror(int code);

/* hipError_t value of the most recent failed launch on this host thread (0 if none). */
int tabed_last_hip_error(void);

/*
 * Alg. 1 (loop body: draft forward, W-Avg, Sample) at in-block position `pos` (0 <= pos < gamma) for all B
 * sequences:  L = H W^T for the n*B rows, q^(j) = softmax(L_j / T),
 * q = sum_j w_j q^(j), y ~ Sample(q) (arg-max for greedy rows).
 *
 *   W            [V,d]            in   LM-head matrix shared by all drafts (w_dtype)
 *   H            [B,n,d]          in   last hidden state of every draft (w_dtype)
 *   weights      [B,n]     fp32   in   w*_t, constant over the block (Sec. 5.1)
 *   temperature  [B]       fp32   in   0 => greedy row
 *   u_draft      [B,gamma] fp32   in   optional explicit uniforms, column pos is read; NULL => Philox
 *   draft_logits [gamma,B,n,V] fp32 out slot pos is written
 *   draft_lse    [gamma,B,n] fp64 out  log-sum-exp of L_j / T, slot pos is written
 *   draft_tokens [B,gamma] int32  out  column pos is written
 *   draft_q      [B,gamma] fp32   out  q(y), column pos is written
 *   flags        [B,gamma] uint8  out  column pos is written
 */
int tabed_draft_step(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t pos,
                     const void* W, const void* H, const float* weights, const float* temperature,
                     const float* u_draft,
                     float* draft_logits, double* draft_lse, int32_t* draft_tokens, float* draft_q,
                     uint8_t* flags, void* stream);

/*
 * tabed_draft_step without a workspace argument, for callers that cannot allocate device memory at all: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels
 * and bit-identical results; the scratch memory is a buffer of TABED_STATIC_SCRATCH_BYTES built into the
 * library's code object (every GPU the library runs on holds one copy until the process ends), so the call
 * neither allocates nor frees anything, directly or through a library.
 *   - returns TABED_ETOOBIG when tabed_workspace_bytes(cfg) exceeds TABED_STATIC_SCRATCH_BYTES (e.g. the
 *     512-row stress shape); nothing is enqueued then.
 *   - every call on a GPU uses that GPU's one buffer, which keeps the previous call's contents; the call
 *     clears what must start at zero itself (a fill kernel on `stream`).  Calls that overlap on one GPU
 *     (different streams, or threads) race on it: serialise them, or use tabed_draft_step with one
 *     workspace per stream.
 *   - the buffer's device address is looked up on the first call on each device (with that device current);
 *     make that first call outside graph capture.
 */
#define TABED_STATIC_SCRATCH_BYTES (8u << 20)
int tabed_draft_step_static(const tabed_cfg* cfg, uint64_t round, int32_t pos,
                            const void* W, const void* H, const float* weights, const float* temperature,
                            const float* u_draft,
                            float* draft_logits, double* draft_lse, int32_t* draft_tokens, float* draft_q,
                            uint8_t* flags, void* stream);

/*
 * Sec. 3 items 2-3 for all B sequences, given the target's logits at the
 * gamma drafted positions and one position beyond; plus D(p_i, q_i^(j)) for
 * every drafted position i and draft j (Sec. 5.1).
 *
 *   target_logits [B,gamma+1,V] fp32 in
 *   draft_logits, draft_lse, draft_tokens, draft_q, weights, temperature: as written by / passed to
 *                 the gamma tabed_draft_step calls of this round
 *   u_acc         [B,gamma] fp32  in   optional explicit accept-test uniforms; NULL => Philox
 *   u_res         [B]       fp32  in   optional explicit uniform of the corrected/bonus sample
 *   accept_len    [B]       int32 out  k = number of accepted draft tokens, 0..gamma
 *   out_tokens    [B,gamma+1] int32 out k accepted tokens, then one corrected (k < gamma) or bonus
 *                 (k = gamma) token, then -1
 *   dev           [B,gamma,DW] fp32 out D(p_i, q_i^(j)) for every draft j (DW = n), or with policy = 2
 *                 D(p_i, (1-c/10) q_i^(1) + (c/10) q_i^(2)) for c = 0..10 (DW = 11); meaningful for i < n_valid[b]
 *   n_valid       [B]       int32 out  min(k+1, gamma): positions whose distances enter the window
 *   flags         [B,gamma+1] uint8 out flags of the accept test at i and of the sample emitted at i
 *                 (hard labels with the two-draft grid: TABED_FLAG_SAMPLE_MARGIN at a labelled position i <= k also
 *                 when the two largest entries of a candidate mixture there are closer than 1e-6 relative)
 *   ring, ring_head, ring_count, next_weights: optional, all four or all NULL.  When given, the call also
 *                 performs the tabed_update_weights() that would open round + 1 (same arguments, same
 *                 result: the window takes the n_valid verified positions and next_weights [B,n] receives the
 *                 weights of the next block), saving that call's launch.  next_weights may alias weights.
 * A drafted token outside [0,V) is rejected and flagged TABED_FLAG_DEGENERATE.
 */
int tabed_verify(const tabed_cfg* cfg, void* ws, uint64_t round,
                 const float* target_logits, const float* draft_logits, const double* draft_lse,
                 const int32_t* draft_tokens, const float* draft_q, const float* weights,
                 const float* temperature, const float* u_acc, const float* u_res,
                 int32_t* accept_len, int32_t* out_tokens, float* dev, int32_t* n_valid,
                 uint8_t* flags, float* ring, int32_t* ring_head, int32_t* ring_count, float* next_weights,
                 void* stream);

/*
 * Token tree (Sec. 6.1, paragraph "Verification: Integrating Token Tree"; results in App. D for widths 2 and 3).
 * The paper names the tree width and nothing else; the construction taken here: at every in-block position the
 * draft proposes tree_width sibling candidates for the same prefix, all from that position's ensembled
 * distribution q_i.  Candidate 0 is the token tabed_draft_step samples (the trunk: the only candidate the draft
 * model extends), candidates 1..tree_width-1 are leaves: a sampling row draws them independently from q_i, a
 * greedy row takes the next-largest entries of q_i.  tree_width = 1 is the chain.
 *
 * tabed_draft_siblings draws the siblings of position pos.  Call it after tabed_draft_step(pos) and before
 * tabed_draft_step(pos + 1): it works from the softmax partials that call left in `ws`.
 *   draft_logits [gamma,B,n,V], draft_tokens [B,gamma]: as written by tabed_draft_step (slot / column pos)
 *   u_sib        [B,gamma,tree_width-1] fp32 in   optional explicit uniforms; NULL => Philox block of counter
 *                (round, b, pos + s * 65536) for sibling s >= 1: word 0 draws it, word 1 is its accept uniform
 *   sib_tokens, sib_q, sib_flags [B,gamma,tree_width-1] out  entries (b, pos, :) are written: token, q_i(token), flags
 */
int tabed_draft_siblings(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t pos, int32_t tree_width,
                         const float* draft_logits, const int32_t* draft_tokens, const float* weights,
                         const float* temperature, const float* u_sib,
                         int32_t* sib_tokens, float* sib_q, uint8_t* sib_flags, void* stream);

/*
 * Verification of the token tree.  The trunk is verified exactly as tabed_verify does (same arguments, same
 * results for accept_len = k, dev, n_valid, the window update).  At the position k where the trunk token is
 * rejected the siblings are tried in order by multi-round rejection sampling, the lossless rule for several
 * candidates from one proposal: with f_0 = p_k, Z_0 = 1 and f_c = max(0, f_{c-1} / Z_{c-1} - q_k), Z_c = sum f_c,
 * sibling c is accepted iff u_c q_k(y_c) Z_c < f_c(y_c).  An accepted sibling is emitted and followed by one
 * bonus token from the target's distribution after it (leaf_logits); if every candidate is rejected the
 * corrected token is drawn from f_width / Z_width.  Greedy rows: a candidate is accepted iff it equals
 * arg-max p_k.  The round's one final draw uses u_res, as in the chain.
 *   leaf_logits  [B,gamma,tree_width-1,V] fp32 in  target logits after sibling s of position i
 *   sib_tokens, sib_q [B,gamma,tree_width-1]   in  as written by tabed_draft_siblings
 *   u_acc_sib    [B,gamma,tree_width-1] fp32   in  optional explicit accept uniforms of the siblings
 *   out_tokens   [B,gamma+1]  k trunk tokens, then the accepted sibling and its bonus token, or the corrected /
 *                bonus token of the chain, then -1
 *   leaf         [B] int32 out  0, or the index s of the accepted sibling
 *   n_out        [B] int32 out  tokens emitted: k + 1, or k + 2 after a leaf
 *   flags        [B,gamma+1]    column k also carries the sibling tests' margin bits, column k + 1 the draw after a leaf
 * next_weights must not alias weights here (the tree passes read this block's weights after the window update).
 * cfg->distance = 2 (hard labels) is not defined for trees: TABED_EUNSUPPORTED.
 */
int tabed_verify_tree(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t tree_width,
                      const float* target_logits, const float* leaf_logits, const float* draft_logits,
                      const double* draft_lse, const int32_t* draft_tokens, const float* draft_q,
                      const int32_t* sib_tokens, const float* sib_q, const float* weights, const float* temperature,
                      const float* u_acc, const float* u_res, const float* u_acc_sib,
                      int32_t* accept_len, int32_t* out_tokens, float* dev, int32_t* n_valid, uint8_t* flags,
                      int32_t* leaf, int32_t* n_out,
                      float* ring, int32_t* ring_head, int32_t* ring_count, float* next_weights, void* stream);

/*
 * Alg. 1 (weight-selection step) with the policy of App. B.2: push the distances of the
 * n_valid[b] verified positions of the finished block into the window, then
 * w = softmax((1 / max(e_j, eps)) / tau_w) with e_j the window sum (policy 0), or the candidate
 * [1-c/10, c/10] with the smallest window sum, lowest c on ties (policy 2).  An empty
 * window, or policy 1, gives equal weights.  Policy 3 ignores the window (but maintains it):
 * w_j = E_j / sum E with E_j = -ln U_j, U_j = (x + 0.5) 2^-24 from word j % 4 of the Philox block
 * (cfg->seed; round, b, gamma + 1 + j / 4).
 *
 *   round      the round (block) the weights are for: only policy 3 reads it
 *   dev        [B,gamma,DW] fp32 in     may be NULL together with n_valid (nothing to push)
 *   n_valid    [B]         int32 in
 *   ring       [B,h,DW]    fp32  in/out caller-owned window state (zero-initialised); with h = 0 it is
 *                                       [B,1,DW]: the running fp32 sum of all verified positions
 *   ring_head  [B]         int32 in/out next slot to overwrite
 *   ring_count [B]         int32 in/out live slots, <= h (h = 0: positions summed so far)
 *   weights    [B,n]       fp32  out
 */
int tabed_update_weights(const tabed_cfg* cfg, void* ws, uint64_t round, const float* dev, const int32_t* n_valid,
                         float* ring, int32_t* ring_head, int32_t* ring_count, float* weights,
                         void* stream);

/*
 * Draft-model body in front of the LM head (Sec. 5.1, "Ensemble learning via Batched Inference": the m drafting
 * methods share the parameters of the draft model and run as one batch; Sec. 4.1, "Target and Draft Models":
 * LLaMA-style drafts of 68M / 160M parameters).  One decode step for `rows` = n * B rows, each with its own
 * context: token embedding, then per layer RMSNorm, q/k/v projection, rotary position embedding (pairs
 * (i, i + head_dim/2)), attention over the row's own key / value cache, output projection, RMSNorm, SwiGLU MLP;
 * final RMSNorm.  The result H [rows,d] is what tabed_draft_step takes.  Weights, caches and every activation
 * that feeds a projection are bf16; the residual stream and the projections' results are fp32.  No trained
 * weights exist here: the body is exercised with random weights (parity with the oracle, and latency).
 *
 *   cfg, weights   HOST structs; the pointers inside `weights` are device pointers
 *   rows           <= 65535; row r = b * n + j as everywhere
 *   token_src, token_stride, rows_per_token: row r is fed token_src[(r / rows_per_token) * token_stride]
 *                  (in-block position i > 0: token_src = draft_tokens + i - 1, stride gamma, rows_per_token n;
 *                  a token outside [0,V) is clamped)
 *   ctx_len        [rows] int32 in/out  tokens already in the row's cache = position of the token fed now;
 *                  incremented by the call; must stay below cfg->max_ctx
 *   kcache, vcache [layers,rows,max_ctx,d] bf16 in/out  entry ctx_len[r] of every row and layer is written
 *   H              [rows,d] bf16 out
 * `ws` has tabed_body_workspace_bytes(cfg, rows) bytes, is prepared once by tabed_body_workspace_init and also serves steps of
 * fewer rows and of other configurations that fit.  A step leaves state in it for the next one: from the preparation on the memory
 * belongs to the library (prepare it again after other use), and steps that share it must not overlap (one stream, or ordered by
 * events).  A step that could not be completed (none is known that cannot) leaves NaN in H and ctx_len as it was.
 * Every pointer is 16-byte aligned (TABED_EALIGN otherwise); a ctx_len entry outside [0, max_ctx) is clamped into
 * the range, so nothing is written outside a row's cache.
 */
#define TABED_BODY_MAX_LAYERS 16
typedef struct tabed_body_cfg {
    int32_t layers;   /* 1..TABED_BODY_MAX_LAYERS                                   */
    int32_t d;        /* hidden size, multiple of 8, at most 8192                   */
    int32_t heads;    /* d / heads = head_dim, one of 8, 16, 32, 64, 128            */
    int32_t d_ff;     /* MLP width, multiple of 8                                   */
    int32_t V;        /* vocabulary of the embedding table                          */
    int32_t max_ctx;  /* cache length per row, 1..8192                              */
    float rope_theta; /* rotary base (10000)                                        */
    float rms_eps;    /* RMSNorm epsilon                                            */
} tabed_body_cfg;

typedef struct tabed_body_weights {
    const void* embed;                          /* [V,d] bf16                        */
    const float* g_final;                       /* [d]                               */
    const float* g_attn[TABED_BODY_MAX_LAYERS]; /* [d]                               */
    const void* wqkv[TABED_BODY_MAX_LAYERS];    /* [3d,d] bf16: q rows, k rows, v rows */
    const void* wo[TABED_BODY_MAX_LAYERS];      /* [d,d] bf16                        */
    const float* g_mlp[TABED_BODY_MAX_LAYERS];  /* [d]                               */
    const void* wgu[TABED_BODY_MAX_LAYERS];     /* [2*d_ff,d] bf16: gate rows, up rows */
    const void* wdown[TABED_BODY_MAX_LAYERS];   /* [d,d_ff] bf16                     */
} tabed_body_weights;

size_t tabed_body_workspace_bytes(const tabed_body_cfg* cfg, int32_t rows);   /* 0 if cfg is invalid */
int tabed_body_workspace_init(const tabed_body_cfg* cfg, int32_t rows, void* ws, void* stream);
int tabed_draft_body_step(const tabed_body_cfg* cfg, const tabed_body_weights* weights, void* ws, int32_t rows,
                          const int32_t* token_src, int32_t token_stride, int32_t rows_per_token,
                          int32_t* ctx_len, void* kcache, void* vcache, void* H, void* stream);
/*
 * After verification: the caches keep the fed tokens that were kept.  A round fed the round's first token and the
 * drafted tokens y_0 .. y_{gamma-2}; with k accepted, min(k + 1, gamma) of them stay:
 * ctx_len[r] = ctx_base[r] + min(accept_len[r / rows_per_seq] + 1, gamma).  (With k = gamma the last drafted
 * token has not been fed yet; the caller feeds it with one more tabed_draft_body_step.)
 */
int tabed_draft_body_rollback(int32_t rows, int32_t rows_per_seq, int32_t gamma, const int32_t* ctx_base,
                              const int32_t* accept_len, int32_t* ctx_len, void* stream);

/*
 * The draft model's LM head and key / value cache in 8 bits, and the operators that they are made of.  Weights, activations and cached keys and
 * values as int8 (-127 .. 127) with fp32 scales: a value is step * scale.  A scale is 1/127 of the largest magnitude it covers; it is 0, with all
 * steps 0, where no magnitude reaches 2^-100, and NaN, with all steps 0, where some value is not finite (what reads such a row or block gives NaN,
 * not a number that looks right).  Storage types of other operands are given as in tabed_cfg.w_dtype: 0 = fp32, 1 = bf16.  Strides count elements; rows
 * need no more than their type's own alignment unless said otherwise.  rows (M) = 0 and T = 0 are errors, as an empty batch is
 * everywhere in this library.
 *
 * tabed_norm_q8: residual addition, RMSNorm and int8 rows with a scale each.
 *   r = x + delta;  y = r / sqrt(mean r^2 + eps) * gain;  q = round(y / scale), ties to even
 *   x     [rows,d] x_dtype in, row stride ldx            delta [rows,d] delta_dtype in, row stride ldd; NULL: r = x
 *   sum   [rows,d] x_dtype out, row stride lds: r, rounded to that type (the norm is of r before that); may be x itself, with
 *                  lds = ldx; NULL: not stored; without delta: NULL
 *   gain  [d] fp32 in; NULL: no norm, y = r (quantises weights, or activations that are normalised already; eps is not read)
 *   q     [rows,d] int8 out, row stride ldq              scale [rows] fp32 out
 *   d 1 .. 32768, rows up to 2^20; strides at least d; a row whose squares exceed fp32 counts as not finite.
 */
int tabed_norm_q8(int32_t rows, int32_t d, int32_t x_dtype, const void* x, int64_t ldx, int32_t delta_dtype, const void* delta, int64_t ldd,
                  void* sum, int64_t lds, const float* gain, float eps, void* q, int64_t ldq, float* scale, void* stream);

/*
 * tabed_linear_q8: Y[m][n] = (sum_k X[m][k] W[n][k]) * x_scale[m] * w_scale[n].  The sum is exact (int32); then one fp32 product for
 * each scale, and the rounding to bf16 where y_dtype = 1.
 *   X [M,K] int8 in, row stride ldx (a multiple of 16)    W [N,K] int8 in     x_scale [M], w_scale [N] fp32 in
 *   Y [M,N] y_dtype out, row stride ldy >= N
 *   K a multiple of 16 (pad with zeros), 16 .. 131056, for which the sum of any int8 values fits; N 1 .. 2^24; M 1 .. 2^20; M N up to 2^36; ldx up to 2^22; X and W
 *   16-byte aligned.
 */
int tabed_linear_q8(int32_t M, int32_t N, int32_t K, const void* X, int64_t ldx, const float* x_scale, const void* W, const float* w_scale,
                    int32_t y_dtype, void* Y, int64_t ldy, void* stream);

/*
 * Key / value cache in 8 bits: a pool of blocks of TABED_CACHE_BLOCK tokens, and for every row a table of the blocks that hold its
 * tokens, position p in entry p / TABED_CACHE_BLOCK.  Rows may share blocks that are full (a common beginning); a block that
 * tokens are still appended to belongs to one row.  A table entry outside [0, blocks) is no block: its positions are not there.
 *   k, v           [blocks, kv_heads, 64 * head_dim] int8; within a block of one head
 *                  keys   [token / 4 % 4][dim / 16][token / 16][token % 4][dim % 16]
 *                  values [dim / 16][token / 16][dim % 16][token % 16]
 *                  (the order in which v_mfma_i32_16x16x64_i8 takes them)
 *   kscale, vscale [blocks, kv_heads] fp32, none below 0 (appending leaves none)
 *   table          [rows, max_blocks] int32
 * A HOST struct of device pointers; k and v 16-byte aligned.
 */
#define TABED_CACHE_BLOCK 64
typedef struct tabed_cache_q8 {
    int32_t kv_heads;   /* 1..1024                                   */
    int32_t head_dim;   /* 32, 64, 96, 128 or 256                    */
    int32_t blocks;     /* of the pool, >= 1                         */
    int32_t max_blocks; /* entries of a row of the table, 1..2^24    */
    void* k;
    void* v;
    float* kscale;
    float* vscale;
    const int32_t* table;
} tabed_cache_q8;

/*
 * tabed_cache_append_q8: quantises the keys and values of up to T new tokens a row into the cache.
 *   k, v     [rows, T, kv_heads, head_dim] kv_dtype in; row_stride, tok_stride: of a row and of a token; a token's heads lie side by side
 *   ctx_len  [rows] int32 in   tokens the row holds already; token t goes to position ctx_len[r] + t (not changed by the call; below 0: 0)
 *   n_new    [rows] int32 in   new tokens of the row, clamped to 0 .. T; NULL: T
 * A block's scale covers the tokens that it keeps (those before ctx_len) and the new ones: the larger of the old scale, if
 * any token is kept, and 1/127 of the new tokens' largest magnitude.  Where it grows the kept tokens are rounded again:
 * q = round(q * old / new).  A token taken back (a smaller ctx_len) leaves the scale it has raised until its block begins anew.
 * Tokens past the table, or whose entry is no block, are dropped.  Calling again with the same arguments changes nothing.
 */
int tabed_cache_append_q8(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t kv_dtype, const void* k, const void* v,
                          int64_t row_stride, int64_t tok_stride, const int32_t* ctx_len, const int32_t* n_new, void* stream);

/*
 * tabed_attention_q8: causal attention of the T new tokens of every row over its cache, in which they are already
 * (tabed_cache_append_q8 with the same ctx_len and n_new).  Token t sees positions 0 .. ctx_len[r] + t; query head i reads
 * key / value head i / (q_heads / kv_heads).  Scores, softmax and sums are in fp32 or exact; what is rounded before the products:
 *   T * q_heads / kv_heads up to 4: a query to whole steps of its largest magnitude times 2^-30, probabilities to 2^-30 of the largest so far
 *     (their sum is of the unrounded ones: n tokens below 2^-31 of the largest can be missing in an output, n 2^-31 max |v| at most)
 *   more: a query to whole steps of its largest magnitude / 0x7f7f78, probabilities to 22 bits (and 2^-38 of the largest so far)
 * A query with one dimension far larger than the others loses of these what fp32 would keep: the error of a score goes with max |q| sum |k|.
 * A block whose scale is not finite makes the results of the tokens that see one of its positions NaN, and of no others.
 *   q    [rows, T, q_heads, head_dim] q_dtype in     out  the same, out_dtype, out; both with strides of a row and of a token
 *   lse  [rows, T, q_heads] fp32 out, optional: natural logarithm of the sum of exp(scale * score)
 *   scale > 0, commonly 1 / sqrt(head_dim)
 * A token that sees nothing (its blocks are not there) gets zeros and an lse of -inf.  Entries of tokens from n_new[r] on are left as
 * they were.  q_heads is a multiple of kv_heads, T * q_heads at most 2^20.
 * `ws`: tabed_attention_q8_workspace_bytes bytes, prepared once by ..._init; it then serves calls of any sizes that need no more bytes.
 * Calls that share a workspace must not overlap.
 */
size_t tabed_attention_q8_workspace_bytes(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t q_heads);   /* 0: invalid */
int tabed_attention_q8_workspace_init(const tabed_cache_q8* cache, int32_t rows, int32_t T, int32_t q_heads, void* ws, void* stream);
int tabed_attention_q8(const tabed_cache_q8* cache, void* ws, int32_t rows, int32_t T, int32_t q_heads, int32_t q_dtype, const void* q,
                       int64_t q_row_stride, int64_t q_tok_stride, const int32_t* ctx_len, const int32_t* n_new, float scale,
                       int32_t out_dtype, void* out, int64_t out_row_stride, int64_t out_tok_stride, float* lse, void* stream);

/*
 * tabed_draft_step with the LM head in 8 bits: L = (H8 W8^T) * h_scale * w_scale, everything after the logits as there.
 *   W [V,d] int8, w_scale [V] fp32: tabed_norm_q8 without a gain over the rows of a bf16 or fp32 matrix
 *   H [B,n,d] int8, h_scale [B,n] fp32: as tabed_draft_body_step_q8 or tabed_norm_q8 leave them
 * cfg->w_dtype is not read beyond its check; d is a multiple of 16, at most 131056, n B V at most 2^36.  `ws` as for tabed_draft_step, which may
 * use the same one in between; siblings, verification and trees follow as after that call.
 */
int tabed_draft_step_q8(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t pos, const void* W, const float* w_scale, const void* H,
                        const float* h_scale, const float* weights, const float* temperature, const float* u_draft,
                        float* draft_logits, double* draft_lse, int32_t* draft_tokens, float* draft_q, uint8_t* flags, void* stream);

/*
 * tabed_draft_body_step over an 8-bit cache (half the bytes of keys and values, and blocks that rows may share), with the hidden
 * states in bf16, in int8 for tabed_draft_step_q8, or both.  Weights and projections stay in bf16.  It is six launches a layer for any number of
 * rows, and pays from about 32 rows on: with fewer it saves memory, not time, above all where tabed_draft_body_step is one launch (up to 16 rows).  12 layers
 * of d = 768, 256 to 768 positions, 8 / 16 bits in us: 351 / 215 at 4 rows, 402 / 264 at 16, 410 / 406 at 17, 464 / 468 at 32, 568 / 601 at 64; two layers 60 / 45,
 * 64 / 52, 68 / 66, 75 / 71, 89 / 96.
 *   cache    k, v [layers, blocks, heads, 64 * head_dim], kscale, vscale [layers, blocks, heads], one table for all layers;
 *            kv_heads = heads, head_dim = d / heads (32, 64 or 128), max_blocks * 64 >= cfg->max_ctx.  The block that a row's next token goes to
 *            belongs to that row.
 *   H        [rows,d] bf16 out, or NULL      H8, h_scale  [rows,d] int8 and [rows] fp32 out, or both NULL (not with H NULL)
 * Other arguments and the positions as for tabed_draft_body_step, tabed_draft_body_rollback included; a ctx_len entry outside [0, max_ctx) is
 * an error of the caller: nothing is written outside the table's blocks, the results are not defined.
 * `ws`: tabed_body_q8_workspace_bytes bytes, prepared once by ..._init; it then serves steps of any sizes and rows that need no more bytes
 * (not shared with other calls that run at the same time).
 */
size_t tabed_body_q8_workspace_bytes(const tabed_body_cfg* cfg, const tabed_cache_q8* cache, int32_t rows);   /* 0: invalid */
int tabed_body_q8_workspace_init(const tabed_body_cfg* cfg, const tabed_cache_q8* cache, int32_t rows, void* ws, void* stream);
int tabed_draft_body_step_q8(const tabed_body_cfg* cfg, const tabed_body_weights* weights, void* ws, int32_t rows, const int32_t* token_src,
                             int32_t token_stride, int32_t rows_per_token, int32_t* ctx_len, const tabed_cache_q8* cache, void* H, void* H8,
                             float* h_scale, void* stream);

/*
 * Trees of drafted tokens of any shape: the forward pass of a model over the nodes of a tree, and the tree's verification.  (The token tree above
 * has candidates that only its trunk continues, and takes the target's logits as given.)
 *
 * A tree has up to TABED_MAX_NODES nodes, in an order in which parents come before their children.  Node 0 is the last token emitted, which the cache does
 * not hold yet; the others are drafted tokens.
 *   parents  [rows,N] int32 in   the node that node j follows, below j; anything else makes j a root of its own (node 0: -1).  NULL: chains, node j follows j - 1
 *   n_nodes  [rows] int32 in     nodes of a row's tree, clamped to 0 .. N; NULL: N
 * In the cache node j has position ctx_len[r] + j, in its own order of things position ctx_len[r] + the number of nodes above it.  It sees the positions
 * before ctx_len[r], the nodes above it, and itself.  A ctx_len below 0 counts as 0.
 *
 * The cache: a pool of blocks of TABED_CACHE_BLOCK tokens in every layer and for every row a table of the blocks that hold its tokens, one table for
 * all layers; position p is in entry p / TABED_CACHE_BLOCK.  Rows may share full blocks; the blocks that nodes are written to belong to one row.  A table
 * entry outside [0, blocks) is no block: its positions are not there.
 *   k, v           entry of (layer, block, head, token): head_dim values that lie side by side, at layer * layer_stride + block * block_stride +
 *                  head * head_stride + token * tok_stride elements; entries must not overlap.  Every stride is at least head_dim and a multiple of 16 bytes, tok_stride at most 2^24.
 *                  (The caches of tabed_draft_body_step are one, for a max_ctx that is a multiple of 64: blocks of a row side by side, block_stride 64 d,
 *                  tok_stride d, head_stride head_dim.)
 *   kscale, vscale [layers, blocks, kv_heads, 64] fp32, type 2 only: a value is e4m3 * scale, with a scale of 1/448 of the largest magnitude of the
 *                  token in the head, so that a token can be moved without loss; the scale is 0, with all values 0, where no magnitude reaches 2^-100, and
 *                  NaN, with all values 0, where some value is not finite.  Values are the division x / scale, rounded to even.
 *   table          [rows, max_blocks] int32
 * A HOST struct of device pointers; k and v 16-byte aligned.
 */
#define TABED_MAX_NODES 256
typedef struct tabed_cache_paged {
    int32_t layers;     /* 1..1024                                   */
    int32_t kv_heads;   /* 1..1024                                   */
    int32_t head_dim;   /* 32, 64, 96, 128 or 256                    */
    int32_t blocks;     /* of the pool, >= 1                         */
    int32_t max_blocks; /* entries of a row of the table, 1..2^24    */
    int32_t type;       /* of k and v: 1 = bf16, 2 = e4m3 (8 bits, largest value 448) with scales */
    int64_t layer_stride;
    int64_t block_stride;
    int64_t head_stride;
    int64_t tok_stride;
    void* k;
    void* v;
    float* kscale;
    float* vscale;
    const int32_t* table;
} tabed_cache_paged;

/*
 * tabed_cache_append_nodes: rotates the queries and keys of a tree's nodes and writes keys and values into the cache.
 *   layer        0 .. layers - 1
 *   k, v         [rows,N,kv_heads,head_dim] dtype in; kv_row_stride, kv_tok_stride: of a row and of a node; a node's heads lie side by side
 *   q            [rows,N,q_heads,head_dim] dtype in, q_out the same in bf16 out, each with strides of its own; both NULL: no queries.  q_out may be q itself
 *                (dtype 1, the same strides)
 *   rope_theta   rotary base: pairs (i, i + head_dim/2) turn by position * rope_theta^(-2 i / head_dim), the angles in 64 bits; 0: nothing turns
 * What is turned is rounded once, to bf16 or to e4m3; dtype 0 = fp32, 1 = bf16.  Nodes from n_nodes[r] on are not written, in q_out neither; keys and values whose
 * position is past the table, or in no block, are dropped.  Calling again with the same arguments changes nothing (unless q_out is q).
 */
int tabed_cache_append_nodes(const tabed_cache_paged* cache, int32_t layer, int32_t rows, int32_t N, int32_t dtype, const void* k, const void* v,
                             int64_t kv_row_stride, int64_t kv_tok_stride, int32_t q_heads, const void* q, int64_t q_row_stride, int64_t q_tok_stride,
                             void* q_out, int64_t out_row_stride, int64_t out_tok_stride, const int32_t* ctx_len, const int32_t* parents,
                             const int32_t* n_nodes, float rope_theta, void* stream);

/*
 * tabed_attention_nodes: attention of a tree's nodes over the cache, in which they are already (tabed_cache_append_nodes with the same ctx_len, parents
 * and n_nodes).  Query head i reads key / value head i / (q_heads / kv_heads).
 *   q, out  [rows,N,q_heads,head_dim] bf16, strides of a row and of a node each; out may be q itself (the same strides) and overlaps it in no other way
 *   lse     [rows,N,q_heads] fp32 out, optional: natural logarithm of the sum of exp(scale * score)
 *   scale   > 0, commonly 1 / sqrt(head_dim)
 * Products of bf16 (and e4m3) values are exact, their sums, the softmax and its sum are in fp32; probabilities are rounded before the product with the
 * values, to bf16 (2^-8 of themselves), or with e4m3 values, and then times the values' scales: to fp16 (2^-11) relative to a query's largest such product, or to bf16 where they are
 * too far apart for that (below 2^-22 to 2^-29 of the largest; the context's others, too, from there on).  Products below 2^-130 of the largest, in
 * which a scale above 2^38 counts as that, and probabilities below 2^-95 of the largest may be lost.  Sums are of probabilities up to 2^8 times values: magnitudes of values stay below
 * 2^100.  What a node does not see has no influence, whatever it holds.  A node that sees nothing (its blocks are not there) gets zeros and an lse of -inf.  Entries of nodes from n_nodes[r] on are left as they were.
 * q_heads is a multiple of kv_heads, at most 16384.
 * `ws`: tabed_attention_nodes_workspace_bytes bytes, prepared once by ..._init; it then serves calls of any sizes and caches that need no more bytes, calls with
 * fewer rows or nodes among them.
 * Calls that share a workspace must not overlap.
 */
size_t tabed_attention_nodes_workspace_bytes(const tabed_cache_paged* cache, int32_t rows, int32_t N, int32_t q_heads);   /* 0: invalid */
int tabed_attention_nodes_workspace_init(const tabed_cache_paged* cache, int32_t rows, int32_t N, int32_t q_heads, void* ws, void* stream);
int tabed_attention_nodes(const tabed_cache_paged* cache, int32_t layer, void* ws, int32_t rows, int32_t N, int32_t q_heads, const void* q,
                          int64_t q_row_stride, int64_t q_tok_stride, const int32_t* ctx_len, const int32_t* parents, const int32_t* n_nodes, float scale,
                          void* out, int64_t out_row_stride, int64_t out_tok_stride, float* lse, void* stream);

/*
 * tabed_verify_nodes: verification of a tree by multi-round rejection sampling, from its root down.  At a node, with p the target's distribution
 * there and q = sum_j w_j q^(j) the mixture that its children were drawn from (independently, in index order):  f_0 = p, Z_0 = 1; child c is accepted iff
 * u_c q(y_c) Z_c < f_c(y_c), and the walk goes on there; else f_{c+1} = max(0, f_c / Z_c - q), Z_{c+1} = sum f_{c+1}, and the next child is tried.  Where no child
 * is accepted, or there is none, one more token is drawn from f / Z: the smallest v with sum_{v' <= v} f(v') > u Z.  An f without mass is replaced by p for that
 * draw and flagged.  Greedy rows: a child is accepted iff it is arg-max p; else that arg-max is the token.  The emitted sequence is distributed as the
 * target's.  A chain of N = gamma + 1 nodes is verified as tabed_verify does it.  Decisions are in fp64.
 *   cfg           V, n, B, gamma, distance, policy and seed are read
 *   target_logits [B,N,V] fp32 in   target's logits after every node
 *   draft_logits  [N,B,n,V] fp32, draft_lse [N,B,n] fp64 in   of the drafts after every node, slot j as tabed_draft_step writes slot pos; only those of
 *                 nodes that have children are read
 *   tokens        [B,N] int32 in    the nodes' tokens (node 0's is not read); a token outside [0,V) is rejected and flagged TABED_FLAG_DEGENERATE
 *   node_q        [B,N] fp32 in     q(token) in the mixture of the node's parent (node 0's is not read), as draft_q of tabed_draft_step, sib_q
 *   parents, n_nodes   as above, rows = B; a root other than node 0 is not reached.  A row without nodes emits nothing
 *   weights [B,n], temperature [B]  as passed to the draft steps
 *   u_acc         [B,N] fp32 in     optional uniforms of the nodes' tests (node 0's is not read); NULL: word 1 of the Philox block of counter (round, b, j - 1)
 *   u_res         [B] fp32 in       optional uniform of the last draw; NULL: word 0 of the block of counter (round, b, N - 1)
 *   path          [B,N] int32 out   node 0 and the nodes accepted, in order, then -1: what tabed_cache_keep_nodes takes
 *   n_path        [B] int32 out     nodes of the path = tokens emitted
 *   out_tokens    [B,N] int32 out   tokens of the nodes accepted, the one token drawn, then -1
 *   flags         [B,N] uint8 out   of the test of node j; entry 0: of the last draw; 0 for nodes that were not tested.  Greedy decisions compare
 *                 fp32 inputs and are never near ties
 *   dev           [B,gamma,n] fp32 out   D(p, q^(j)) at the path's nodes that have children, the first gamma of them; other entries are left as they were
 *   n_valid       [B] int32 out     how many: what tabed_update_weights takes.  dev and n_valid may both be NULL.  cfg->distance 0 or 1 and policies other
 *                 than the grid (2) then; else TABED_EUNSUPPORTED
 * `ws`: tabed_verify_nodes_workspace_bytes bytes, prepared once by ..._init; it then serves calls of any sizes that need no more bytes, all that are smaller in
 * everything among them.  It belongs to the library from the preparation on; calls that share it must not overlap.
 * A sequence's workgroups wait for each other: V / 1024 of them, rounded up, with few sequences, else V / 2048, at most 128.  Launches that run at the same time on a device, those of
 * other processes included, may hold (sequence's workgroups - 1) each of the 768 that run at a time (three a compute unit) waiting, and must leave some: six launches for V = 262144, ten for
 * V = 152064, 24 for V = 32000 and few sequences.  The four hardware queues of one process are within that.  Kernels of others that wait for workgroups of their own in this way take from the 768.
 * A row whose workgroups waited for each other in vain, for some seconds, has no path: n_path and n_valid 0, path and out_tokens -1, flags[b][0] TABED_FLAG_DEGENERATE.
 * So have, at once, all rows of a call with a workspace that was prepared for fewer bytes than it needs, or never.
 */
size_t tabed_verify_nodes_workspace_bytes(const tabed_cfg* cfg, int32_t N);   /* 0: invalid */
int tabed_verify_nodes_workspace_init(const tabed_cfg* cfg, int32_t N, void* ws, void* stream);
int tabed_verify_nodes(const tabed_cfg* cfg, void* ws, uint64_t round, int32_t N, const float* target_logits, const float* draft_logits,
                       const double* draft_lse, const int32_t* tokens, const float* node_q, const int32_t* parents, const int32_t* n_nodes,
                       const float* weights, const float* temperature, const float* u_acc, const float* u_res, int32_t* path, int32_t* n_path,
                       int32_t* out_tokens, uint8_t* flags, float* dev, int32_t* n_valid, void* stream);

/*
 * tabed_cache_keep_nodes: after verification the cache keeps the path: in all layers the entry of position ctx_base[r] + path[r][i] moves to
 * ctx_base[r] + i, and ctx_len[r] = ctx_base[r] + the number of nodes kept.
 *   path    [rows,N] int32 in   ascending nodes (path[r][0] = 0 as a rule); the path ends where an entry is not above the one before it, or not below N
 *   n_path  [rows] int32 in     entries of the path, clamped to 0 .. N
 *   ctx_len [rows] int32 out    overlaps none of the others
 * Entries whose source or destination is past the table or in no block are not moved (the positions count all the same).
 */
int tabed_cache_keep_nodes(const tabed_cache_paged* cache, int32_t rows, int32_t N, const int32_t* ctx_base, const int32_t* path, const int32_t* n_path,
                           int32_t* ctx_len, void* stream);

/*
 * The uniforms tabed_draft_step and tabed_verify would draw: out[b,pos,word] for b < B,
 * pos <= gamma, word in {0,1}.  out is [B,gamma+1,2] fp32.
 */
int tabed_philox_uniforms(const tabed_cfg* cfg, uint64_t round, float* out, void* stream);

/*
 * Per-kernel timing.  While enabled, every kernel is launched with a start and a stop HIP event attached to
 * its dispatch (hipExtLaunchKernelGGL), so the pair brackets the kernel's own execution on the launch
 * stream; tabed_prof_read() waits for them and returns accumulated milliseconds and launch count of kernel
 * `id` (TABED_K_*), and keeps the totals until tabed_prof_reset().  Off by default; these calls create and
 * destroy events and synchronise, unlike the rest of the library.
 */
#define TABED_K_LMHEAD 0  /* LM-head GEMM + softmax partials    */
#define TABED_K_SAMPLE 1  /* ensemble + draft token             */
#define TABED_K_STATS 2   /* target statistics + distances + accept chain */
#define TABED_K_RESID 3   /* corrected / bonus token            */
#define TABED_K_WEIGHTS 4 /* window + weights                   */
#define TABED_K_DIST 5    /* the launch that holds total variation (RESID's) or hard labels (STATS'), counted there too */
#define TABED_K_TREE 6    /* token tree: the first pass of the walk (the second, of width 3, is not timed); tabed_verify_nodes */
#define TABED_K_BODY 7    /* draft-model body: every kernel of tabed_draft_body_step and ..._q8; the 8-bit operators and those of a tree's nodes called by themselves */
#define TABED_K_NULL 8    /* empty kernel, see tabed_prof_null  */
#define TABED_K_COUNT 9
int tabed_prof_enable(int on);
int tabed_prof_read(int id, double* total_ms, int64_t* launches);
int tabed_prof_reset(void);
const char* tabed_kernel_name(int id);
/* Launches an empty kernel on `stream`, timed like the others when timing is enabled: what
 * tabed_prof_read(TABED_K_NULL, ...) then reports is the floor of the method. */
int tabed_prof_null(void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TABED_H */
