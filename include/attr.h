/*
 * attr.h -- C ABI of the MI355X (gfx950) gradient-attribution hot path.
 *
 * The library implements the data-parallel core of gradient-based data
 * attribution as described in "Bergson: An Open Source Library for Data
 * Attribution":
 *   (1) per-example double-sided random projection of linear-layer
 *       gradients (Figure 1 caption; Appendix B, paragraph "Gradients");
 *   (2) unit normalisation and second-moment preconditioning of the
 *       compressed rows (section "Attribution Pipelines": processing may
 *       include unit normalisation and preconditioning; the flat
 *       autocorrelation / empirical Fisher of the method-family table);
 *   (3) exact top-k lookup of a query against the gradient store (section
 *       "Attribution Pipelines": every store supports exact top-k).
 * Beside that core stand the training steps it attributes:
 *   (4) token log-probabilities, the clipped policy loss with a KL term and
 *       the paired log-ratio preference loss, with their gradients with
 *       respect to the logits (the gradients whose per-example products (1)
 *       projects);
 *   (5) the AdamW step over a model's tensors, whose second moments are the
 *       optimizer states that (1) divides gradients by, and the Muon step over
 *       the modules' matrices;
 *   (6) embedding and layer norm of token rows, what the rows that (1) reads
 *       come from, with their gradients (the norm's for each example, too).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Plain C99.  Pointers are DEVICE pointers (HIP device memory of the
 *   current device) unless marked (host).  Sizes and strides are in
 *   ELEMENTS, row-major, int64.
 * - `stream` is a hipStream_t passed as void*; NULL means the null stream.
 *   Every call only enqueues work on `stream` and returns; results are
 *   valid once the stream has completed.  No call synchronises.
 * - The caller owns every buffer, including the workspace `ws` whose
 *   minimum size the matching *_workspace_size() function returns (0 means
 *   no workspace is needed; `ws` may then be NULL).  The library keeps no
 *   per-call state between calls and never allocates device memory; the one
 *   exception is the static per-GPU scratch array of attr_project_noalloc.
 * - Errors: arguments are validated on the host before anything is
 *   enqueued.  On any error the call enqueues nothing, leaves every output
 *   untouched and returns a non-zero attr_status; attr_last_error() then
 *   describes it.  ATTR_ERR_DEVICE reports a failed kernel launch (which may
 *   also surface an earlier asynchronous error).  No C++ exception crosses
 *   this boundary.  Values inside device arrays (lengths, offsets) cannot be
 *   checked on the host; their documented clamping applies instead.
 * - Calls that share a workspace or an output must be ordered by the
 *   caller (same stream, or events); concurrent calls on different
 *   workspaces are independent.  A call may be several launches: one stream
 *   orders the calls of one host thread, while those that several threads make
 *   on it at the same time may interleave and must not share a workspace.
 */
#ifndef ATTR_H_
#define ATTR_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ATTR_ABI_VERSION 3

typedef enum {
  ATTR_OK = 0,
  ATTR_ERR_INVALID_ARG = 1,  /* null pointer with non-zero size, negative size, bad stride, overlap */
  ATTR_ERR_UNSUPPORTED = 2,  /* dtype / k / mode combination not implemented */
  ATTR_ERR_ALIGNMENT = 3,    /* pointer not 16-byte aligned, width or stride not a multiple of 8 elements */
  ATTR_ERR_WORKSPACE = 4,    /* ws_bytes below the queried size, or ws NULL when needed */
  ATTR_ERR_DEVICE = 5        /* HIP launch / runtime error */
} attr_status;

/* ATTR_E4M3 (8 bits: sign, 4 exponent and 3 mantissa bits, largest value 448)
 * is a type of attr_adamw_step's states only. */
typedef enum { ATTR_F32 = 0, ATTR_BF16 = 1, ATTR_F16 = 2, ATTR_E4M3 = 3 } attr_dtype;

typedef enum {
  ATTR_PRECOND_NONE = 0,  /* identity */
  ATTR_PRECOND_DIAG = 1,  /* per-coordinate scale m (diagonal of H^{-1/2}) */
  ATTR_PRECOND_FULL = 2   /* full matrix M (H^{-1/2}), y = M x */
} attr_precond;

/* ------------------------------------------------------------------------ */
/* (1) attr_project: per-example compressed gradients of linear modules.    */
/* ------------------------------------------------------------------------ */

/* One linear module y = W x with W of shape [d_out, d_in].  Read only during
 * the call (host struct; the pointers inside are device pointers). */
typedef struct {
  const void* a;     /* input activations, rows of d_in elements, row stride lda */
  const void* g;     /* output gradients dL/dy, rows of d_out elements, row stride ldg */
  const void* R;     /* [d_out, k] row-major, same dtype as a/g (output-side projection) */
  const void* S;     /* [d_in,  k] row-major, same dtype as a/g (input-side projection) */
  int64_t lda, ldg;  /* row strides in elements, >= d_in / d_out, multiples of 8 */
  int64_t d_in, d_out;  /* multiples of 64 (bf16) or 32 (fp32); at most 65536 */
  int64_t out_col;   /* first column of this module's k*k block in `out` */
  /* Optional optimizer-state normalisation (Figure 1 caption: Adafactor
   * second moments): the factored second moment v_ij = v_out[i] v_in[j] /
   * sum(v_out) of the module's weight; each per-example gradient is divided
   * elementwise by sqrt(v) before projection (entries where v is 0 or a
   * factor is not positive become 0; no epsilon).  Device fp32 [d_out] and
   * [d_in], both NULL for no normalisation.  Applied by scaling the rows of
   * R and S while they are packed, so the projection itself costs the same. */
  const float* v_out;
  const float* v_in;
} attr_module;

/* Double-sided projection (Figure 1 caption; Appendix B "Gradients"): for
 * every example i and module m, with len_i valid tokens,
 *     P_{i,m} = sum_{t < len_i} (R^T g_t)(S^T a_t)^T          (k x k)
 * which equals R^T G_i S for the per-example weight gradient
 * G_i = sum_t g_t a_t^T, without ever forming G_i.  The result is written
 * row-major into out[i * ldo + out_col + r * k + c] (r: column of R,
 * c: column of S) as fp32; other columns of `out` are not touched.
 *
 * Token t of example i is row (row_offset ? row_offset[i] : i * T) + t of
 * both a and g.  Tokens t >= len_i are never read, so padding may hold any
 * bit pattern including NaN.  Modules that pass the same a pointer with the
 * same lda and d_in (the q/k/v or gate/up projections of one layer) have
 * their shared rows read once for up to three of them (two at k = 64); the
 * results are the same bits as with separate copies of a.  The order of the
 * fp32 sums, and so the last bits of a row, depend on the call (the modules'
 * widths, n_examples, T and whether lengths are given), not on the workspace.
 *
 *   mods       (host) [n_mods] module descriptors; 1 <= n_mods <= 4096
 *   in_dtype   ATTR_BF16 (bf16 MFMA, fp32 accumulate) or ATTR_F32 (fp32 MFMA)
 *   k          16, 32 or 64
 *   n_examples examples in this call (0 is a no-op)
 *   T          tokens per example slot, >= 1
 *   row_offset device int64 [n_examples] or NULL (then i * T)
 *   length     device int32 [n_examples] or NULL (then T); values are
 *              clamped to [0, T]; len 0 gives a zero block
 *   out, ldo   device fp32 [n_examples, ldo]; out_col + k*k <= ldo per module
 *   ws         device workspace of at least
 *              attr_project_workspace_size(mods, n_mods, in_dtype, n_examples, T, k)
 *              bytes, 256-byte aligned; contents on entry are ignored.
 * The module blocks of `out` must not overlap each other.
 */
size_t attr_project_workspace_size(const attr_module* mods, int32_t n_mods,
                                   attr_dtype in_dtype, int64_t n_examples, int64_t T,
                                   int32_t k);
attr_status attr_project(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                         int32_t k, int64_t n_examples, int64_t T,
                         const int64_t* row_offset, const int32_t* length,
                         float* out, int64_t ldo, void* ws, size_t ws_bytes,
                         void* stream);

/* Per-token compressed gradients (Figure 1 caption: attribution scores are
 * per-token or per-sequence): the same projection without the token sum.
 * For every valid token t of example i and module m the k x k block
 *     P_{i,t,m} = (R^T g_t)(S^T a_t)^T
 * is written row-major into out[row * ldo + out_col + r * k + c], where row
 * = (row_offset ? row_offset[i] : i * T) + t is the token's own row in a
 * and g.  Rows of tokens t >= len_i and columns outside the module blocks
 * are not touched; rows >= n_rows are not written (size `out` to cover
 * every valid token's row).  Summing a token's blocks over t gives
 * attr_project's row; unit normalisation and scoring of the token rows use
 * attr_precond_apply and attr_score_topk.  Arguments as attr_project, plus
 *   out, ldo, n_rows  device fp32 [n_rows, ldo]
 *   ws        attr_project_workspace_size(...) bytes (the same query)
 */
attr_status attr_project_tokens(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                                int32_t k, int64_t n_examples, int64_t T,
                                const int64_t* row_offset, const int32_t* length, float* out,
                                int64_t ldo, int64_t n_rows, void* ws, size_t ws_bytes,
                                void* stream);

/* attr_project without a workspace argument, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving loops
 * and harnesses that forbid allocation.  It computes exactly what
 * attr_project computes (same kernels, same bits: the chunks of a call whose
 * partials pass the array come in several rounds) and makes no allocating
 * call: its scratch is a static device array of ATTR_PROJECT_NOALLOC_SCRATCH
 * bytes, one per GPU, created when the library's code first runs on that
 * GPU and held until the process ends.  Every call on a GPU shares that
 * GPU's array, so calls that overlap on one GPU (different streams or host
 * threads without ordering) race and give undefined results; order them.
 * A call whose least workspace (the bytes below which attr_project returns
 * ATTR_ERR_WORKSPACE) exceeds ATTR_PROJECT_NOALLOC_SCRATCH returns ATTR_ERR_WORKSPACE and
 * enqueues nothing.  Arguments and other errors as attr_project.
 */
#define ATTR_PROJECT_NOALLOC_SCRATCH (64ull << 20)
attr_status attr_project_noalloc(const attr_module* mods, int32_t n_mods, attr_dtype in_dtype,
                                 int32_t k, int64_t n_examples, int64_t T,
                                 const int64_t* row_offset, const int32_t* length, float* out,
                                 int64_t ldo, void* stream);

/* ------------------------------------------------------------------------ */
/* (2a) attr_precond_accumulate: second-moment statistics of store rows.    */
/* ------------------------------------------------------------------------ */

/* Accumulates the (unscaled) second moment of the rows of X, the
 * autocorrelation / empirical Fisher preconditioner of the method-family
 * table, restricted to its diagonal (DIAG) or in full (FULL):
 *   DIAG: H[j]       += sum_i X[i,j]^2                    (H: fp32 [D])
 *   FULL: H[p*D + q] += sum_i X[i,p] * X[i,q]  for p <= q (H: fp32 [D, D];
 *         the upper triangle including the diagonal is updated, the strict
 *         lower triangle is never read or written)
 * Accumulation is additive across calls, so a store can be processed in
 * chunks; divide by the total row count afterwards.  Within a call, partial
 * sums are formed in fp32 (DIAG: 8-row groups; FULL: matrix-core products
 * over at most 32768 rows), combined in fp64 in a fixed order and rounded
 * once into H, so results are deterministic.
 *
 *   X, ldx   device [n_rows, D] rows: DIAG takes ATTR_F16, ATTR_BF16 or
 *            ATTR_F32, FULL takes ATTR_F16 or ATTR_BF16; ldx >= D (FULL:
 *            ldx <= 65536, so that 16384 rows span at most 2 GiB)
 *   D        multiple of 8 (DIAG) or of 64 (FULL); FULL needs D <= 32768
 *   mode     ATTR_PRECOND_DIAG or ATTR_PRECOND_FULL
 *   ws       attr_precond_accumulate_workspace_size(n_rows, D, x_dtype, mode)
 */
size_t attr_precond_accumulate_workspace_size(int64_t n_rows, int64_t D, attr_dtype x_dtype,
                                              attr_precond mode);
attr_status attr_precond_accumulate(const void* X, attr_dtype x_dtype, int64_t n_rows,
                                    int64_t D, int64_t ldx, attr_precond mode, float* H,
                                    void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* (2b) attr_precond_apply: precondition, unit-normalise, cast.             */
/* ------------------------------------------------------------------------ */

/* For every row x of X (processing step of section "Attribution Pipelines";
 * grad-cosine when unit_normalize is set):
 *   y = x (NONE), y = M .* x (DIAG, M: fp32 [D]) or y = M x (FULL, M: fp32
 *   [D, D] row-major, symmetric in use: y_p = sum_q M[p*D+q] x_q);
 *   if unit_normalize, y /= ||y||_2 over the whole row (a zero row stays 0);
 *   Y = y cast to y_dtype (round to nearest even).
 * FULL evaluates M as a scaled fp16 pair, A = 2^s M (max|A| <= 2^15),
 * A_hi = fp16(A), A_lo = fp16(A - A_hi), y = 2^-s X (A_hi + A_lo)^T on fp16
 * MFMA with fp32 accumulation (about 22 significant bits of M).  Few rows (a
 * session's queries: up to 2^23 / D, and at most D) take a path that reads M
 * once and scales each of its rows on its own; its sums have another order, so
 * the last bits of a row depend on n_rows.
 * With unit_normalize a row that holds a NaN after the first step keeps it and
 * is zero elsewhere; so does one that holds an infinity (as NaN).  Squares are
 * summed in fp32, and a row whose sum passes fp32's range is written as zeros;
 * FULL on few rows sums them in fp64.
 *
 *   X, ldx   device [n_rows, D], x_dtype ATTR_F32 or ATTR_F16
 *            (FULL: ATTR_F16 only)
 *   Y, ldy   device [n_rows, D], y_dtype ATTR_F16 or ATTR_F32
 *   D        multiple of 8 (NONE/DIAG), of 64 (FULL)
 *   In-place (Y == X) is allowed for NONE/DIAG when dtype and stride match;
 *   any other overlap of X and Y is ATTR_ERR_INVALID_ARG.
 *   ws       attr_precond_apply_workspace_size(n_rows, D, mode)
 */
size_t attr_precond_apply_workspace_size(int64_t n_rows, int64_t D, attr_precond mode);
attr_status attr_precond_apply(const void* X, attr_dtype x_dtype, int64_t n_rows, int64_t D,
                               int64_t ldx, attr_precond mode, const float* M,
                               int32_t unit_normalize, void* Y, attr_dtype y_dtype,
                               int64_t ldy, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* (3) attr_score_topk: query x store scores with exact streaming top-k.    */
/* ------------------------------------------------------------------------ */

/* For every query q: s_qj = <Q_q, G_j> (fp32 accumulation; the cosine when
 * both sides are unit rows) over the n_g store rows, and the k best
 * (index_base + j) ordered by (score desc, index asc); NaN and -inf scores
 * are never selected; missing slots are (-inf, -1).  Exact top-k lookup,
 * section "Attribution Pipelines".  With few queries the scan streams the
 * store once and the score matrix never reaches memory (on stores of
 * 262144 rows or more a first pass over 16384 rows finds, per query, a
 * lower bound on its k-th best score, and rows below it are skipped by the
 * selection: a few KB of workspace); with many fp16
 * queries (n_q >= 128) it is computed chunk by chunk into the workspace
 * (~256 MB per chunk, plus one maximum per 64 rows) and selected exactly
 * from there; after the first chunk only 64-row segments that can still
 * beat a query's running k-th best score are written and read.
 *
 *   Q, ldq       device [n_q, D];  G, ldg: device [n_g, D]; both `dtype`
 *                (ATTR_F16 or ATTR_F32); D a multiple of 64 (fp16) or 32
 *                (fp32); n_q, n_g below 2^31; 256 rows of either operand
 *                must span less than 2 GiB (ld * 256 * element size)
 *   k            1..128
 *   index_base   added to the local row index j (store offset of G), >= 0
 *   merge        0: overwrite top_*;  1: top_* hold a previous sorted
 *                result which is merged with this chunk (streaming over
 *                stores larger than one call)
 *   top_score    device fp32 [n_q, k];  top_index: device int64 [n_q, k]
 *   ws           attr_score_topk_workspace_size(n_q, n_g, D, k)
 * n_q == 0 is a no-op; n_g == 0 leaves top_* unchanged when merge == 1 and
 * fills them with (-inf, -1) when merge == 0.
 */
size_t attr_score_topk_workspace_size(int64_t n_q, int64_t n_g, int64_t D, int32_t k);
attr_status attr_score_topk(const void* Q, int64_t n_q, int64_t ldq, const void* G,
                            int64_t n_g, int64_t ldg, attr_dtype dtype, int64_t D,
                            int32_t k, int64_t index_base, int32_t merge,
                            float* top_score, int64_t* top_index,
                            void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* (4) Losses over token log-probabilities, and their gradients.            */
/* ------------------------------------------------------------------------ */

/* A batch's rows of logits and the token each row predicts.  Token t of
 * example i is row (row_offset ? row_offset[i] : i * T) + t, as in
 * attr_project.  A token COUNTS if t < length[i], its row lies in
 * [0, n_rows), its target in [0, V) and its weight is not 0; the logits of
 * tokens that do not count are never read (padding may hold any bits).
 * With a row's largest logit z_max and s = logit_scale,
 *     logp = s (z_target - z_max) - log sum_j exp(s (z_j - z_max)),
 * exponentials and their sum in fp32 (the order of the sum, and so the last
 * bits, follow the call's sizes and the rows' alignment).  Logits of -inf are
 * vocabulary entries of probability 0; a row that holds a NaN or +inf, or -inf
 * only, has logp NaN.
 * Outputs of rows that do not count: without row_offset every row i * T + t,
 * t < T, is written (logp 0, dlogits zeros); with row_offset the rows of
 * tokens t < length[i] (clamped to [0, T]), and no others, are written.  The
 * ranges of two examples must not overlap, nor may a call's outputs overlap each
 * other or its inputs (but for dlogits over the logits, see below).
 * Read only during the call (host struct with device pointers). */
typedef struct {
  const void* logits;    /* [n_rows, V], row stride ldl >= V; any V, stride and element alignment */
  attr_dtype dtype;      /* ATTR_F32, ATTR_BF16 or ATTR_F16 */
  int64_t n_rows, V, ldl;  /* 1 <= V <= 2^28 */
  float logit_scale;     /* s: one over the sampling temperature; > 0, at most 2e38 */
  const int64_t* target;   /* device [n_rows] */
  const float* weight;     /* device [n_rows] or NULL (1 for every token) */
  int64_t n_examples, T;   /* n_examples * T < 2^31; without row_offset n_rows >= n_examples * T */
  const int64_t* row_offset;  /* device [n_examples] or NULL (then i * T) */
  const int32_t* length;      /* device [n_examples] or NULL (then T); clamped to [0, T] */
} attr_token_rows;

/* logp of every token (see above) into logp, device fp32 [n_rows]: what a
 * rollout records of the tokens it samples (T = 1: one decoding step), and
 * what a reference model gives for whole sequences.
 *   ws  attr_token_logp_workspace_size(rows) bytes, 256-byte aligned */
size_t attr_token_logp_workspace_size(const attr_token_rows* rows);
attr_status attr_token_logp(const attr_token_rows* rows, float* logp, void* ws, size_t ws_bytes,
                            void* stream);

/* Clipped policy loss with a KL term (the GRPO losses whose gradients section
 * "Attribution Pipelines" collects).  For a token that counts, with its
 * weight w, its advantage A and ratio = exp(logp - logp_old):
 *     l = max(-A ratio, -A clip(ratio, 1 - clip_low, 1 + clip_high))
 *         + beta (exp(logp_ref - logp) - (logp_ref - logp) - 1)
 *     loss[i] = sum_t w l          (0 for an example without such tokens)
 *     c = dloss/dlogp = w ((-A ratio if that is the maximum, else 0)
 *                          - beta (exp(logp_ref - logp) - 1))
 *     dlogits[row, j] = s c ([j = target] - exp(logp_j))
 * Beside a finite logp_ref a target of probability 0 (logit -inf) makes the KL
 * term, and so a loss with beta > 0, +inf; its row of dlogits is then not finite.
 * The weights carry the mask and the normalisation (1 / tokens for a mean over
 * each example, one constant for a sum, a loss scale).  Each row of logits is
 * read once and each row of dlogits written once where a row fits a
 * workgroup's registers (256 KB; longer rows, few long rows, which are spread
 * over many CUs, and rows whose largest logit is some 41 / s above the first ones
 * are read again); loss sums are formed in fp64 in a
 * fixed order.
 *   advantage  device fp32 [n_examples], or [n_rows] with per_token != 0
 *   logp_old   device fp32 [n_rows], or NULL: the logits' own (ratio 1)
 *   logp_ref   device fp32 [n_rows]; may be NULL if beta is 0
 *   clip_low, clip_high  >= 0 (clip_high may be infinite); beta >= 0
 *   loss       device fp32 [n_examples]
 *   logp       device fp32 [n_rows] or NULL
 *   dlogits    device [n_rows, V] of the logits' type, row stride ldd >= V, or
 *              NULL (the loss alone); may be the logits themselves with
 *              ldd = ldl, any other overlap is ATTR_ERR_INVALID_ARG
 *   ws         attr_policy_loss_workspace_size(rows) bytes, 256-byte aligned */
size_t attr_policy_loss_workspace_size(const attr_token_rows* rows);
attr_status attr_policy_loss(const attr_token_rows* rows, const float* advantage, int32_t per_token,
                             const float* logp_old, const float* logp_ref, float clip_low,
                             float clip_high, float beta, float* loss, float* logp, void* dlogits,
                             int64_t ldd, void* ws, size_t ws_bytes, void* stream);

/* Preference loss over paired log ratios.  n_examples = 2 n_pairs: pair p's
 * chosen sequence is example p, its rejected one example n_pairs + p.
 *     log_ratio[i] = sum_t w (logp - logp_ref)      (over tokens that count)
 *     h = beta (log_ratio[p] - log_ratio[n_pairs + p]) - margin
 *     loss[p] = pw ((1 - e) softplus(-h) + e softplus(h)),  e = label_smoothing
 *                                  (a term of factor 0 is 0, also at infinite h;
 *                                  so are the loss and the rows of dlogits of a
 *                                  pair of weight 0, whatever its logits hold)
 *     c = dloss/dlogp = +-w pw beta (e sigma(h) - (1 - e) sigma(-h))
 *                                  (+: chosen, -: rejected)
 *     dlogits[row, j] = s c ([j = target] - exp(logp_j))
 * Without logp_ref (NULL) the ratios are the log-probabilities themselves;
 * weights of 1 / tokens make them means.  Sums over tokens are formed in fp64
 * in a fixed order.  The gradient needs both sequences' sums first, so the
 * logits are read twice.
 *   logp_ref     device fp32 [n_rows] or NULL
 *   pair_weight  device fp32 [n_pairs] or NULL (1)
 *   beta, margin finite;  label_smoothing in [0, 1]
 *   loss         device fp32 [n_pairs]
 *   log_ratio    device fp32 [n_examples] or NULL
 *   logp, dlogits, ldd  as attr_policy_loss
 *   ws           attr_preference_loss_workspace_size(rows) bytes */
size_t attr_preference_loss_workspace_size(const attr_token_rows* rows);
attr_status attr_preference_loss(const attr_token_rows* rows, const float* logp_ref,
                                 const float* pair_weight, float beta, float margin,
                                 float label_smoothing, float* loss, float* log_ratio, float* logp,
                                 void* dlogits, int64_t ldd, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* (5) attr_adamw_step: one AdamW step over many tensors.                    */
/* ------------------------------------------------------------------------ */

/* One tensor of n contiguous elements (host struct with device pointers; any
 * element alignment).  With 8-bit states m and v hold E4M3 values in blocks of
 * 256 elements, the last one as long as what is left: m_e = m_scale[b] m[e],
 * and v holds the root of the second moment, v_e = (v_scale[b] v[e])^2; a
 * block's scale is its largest magnitude, or 2^-100 where that is less, over
 * 448.  Zeroed states and scales are those of step 0. */
typedef struct {
  void* p;          /* weights, p_dtype; with a master: its rounding, written and never read */
  const void* g;    /* gradients, g_dtype */
  void* m;          /* first moment, state_dtype */
  void* v;          /* second moment, or its root (8-bit), state_dtype */
  float* master;    /* fp32 weights that the step updates, or NULL: p itself */
  float* m_scale;   /* 8-bit states: fp32 [(n + 255) / 256]; else NULL */
  float* v_scale;
  int64_t n;        /* 0 <= n < 2^40 */
  float lr_scale;   /* times lr for this tensor */
  float weight_decay;
} attr_adamw_tensor;

/* For every element, with g' = grad_scale g (grad_scale a device scalar, so
 * that clipping by the gradients' norm needs no host read; NULL: 1):
 *     m = beta1 m + (1 - beta1) g',   v = beta2 v + (1 - beta2) g'^2
 *     x = x - lr' wd x - lr' (m / (1 - beta1^step))
 *                        / (sqrt(v / (1 - beta2^step) + eps_root) + eps)
 * with lr' = lr lr_scale, x the weight (its master where there is one).  All
 * in fp32 without contraction, so the result does not depend on how the work is
 * split; the step is (m lr'/(1 - beta1^step)) times the reciprocal of the root,
 * both products rounded, the root and the reciprocal within an ulp each.
 * step, lr and the other numbers enter the launch as they are: a graph that
 * captured this call repeats that one step, with its rate and its corrections.
 * 8-bit states are
 * encoded after the update: m to the nearest E4M3 value (ties to even), the
 * root of v likewise but never to zero while v is positive (a second moment
 * rounded to zero would make the next step huge).
 * E4M3 keeps a root within 6.25%: between steps a stored second moment follows
 * its block's scale exactly, and its place in the block only by changes of
 * that size.  A root that is too small for its gradients thus grows only while
 * (1 - beta2) (g'^2 / v - 1) is more than about 0.13: it may stay at half of a
 * steady |g'| with beta2 = 0.95, at a twelfth with 0.999 (steps up to 12 times as
 * long as those of 32-bit states).  A NaN or infinity in a block's new states
 * makes the block's scale NaN.
 *   tensors    (host) [n_tensors], 0 <= n_tensors; their buffers must not
 *              overlap
 *   p_dtype    ATTR_F32, ATTR_BF16 or ATTR_F16 (the last two with or without
 *              masters); g_dtype the same three; state_dtype ATTR_F32 or
 *              ATTR_E4M3
 *   step       >= 1 (the first step is 1)
 *   beta1, beta2 in [0, 1);  lr finite
 *   eps        0 or in [2^-126, 3e38];  eps_root 0 or in [2^-149, 3e38] (fp32
 *              divides by their sums; with both 0 a weight whose second moment
 *              is 0 becomes NaN, as in the formula) */
attr_status attr_adamw_step(const attr_adamw_tensor* tensors, int32_t n_tensors, attr_dtype p_dtype,
                            attr_dtype g_dtype, attr_dtype state_dtype, int64_t step, double lr,
                            double beta1, double beta2, double eps, double eps_root,
                            const float* grad_scale, void* stream);

/* ------------------------------------------------------------------------ */
/* (5b) attr_muon_step: one Muon step over many matrices.                    */
/* ------------------------------------------------------------------------ */

/* One weight matrix of rows x cols contiguous elements, row-major, with its
 * gradient and momentum laid out the same (host struct with device pointers; any
 * element alignment).  A zeroed momentum is that of step 0. */
typedef struct {
  void* p;          /* weights, p_dtype; with a master: its rounding, written and never read */
  const void* g;    /* gradients, g_dtype */
  float* m;         /* momentum */
  float* master;    /* fp32 weights that the step updates, or NULL: p itself */
  int64_t rows, cols;  /* 0 <= rows, cols <= 2^20; see below for their product */
  float lr_scale;   /* times lr for this matrix: of its update and of its decay */
  float weight_decay;  /* to scale the update alone by f: lr_scale f and weight_decay / f */
} attr_muon_matrix;

/* For every matrix, with g' = grad_scale g (a device scalar, or NULL: 1):
 *     m = momentum m + (1 - momentum) g'
 *     u = momentum m + (1 - momentum) g'   (nesterov; with the new m), else m
 *     X = u / |u|_F, then `steps` times, with A = X X^T:
 *     X = a X + (b A + c A A) X,   a = 3.4445, b = -4.7750, c = 2.0315
 * (the coefficients published with the method; K. Jordan and others, 2024)
 *     x = x - lr' wd x - lr' X,    lr' = lr lr_scale
 * The polynomial takes singular values in (0, 1] towards 1 (after five steps those from
 * 0.002 on lie in [0.68, 1.21]), so X approaches the orthogonal factor of u.
 * Where a matrix is not square its longer side is multiplied last.  A matrix
 * whose u is zero has X = 0; one with a NaN or an infinity in u becomes NaN.
 * m is fp32 without contraction, the norm fp64; the iteration runs on the matrix
 * cores with fp32 sums and its operands (X, A, a I + b A + c A A) rounded
 *   pairs = 0  to fp16, 11 bits: X is off by 1.2e-3 to 1.5e-3 of its norm, where a few
 *              directions carry most of u by more (four of 512 with 10 times the rest's
 *              norm: 3e-3 to 5e-3, with 100 times 2e-2 to 4e-2);
 *   pairs = 1  to pairs of fp16, 22 bits: three times the products, X off by 1e-6 to 4e-6
 *              (such directions with 100 times the rest: 7e-6).
 * Matrices whose shorter side is at most 64 run in fp64 on their products by themselves,
 * whatever `pairs`: X off by some 1e-7.  The same call gives the same bits; the order of
 * a larger matrix's sums depends on the sizes of all matrices of the call.
 * The numbers enter the launches as they are: a graph that captured this call
 * repeats the step with its rate.
 *   mats       (host) [n_mats], 0 <= n_mats; their buffers must not overlap (gradients
 *              may overlap gradients).  With t the longer side and s' the shorter one
 *              rounded up to a multiple of 64, t s' < 2^30
 *   p_dtype, g_dtype  ATTR_F32, ATTR_BF16 or ATTR_F16
 *   momentum   in [0, 1);  steps 1 to 16;  lr finite
 *   ws         attr_muon_step_workspace_size(mats, n_mats, pairs) bytes, 256-byte
 *              aligned: some 8 bytes (pairs: 16) for each element of the matrices that
 *              are worked on together, which are taken in turn where they are many,
 *              and up to 64 MB for sums of parts where they are few */
size_t attr_muon_step_workspace_size(const attr_muon_matrix* mats, int32_t n_mats, int32_t pairs);
attr_status attr_muon_step(const attr_muon_matrix* mats, int32_t n_mats, attr_dtype p_dtype,
                           attr_dtype g_dtype, double lr, double momentum, int32_t nesterov,
                           int32_t steps, int32_t pairs, const float* grad_scale, void* ws,
                           size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* (6) Embedding and layer norm of token rows, and their gradients.          */
/* ------------------------------------------------------------------------ */

/* The rows of a batch: token t of example i is row (row_offset ? row_offset[i] :
 * i * T) + t, as in attr_project.  Rows of tokens t < length[i] that lie in
 * [0, n_rows) are INSIDE; nothing else is read.  Of the outputs the rows inside are
 * written, and without row_offset the padding rows i * T + t, t < T, too (as
 * zeros); no others.  The ranges of two examples must not overlap.
 * Read only during the call (host struct with device pointers). */
typedef struct {
  int64_t n_rows;          /* rows of every token tensor of the call */
  int64_t n_examples, T;   /* n_examples * T < 2^31; without row_offset n_rows >= n_examples * T */
  const int64_t* row_offset;  /* device [n_examples] or NULL (then i * T) */
  const int32_t* length;      /* device [n_examples] or NULL (then T); clamped to [0, T] */
} attr_rows;

/* out[row] = scale * table[token[row]] for the rows inside; a row whose token is
 * outside [0, V) is zeros.  The product is fp32, rounded once.
 *   token       device int64 [n_rows]
 *   table       device [V, d], row stride ldt >= d, any type, stride and element
 *               alignment; 1 <= V <= 2^28, 1 <= d <= 65536
 *   out         device [n_rows, d], row stride ldo >= d; overlaps no input */
attr_status attr_embed(const attr_rows* rows, const int64_t* token, const void* table,
                       attr_dtype table_dtype, int64_t V, int64_t d, int64_t ldt, float scale,
                       void* out, attr_dtype out_dtype, int64_t ldo, void* stream);

/* The table's gradient:
 *     dtable[v] = scale * sum of dout[row] over the rows inside whose token is v
 * for every v in [0, V) (zeros where there is none), or with accumulate added to
 * the rows of dtable whose tokens the batch holds, the others left alone.  A token's
 * rows are added up in fp32 in the order of their slots, up to 128 of them at a time
 * (of a sorted batch: 64), and these sums in fp64.  The same bits for the same call.
 *   dout        device [n_rows, d], row stride ldd >= d; n_rows below 2^32
 *   dtable      device [V, d], row stride ldt >= d; overlaps no input
 *   ws          attr_embed_backward_workspace_size(rows, V, d) bytes, 256-byte aligned */
size_t attr_embed_backward_workspace_size(const attr_rows* rows, int64_t V, int64_t d);
attr_status attr_embed_backward(const attr_rows* rows, const int64_t* token, const void* dout,
                                attr_dtype dout_dtype, int64_t ldd, int64_t V, int64_t d,
                                float scale, void* dtable, attr_dtype dtable_dtype, int64_t ldt,
                                int32_t accumulate, void* ws, size_t ws_bytes, void* stream);

/* Layer norm of every row x inside:
 *     mean = sum_j x_j / d,   rstd = 1 / sqrt(sum_j (x_j - mean)^2 / d + eps)
 *     y_j = (x_j - mean) rstd w_j + b_j
 * in fp32 (the sums over a row too), y rounded once.  A row whose squares pass
 * fp32's range has rstd 0, one whose sum does becomes NaN; with eps = 0 a row of equal
 * values may be NaN.
 *   x, y        device [n_rows, d], any types, strides >= d and element alignment;
 *               1 <= d <= 32768.  y may be x itself with the same type and stride; any
 *               other overlap is ATTR_ERR_INVALID_ARG
 *   weight, bias  device [d] of w_dtype, or NULL (1 and 0)
 *   eps         finite, >= 0
 *   mean, rstd  device fp32 [n_rows] or NULL: what the backward pass takes (padding
 *               rows: 0) */
attr_status attr_layer_norm(const attr_rows* rows, const void* x, attr_dtype x_dtype, int64_t d,
                            int64_t ldx, const void* weight, const void* bias, attr_dtype w_dtype,
                            float eps, void* y, attr_dtype y_dtype, int64_t ldy, float* mean,
                            float* rstd, void* stream);

/* Its gradient.  With u = (x - mean) rstd and e = dy w for every row inside:
 *     dx_j = rstd (e_j - sum_k e_k / d - u_j sum_k e_k u_k / d)
 *     dweight_j = sum of dy_j u_j,   dbias_j = sum of dy_j
 * summed over all rows inside, or with per_example over those of each example: the
 * gradients that attribution compresses and stores are per example.  accumulate adds
 * to what dweight and dbias hold.  Sums over a workgroup's rows are fp32, those of
 * workgroups fp64, in a fixed order.
 *   dy          device [n_rows, d] of dy_dtype, stride lddy >= d
 *   x, mean, rstd  what the forward pass took and gave
 *   dx          device [n_rows, d] of x's type, stride lddx, or NULL; may be x or dy
 *               itself with the same type and stride
 *   dweight     device fp32 [d], or with per_example [n_examples, d] of row stride
 *               ldw >= d (the columns of a wider row of gradients); or NULL
 *   dbias       likewise with ldb
 *   ws          attr_layer_norm_backward_workspace_size(rows, d, per_example) bytes */
size_t attr_layer_norm_backward_workspace_size(const attr_rows* rows, int64_t d, int32_t per_example);
attr_status attr_layer_norm_backward(const attr_rows* rows, const void* dy, attr_dtype dy_dtype,
                                     int64_t lddy, const void* x, attr_dtype x_dtype, int64_t d,
                                     int64_t ldx, const float* mean, const float* rstd,
                                     const void* weight, attr_dtype w_dtype, void* dx, int64_t lddx,
                                     float* dweight, int64_t ldw, float* dbias, int64_t ldb,
                                     int32_t per_example, int32_t accumulate, void* ws,
                                     size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* Calibration (not part of the method): the rates this GPU sustains, used  */
/* as measured peaks beside the nominal ones.                               */
/* ------------------------------------------------------------------------ */

/* Streams `bytes` (a multiple of 16, x 16-byte aligned) from device memory
 * once with non-temporal 16-byte loads and no write stream (the result is
 * folded into registers; `sink`, a device word, is written only on an
 * improbable value).  Time it to get the achievable HBM read bandwidth. */
attr_status attr_probe_read(const void* x, size_t bytes, void* sink, void* stream);
/* Runs n_mfma (a multiple of 8, > 0) fp16 16x16x32 MFMAs per wave on 512
 * workgroups of four waves (two waves per SIMD on 256 CUs), operands in
 * registers: 2 * 16 * 16 * 32 * n_mfma * 2048 flops.  Time it to get the
 * achievable dense fp16 matrix-core rate.  `sink`: a device float. */
attr_status attr_probe_mfma(int64_t n_mfma, void* sink, void* stream);

/* ------------------------------------------------------------------------ */
/* Diagnostics.                                                             */
/* ------------------------------------------------------------------------ */

/* Message of the last failed call on this thread ("" if none); valid until
 * the next call on this thread. */
const char* attr_last_error(void);
/* Static name of a status code. */
const char* attr_status_string(attr_status status);
/* ATTR_ABI_VERSION of the loaded library. */
int attr_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* ATTR_H_ */
