/*
 * compactor.h - C ABI of the B200 (sm_100a) implementation of Compactor's prefill-time KV-cache
 * compression pass: approximate leverage scoring of the keys (Algorithm 1), optional blend with
 * a caller-supplied attention score (Eq. 6), per-head top-ceil(r N) selection (Section 3.4) and
 * compaction of the retained K/V rows into a dense per-head cache.
 *
 * Conventions
 *   - Every function returns an int status: COMPACTOR_OK (0) or a negative COMPACTOR_E_* code.
 *     Nothing throws.  Argument errors are detected before any work is enqueued.
 *   - "device" pointers are CUDA device pointers of the current device; "host" pointers are
 *     ordinary host memory, read before the call returns.  The library never allocates or frees
 *     device memory: every buffer, including the workspace, belongs to the caller.
 *   - Device work is enqueued on the caller's stream (`stream` is a cudaStream_t passed as
 *     void*; NULL is the default stream) and the call returns without synchronising.  Everything
 *     enqueued is a kernel or a memset (the prefix tables travel as kernel arguments, 239
 *     sequences per small launch), so the call can be recorded into a CUDA graph and replayed on
 *     new contents of the same buffers.
 *   - Keys/values are bf16 with the d channels of a token contiguous; the other three strides
 *     (layer, KV head, token) are given in ELEMENTS and must be multiples of 8 (16 bytes); base
 *     pointers must be 16-byte aligned.  d must be 128.  1 <= m <= 128.
 *   - Sequences are packed back to back along the token axis: sequence b owns tokens
 *     [cu_seqlens[b], cu_seqlens[b+1]) of every (layer, head).  A "unit" is one
 *     (layer, head, sequence) triple; unit id = (layer * heads + head) * batch + b.
 *     Units are scored and selected independently (Section 3, Notation: heads are treated
 *     one by one).
 *   - Kept rows of sequence b occupy rows [cu_keep[b], cu_keep[b+1]) of every (layer, head)
 *     block of the outputs, cu_keep = prefix sums of keep_counts; total_keep = cu_keep[batch].
 *   - Outputs must not alias inputs or the workspace.
 *   - `status` (device, int32 [layers*heads*batch], may be NULL) receives per-unit flags once the
 *     stream has run: bit 0 = the unit's Gram matrix held a non-finite value (scores of the unit
 *     are unspecified), bit 1 = the sketched Gram matrix was numerically rank deficient (the
 *     singular directions contribute nothing, as a pseudo-inverse would), bit 2 = a bounded
 *     device-side wait ran out.
 *   - On problems with at most 600 MB of keys the kernels of a call are launched as a chain of
 *     programmatic dependent launches (each may set up while its predecessor drains); results do
 *     not depend on it.  The library reads a few environment variables at every call, none of which
 *     changes a result: COMPACTOR_NO_PDL=1 (no chained launches), COMPACTOR_PDL_MASK,
 *     COMPACTOR_GRAM_BLOCK / COMPACTOR_SCORE_BLOCK (block lengths of the two sweeps, a power of two
 *     from 256 to 65536 tokens), COMPACTOR_FUSED_SWEEP and its companions (an experimental
 *     one-kernel sweep).  They are measuring aids; leave them unset.
 */
#ifndef COMPACTOR_H_
#define COMPACTOR_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define COMPACTOR_OK                  0
#define COMPACTOR_E_INVALID_ARGUMENT -1   /* null pointer, bad size, bad stride or alignment      */
#define COMPACTOR_E_UNSUPPORTED      -2   /* d != 128, m outside [1, 128], more than 64 query heads per KV head */
#define COMPACTOR_E_WORKSPACE        -3   /* workspace smaller than compactor_workspace_bytes()  */
#define COMPACTOR_E_CUDA             -4   /* a CUDA runtime call failed (see cudaGetLastError)   */
#define COMPACTOR_E_TOO_LARGE        -5   /* problem exceeds the library's built-in scratch      */

#define COMPACTOR_STATUS_NONFINITE   1
#define COMPACTOR_STATUS_RANK        2
#define COMPACTOR_STATUS_TIMEOUT     4
#define COMPACTOR_STATUS_PAGE        8    /* a page that is none (paged cache)           */
#define COMPACTOR_STATUS_CAPACITY   16    /* a length beyond the unit's pages            */

/* Small factorisations for compactor_score_variant (Appendix C). */
#define COMPACTOR_FACTOR_CHOLESKY    0    /* G = L L^T: the R factor of the QR route          */
#define COMPACTOR_FACTOR_EIG         1    /* G = V Lambda V^T with a floor on the eigenvalues */

/* A strided bf16 tensor [layers][heads][total_tokens][d] in device memory. */
typedef struct compactor_mat {
    const void* ptr;          /* device, 16-byte aligned                           */
    int64_t stride_layer;     /* elements between consecutive layers               */
    int64_t stride_head;      /* elements between consecutive KV heads             */
    int64_t stride_token;     /* elements between consecutive tokens (>= d)        */
} compactor_mat;

/* Problem shape.  cu_seqlens is a HOST array of batch+1 non-decreasing offsets starting at 0. */
typedef struct compactor_shape {
    int32_t layers;
    int32_t heads;
    int32_t d;                /* head dimension; must be 128                       */
    int32_t m;                /* sketch dimension, 1..128 (the paper uses 48)      */
    int32_t batch;            /* number of packed sequences                        */
    const int32_t* cu_seqlens;/* host, [batch+1]                                   */
} compactor_shape;

/* Library version (major*10000 + minor*100 + patch). */
int compactor_version(void);

/* Static description of a status code. */
const char* compactor_error_string(int code);

/*
 * Algorithm 1, line 1: a Gaussian sketch Phi [d][m] (row-major fp32, HOST memory) with iid
 * N(0, 1/m) entries from a counter-based generator, so that any caller can reproduce it:
 * word i = splitmix64 finaliser of seed + (i+1)*0x9E3779B97F4A7C15; words (2p, 2p+1) give
 * u1 = ((x>>11)+1) 2^-53 and u2 = (x>>11) 2^-53; Box-Muller (sqrt(-2 ln u1) cos/sin(2 pi u2))
 * gives row-major entries 2p and 2p+1, each divided by sqrt(m) in double and rounded to fp32.
 * Any other Phi may be passed to the scoring calls instead; scores do not depend on its scale.
 */
int compactor_make_sketch(uint64_t seed, int32_t d, int32_t m, float* phi_host);

/*
 * Appendix D: a subsampled randomised Hadamard sketch, written out as a matrix Phi [d][m] (HOST,
 * row-major fp32) that the scoring calls take like any other sketch: Phi = (1/sqrt(m)) D H R^T with
 * D random signs, H the Sylvester-Walsh-Hadamard matrix of order d (d a power of two) and R a
 * choice of m columns without replacement.  Random bits come from the splitmix64 stream of
 * compactor_make_sketch: word i (i < d) gives the sign of row i (bit 0 set = minus); word d + j
 * drives step j of a Fisher-Yates shuffle of 0..d-1 (swap position j with j + word mod (d - j)),
 * whose first m entries are the chosen columns.
 */
int compactor_make_sketch_srht(uint64_t seed, int32_t d, int32_t m, float* phi_host);

/*
 * Number of retained tokens for a sequence of n tokens at retention ratio r (Section 3,
 * Preliminaries: k = ceil(r N)): ceil evaluated on the double product, clamped to [1, n];
 * 0 when n <= 0.  Returns the count (never an error code).
 */
int64_t compactor_keep_count(int64_t n, double r);

/*
 * Context-calibrated retention (Section 3.5): with b = alpha*nll + beta and the fitted curve
 * f(r) = (exp(rb-b) - exp(-b)) / (1 - exp(-b)), writes the r with f(r) = tau, i.e.
 * r* = log(1 + tau*(e^b - 1)) / b (r* = tau when b = 0).  tau must lie in (0, 1].
 */
int compactor_calibrated_ratio(double nll, double alpha, double beta, double tau, double* r_out);

/*
 * Fit of the calibration curve (Section 3.5): finds (alpha, beta) minimising the asymmetric mean
 * squared error sum_i w_i (f_{alpha,beta}(r_i, nll_i) - y_i)^2 / n over n training triples, where
 * f is the curve of compactor_calibrated_ratio with b = alpha*nll_i + beta, y_i is the measured
 * NLL ratio at retention r_i, and w_i = under_weight (>= 1) when the curve predicts more quality
 * than was measured (which would make r* too small), else 1; the paper weights those errors
 * higher without giving the weight.  Host arrays, host computation (Levenberg-Marquardt from a
 * grid of starting points); loss_out may be NULL.
 */
int compactor_fit_calibration(int64_t n, const double* r, const double* nll, const double* y,
                              double under_weight, double* alpha_out, double* beta_out, double* loss_out);

/*
 * Token-averaged negative log-likelihood (Section 3.5): for each of `batch` sequences, the mean
 * over its scored rows of -log softmax(logits_i)[targets_i].  This is the context statistic NLL(c)
 * that compactor_calibrated_ratio turns into a retention ratio.
 *   logits       device, [rows][vocab] with `row_stride` elements between rows; bf16
 *                (logits_dtype COMPACTOR_DTYPE_BF16) or fp32 (COMPACTOR_DTYPE_F32); 16-byte aligned,
 *                row_stride * element size a multiple of 16.
 *   targets      device int32 [rows]: the token each row is scored on; a negative id (or one
 *                >= vocab) leaves the row unscored: its row result is 0 and it does not count in
 *                the average.
 *   cu_rows      HOST int32 [batch+1], non-decreasing from 0 to rows: the rows of each sequence.
 *   row_nll_out  device fp32 [rows], required: the per-row terms (also the kernel's scratch).
 *   nll_out      device fp64 [batch]: the averages (0 for a sequence with no scored row).
 * Arithmetic: one streaming pass in fp32 (running maximum, base-2 exponentials), averages in fp64
 * in a fixed order.  No workspace.  Errors: COMPACTOR_E_INVALID_ARGUMENT for null pointers, bad
 * alignment, vocab < 1, an unknown dtype or an inconsistent cu_rows.
 */
#define COMPACTOR_DTYPE_BF16 0
#define COMPACTOR_DTYPE_F32  1
int compactor_nll(const void* logits, int32_t logits_dtype, int64_t rows, int32_t vocab, int64_t row_stride,
                  const int32_t* targets, int32_t batch, const int32_t* cu_rows,
                  float* row_nll_out, double* nll_out, void* stream);

/*
 * Bytes of device workspace that compactor_score and compactor_compress need for this shape.
 * compactor_select and compactor_compact only need a small table at its start and accept any
 * workspace of at least 16*(batch+1) bytes rounded up to 256 (compactor_select uses whatever
 * follows the table as scratch, see there).  The workspace must be 256-byte aligned; its
 * contents need not be preserved between calls.  Returns 0 for an invalid shape.
 */
size_t compactor_workspace_bytes(const compactor_shape* shape);

/*
 * Approximate leverage scores of every unit (Algorithm 1, lines 2-6) and the blend of Eq. 6.
 *   k_score      keys to score (the paper scores the keys before positional encoding).
 *   phi          device, fp32 [d][m] row-major: the sketch, shared by all units.
 *   attn_scores  device fp32 [layers][heads][total_tokens] or NULL.  If given, the output is
 *                s = z(attn) + lambda * z(o) per unit (population std; a term with zero std
 *                contributes 0); if NULL the output is the outlier score o itself.
 *   scores_out   device fp32 [layers][heads][total_tokens].
 * With m = d and any invertible phi (the identity, say) the result is the exact leverage score
 * of Definition 1 / Eq. 1, the paper's "exact" ablation; sketches wider than 64 columns run in a
 * slower configuration of the same kernels.
 * The small factorisation is a Cholesky factorisation of G = (K Phi)^T (K Phi) in fp64 - one of
 * the algebraically equal routes the paper allows (Section 3.2, Appendix C); Gram sums are fp32
 * within runs of 512 tokens and fp64 beyond.
 */
int compactor_score(const compactor_shape* shape, compactor_mat k_score, const float* phi,
                    const float* attn_scores, float lambda, float* scores_out,
                    int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * compactor_score with the small factorisation chosen by the caller (Appendix C).
 *   factorization  COMPACTOR_FACTOR_CHOLESKY: exactly compactor_score.  Cholesky of G is the R
 *                  factor of the appendix's QR route (K Phi = Q R, score = squared row norm of Q).
 *                  COMPACTOR_FACTOR_EIG: the appendix's eigendecomposition route.  G = V Lambda V^T
 *                  (cyclic Jacobi, fp64), every eigenvalue raised to at least eig_floor,
 *                  score_i = || k_i Phi V Lambda^-1/2 ||^2.  Unlike the other routes the result
 *                  depends on the scale of Phi once the floor is active; the status bit
 *                  COMPACTOR_STATUS_RANK then reports that some eigenvalue was below the floor.
 *   eig_floor      the floor (the paper suggests about 1e-6); must be positive and finite;
 *                  ignored for COMPACTOR_FACTOR_CHOLESKY.
 * The eigendecomposition route takes m <= 64 (COMPACTOR_E_UNSUPPORTED beyond).
 * All other arguments, the workspace and the error behaviour are those of compactor_score.
 */
int compactor_score_variant(const compactor_shape* shape, compactor_mat k_score, const float* phi,
                            int32_t factorization, double eig_floor,
                            const float* attn_scores, float lambda, float* scores_out,
                            int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Per-unit top-k (Section 3.4: the ceil(r N) highest-scoring tokens are kept, here per head).
 *   scores       device fp32 [layers][heads][total_tokens].
 *   keep_counts  host int32 [batch]: tokens kept per sequence (0 <= keep <= length), the same
 *                for every layer and head.
 *   idx_out      device int32 [layers][heads][total_keep]: for each unit the indices (local to
 *                the sequence, 0-based) of its keep_counts[b] largest scores, ascending.  Equal
 *                scores are ranked by lower index first.  NaN scores rank above +inf.
 * One CTA selects a unit.  Where that would leave most of the GPU idle (fewer units than SMs and
 * sequences of 10^5 tokens or more) and the workspace is the size compactor_workspace_bytes()
 * gives, every score vector is cut into slices that share a histogram and a candidate list in the
 * workspace; the indices are the same either way.
 */
int compactor_select(const compactor_shape* shape, const float* scores,
                     const int32_t* keep_counts, int32_t* idx_out,
                     int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Compaction: k_out[l][h][cu_keep[b]+j][:] = k_cache[l][h][cu_seqlens[b]+idx[l][h][cu_keep[b]+j]][:]
 * and likewise for v, as bit copies.  k_out / v_out are dense bf16 [layers][heads][total_keep][d].
 * Indices outside [0, length) are skipped (their output rows are left untouched).
 */
int compactor_compact(const compactor_shape* shape, compactor_mat k_cache, compactor_mat v_cache,
                      const int32_t* idx, const int32_t* keep_counts,
                      void* k_out, void* v_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The whole pass: score k_score, select, and gather rows of k_cache / v_cache.
 * k_score may be the same tensor as k_cache.  scores_out may be NULL (scores then live only in
 * the workspace); idx_out, k_out, v_out as above.
 */
int compactor_compress(const compactor_shape* shape, compactor_mat k_score, compactor_mat k_cache,
                       compactor_mat v_cache, const float* phi, const float* attn_scores,
                       float lambda, const int32_t* keep_counts,
                       float* scores_out, int32_t* idx_out, void* k_out, void* v_out,
                       int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * compactor_compress with stage markers, for measurement (the paper reports one wall-clock
 * number per context length, Fig. 1; this splits ours by stage).  stage_events is a HOST array of
 * n_events cudaEvent_t handles created by the caller (NULL entries are skipped).  They are
 * recorded on the stream: [0] before the first kernel, [1] after the Gram pass, [2] after the
 * factorisation, [3] after the scoring pass, [4] after the blend (recorded even when there is
 * none), [5] after selection, [6] after compaction.  Results are identical to compactor_compress.
 */
#define COMPACTOR_N_STAGE_EVENTS 7
int compactor_compress_profiled(const compactor_shape* shape, compactor_mat k_score, compactor_mat k_cache,
                                compactor_mat v_cache, const float* phi, const float* attn_scores,
                                float lambda, const int32_t* keep_counts,
                                float* scores_out, int32_t* idx_out, void* k_out, void* v_out,
                                int32_t* status, void* workspace, size_t workspace_bytes, void* stream,
                                void* const* stage_events, int32_t n_events);

/*
 * Attention term of the score (Eq. 5): for every unit, a = concat_i 1^T softmax(scale * Q[i] K[i]^T)
 * over chunks i of `chunk` consecutive tokens of the sequence (no causal mask), summed over the
 * q_per_kv query heads that share the KV head, then mean-pooled.  The result is what
 * compactor_score / compactor_compress take as attn_scores.
 *   q        bf16 [layers][heads * q_per_kv][total_tokens][d]; query head j of KV head h is
 *            head index h * q_per_kv + j.  Same stride and alignment rules as the keys.
 *   chunk    must be 256 (the paper's setting).
 *   scale    > 0; the paper's equation prints no scale, attention layers use 1/sqrt(d).
 *   pool     odd window of the mean pooling (1 = none): centred, zero beyond the ends of the
 *            sequence, divided by `pool` (the paper pools but does not give the window).
 *   attn_out device fp32 [layers][heads][total_tokens].
 * The last, shorter chunk of a sequence is a softmax over its own keys.  Exponentials are
 * rounded to fp16 before they are summed over the query rows on the tensor cores (fp32
 * accumulation).  Workspace: compactor_workspace_bytes() suffices (16*(batch+1) bytes rounded up
 * to 256, plus 4 bytes per output element when pool > 1).
 */
int compactor_attention_scores(const compactor_shape* shape, compactor_mat q, compactor_mat k,
                               int32_t q_per_kv, int32_t chunk, float scale, int32_t pool,
                               float* attn_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * compactor_attention_scores (Eq. 5) with the per-unit status word of the other device calls:
 * `status` (device int32 [layers*heads*batch], may be NULL) is cleared when the call starts and
 * receives COMPACTOR_STATUS_TIMEOUT for every unit of a CTA one of whose bounded device-side waits
 * ran out (the attention term of such a unit is unspecified).  Everything else as above.
 */
int compactor_attention_scores_status(const compactor_shape* shape, compactor_mat q, compactor_mat k,
                                      int32_t q_per_kv, int32_t chunk, float scale, int32_t pool,
                                      float* attn_out, int32_t* status, void* workspace, size_t workspace_bytes,
                                      void* stream);

/*
 * Selection across the heads of a layer (Section 3.4 allows the top scores to be taken over all
 * heads instead of within each head; the paper's experiments use such head-adaptive budgets).
 * For every (layer, sequence b) the heads * keep_counts[b] largest scores over all heads are kept,
 * ranked by (score descending, head ascending, index ascending), so heads keep different numbers
 * of tokens while the layer keeps as many as per-head selection would.
 *   idx_out           device int32 [layers][heads * total_keep]: layer l, sequence b owns entries
 *                     [heads * cu_keep[b], heads * cu_keep[b+1]); inside that block head h owns
 *                     [off[h], off[h+1]) with off = head_offsets_out[l][b][0 .. heads]; indices are
 *                     local to the sequence and ascending within a head.
 *   head_offsets_out  device int32 [layers][batch][heads + 1], off[0] = 0, off[heads] = heads * keep_counts[b].
 * heads must not exceed 64.  Workspace: compactor_across_heads_workspace_bytes() (the tables, and
 * per (layer, sequence) a histogram, a candidate list and per-slice counts: every head's scores are
 * cut into slices that are counted and emitted by CTAs of their own).
 * compactor_compact_across_heads gathers K/V rows in exactly that order into
 * k_out / v_out [layers][heads * total_keep][d] (bit copies; out-of-range indices are skipped).
 */
size_t compactor_across_heads_workspace_bytes(const compactor_shape* shape);
int compactor_select_across_heads(const compactor_shape* shape, const float* scores,
                                  const int32_t* keep_counts, int32_t* idx_out, int32_t* head_offsets_out,
                                  void* workspace, size_t workspace_bytes, void* stream);
int compactor_compact_across_heads(const compactor_shape* shape, compactor_mat k_cache, compactor_mat v_cache,
                                   const int32_t* idx, const int32_t* head_offsets,
                                   const int32_t* keep_counts, void* k_out, void* v_out,
                                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * The paper's whole method in one call: attention term (Eq. 5) -> leverage scores (Algorithm 1)
 * -> blend (Eq. 6) -> selection within each head or across the heads of a layer (Section 3.4) ->
 * gather.  The experiments of Section 4 use chunk 256, lambda 0.3, m 48 and selection across heads.
 *   options      HOST struct:
 *     selection      COMPACTOR_SELECT_PER_HEAD or COMPACTOR_SELECT_ACROSS_HEADS.
 *     factorization  COMPACTOR_FACTOR_CHOLESKY or COMPACTOR_FACTOR_EIG (with eig_floor), as in
 *                    compactor_score_variant.
 *     lambda         weight of the leverage term in Eq. 6 (ignored without an attention term).
 *     q_per_kv       query heads per KV head; 0 = no attention term: the score is the leverage
 *                    score alone and q is ignored.
 *     chunk, scale, pool   as in compactor_attention_scores (chunk must be 256).
 *   q            queries, bf16 [layers][heads * q_per_kv][total_tokens][d] (ignored if q_per_kv = 0).
 *   k_score      keys scored by Algorithm 1 (the paper: before positional encoding);
 *   k_cache      keys the attention term is taken against and the rows are gathered from (may be
 *                the same tensor as k_score);  v_cache likewise for the values.
 *   scores_out   device fp32 [layers][heads][total_tokens] or NULL: the final (blended) score.
 *   idx_out, k_out, v_out
 *                per-head selection: the layouts of compactor_select / compactor_compact;
 *                across heads: those of compactor_select_across_heads / compactor_compact_across_heads.
 *   head_offsets_out  device int32 [layers][batch][heads + 1]; across heads only (else may be NULL).
 *   status       device int32 [layers*heads*batch] or NULL; cleared once, then collects the flags of
 *                the attention and the scoring kernels.
 * Workspace: compactor_compress_full_workspace_bytes(shape, options), 256-byte aligned.  Errors as for
 * the calls it is made of; everything is checked before anything is enqueued.
 */
#define COMPACTOR_SELECT_PER_HEAD      0
#define COMPACTOR_SELECT_ACROSS_HEADS  1
typedef struct compactor_options {
    int32_t selection;
    int32_t factorization;
    double  eig_floor;
    float   lambda;
    int32_t q_per_kv;
    int32_t chunk;
    float   scale;
    int32_t pool;
} compactor_options;
size_t compactor_compress_full_workspace_bytes(const compactor_shape* shape, const compactor_options* options);
int compactor_compress_full(const compactor_shape* shape, const compactor_options* options, compactor_mat q,
                            compactor_mat k_score, compactor_mat k_cache, compactor_mat v_cache,
                            const float* phi, const int32_t* keep_counts, float* scores_out,
                            int32_t* idx_out, int32_t* head_offsets_out, void* k_out, void* v_out,
                            int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Paged cache: what the retained rows live in while a model decodes.  The paper compresses a prefill and
 * leaves the cache to the engine around it; since heads keep different tokens (and, selected across
 * heads, different numbers of them), every unit has a row of the page table and a length of its own.
 *   k_pages, v_pages  device bf16; row (page p, slot s) is the d elements at p * stride_page + s * stride_token
 *                     of either pool.  16-byte aligned; strides in elements, multiples of 8, stride_token >= d,
 *                     stride_page >= page_tokens * stride_token.  A pool may exceed 2^32 elements.
 *   mass              device fp32 [n_pages][page_tokens] or NULL: accumulated attention weight per slot; 16-byte aligned.
 *   positions         device int32 [n_pages][page_tokens] or NULL: position of the slot's token; 16-byte aligned.
 *   page_table        device int32 [layers*heads*batch][max_pages]: token t of unit u lies in slot
 *                     t % page_tokens of page page_table[u][t / page_tokens].  Entries behind a unit's
 *                     last token are not read.  A page that is written (filled, appended to, accumulated
 *                     into or evicted from) must belong to one unit only and occur once in its row; pages that
 *                     are only read may be shared.
 *   page_tokens       a power of two, 8..1024.  d must be 128.
 * Lengths are device int32 [layers*heads*batch] arrays of the caller, indexed by unit id, so that a recorded
 * call follows them; a negative length marks a row without a sequence: it is neither read nor written.
 * The calls do not change lengths except through their lengths_out arguments.  Slots behind a unit's last
 * token keep what they hold and may hold anything, not-a-number included.
 * `status` (device int32 [layers*heads*batch], may be NULL): the entries of the layers of a call are cleared when
 * it starts; COMPACTOR_STATUS_PAGE = a page id outside [0, n_pages) was met where a row was needed,
 * COMPACTOR_STATUS_CAPACITY = the unit's tokens do not fit its pages (or max_length).
 * Calls that share pages, lengths or a workspace are ordered by the caller (one stream, or events); two calls on
 * different layers may run at once if their workspaces differ.
 */
typedef struct compactor_paged_cache {
    void* k_pages;
    void* v_pages;
    int64_t stride_page;
    int64_t stride_token;
    float* mass;
    int32_t* positions;
    const int32_t* page_table;
    int32_t n_pages;
    int32_t page_tokens;
    int32_t max_pages;
    int32_t layers;
    int32_t heads;            /* KV heads */
    int32_t batch;
    int32_t d;
} compactor_paged_cache;

/* One row of d elements per (sequence, head): bf16, 16-byte aligned, strides in elements, multiples of 8. */
typedef struct compactor_rows {
    void* ptr;
    int64_t stride_seq;
    int64_t stride_head;
} compactor_rows;

/*
 * Compaction into pages: the counterpart of compactor_compact / compactor_compact_across_heads for a paged
 * cache.  Row j of a unit's kept rows goes to slot lengths[u] + j as a bit copy.
 *   shape         the prefill (heads and batch those of the cache); its layers go to the cache's layers
 *                 first_layer .. first_layer + shape->layers - 1.  m is not used (any valid value).
 *   idx           device int32 in the layout of compactor_select, or of compactor_select_across_heads when
 *                 head_offsets is given; NULL (without head_offsets, or where nothing is kept): rows 0 .. keep_counts[b] - 1
 *                 of every sequence, i.e. the tokens are appended as they are.
 *   head_offsets  device int32 [shape->layers][batch][heads + 1] from compactor_select_across_heads, or NULL.
 *   keep_counts   HOST int32 [batch], as in compactor_compact.
 *   mass_in       device fp32 [shape->layers][heads][total_tokens] (the attention term of Eq. 5 without
 *                 pooling, say) or NULL: the slots' accumulated weight starts at mass_in[token], else 0.
 *   first_position device int32 [batch] or NULL (0): the slots' positions are first_position[b] + token index.
 *   lengths       device int32 [units of the cache] or NULL (all 0): tokens a unit holds before the call.
 *   lengths_out   the same layout or NULL, may be `lengths`: tokens it holds after it (entries of other layers are
 *                 left alone).
 * A unit whose rows do not all fit its pages is left alone (COMPACTOR_STATUS_CAPACITY, length unchanged); rows whose
 * index lies outside [0, length of the sequence) are skipped and leave their slot untouched; rows whose
 * page is none are skipped (COMPACTOR_STATUS_PAGE).  No workspace.
 */
int compactor_paged_fill(const compactor_paged_cache* cache, int32_t first_layer, const compactor_shape* shape,
                         compactor_mat k_cache, compactor_mat v_cache, const int32_t* idx,
                         const int32_t* head_offsets, const int32_t* keep_counts, const float* mass_in,
                         const int32_t* first_position, const int32_t* lengths, int32_t* lengths_out,
                         int32_t* status, void* stream);

/*
 * Attention of one new token per sequence over one layer of a paged cache:
 *   y_j = scale q.k_j, capped as softcap * tanh(y_j / softcap) when softcap > 0;  p = softmax(y);
 *   out = sum_j p_j v_j;  lse = log sum_j exp(y_j).
 *   q, out       rows [batch][heads * q_per_kv]; query head j of KV head h is head h * q_per_kv + j.
 *                1 <= q_per_kv <= 64.  Rows of out must not overlap.
 *   k_new, v_new rows [batch][heads] of the new token (or both ptr NULL: attend to the cached tokens only).  The
 *                token is attended to and written to slot lengths[u] of its unit (its page must be in the table), with position
 *                new_positions[b] (device int32 [batch]; NULL: the slot's number).  `lengths` is not
 *                changed: all layers of a step see the same lengths, the caller adds 1 after the last.
 *   lengths      device int32 [units of the cache]: cached tokens, without the new one.
 *   lse_out      device fp32 [batch][heads * q_per_kv] or NULL.
 *   options (HOST): q_per_kv, scale (> 0), softcap (0: none; scale log2(e), scale / softcap and softcap log2(e) have to be normal fp32
 *                numbers), accumulate, and max_length, the most tokens a unit may have
 *                in this call, the new one included (what lies beyond the table's pages does not count).
 *                accumulate != 0 adds sum over the KV head's query heads of p_j to the weight of every cached
 *                token (cache->mass) and sets the new token's; otherwise the new token's is set to 0.
 * A unit without tokens (or with a negative length, or beyond its capacity: COMPACTOR_STATUS_CAPACITY) gives zero rows and
 * lse = -inf.  Cached tokens on a page that is none are left out (COMPACTOR_STATUS_PAGE); the new token is attended to
 * whatever its page, and not written where that is none (COMPACTOR_STATUS_PAGE).
 * Scores and sums are fp32; for the product with V a weight is the sum of two bf16 terms (within 2^-16 of it).  Results
 * do not depend on timing: a unit's partial sums are joined in a fixed order.
 * Workspace: compactor_paged_attention_workspace_bytes(), 256-byte aligned, contents not preserved; 0 = bad arguments.  When
 * accumulating it holds 4 bytes per query head for every token up to max_length (or the table's pages) of every sequence of
 * the layer: keep max_length close to what the units hold.
 */
typedef struct compactor_decode_options {
    int32_t q_per_kv;
    int32_t max_length;
    float   scale;
    float   softcap;
    int32_t accumulate;
} compactor_decode_options;
size_t compactor_paged_attention_workspace_bytes(const compactor_paged_cache* cache, const compactor_decode_options* options);
int compactor_paged_attention(const compactor_paged_cache* cache, int32_t layer, const compactor_decode_options* options,
                              compactor_rows q, compactor_rows k_new, compactor_rows v_new, const int32_t* new_positions,
                              const int32_t* lengths, compactor_rows out, float* lse_out, int32_t* status,
                              void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eviction by accumulated attention weight, for the units of `layers` layers from first_layer on.  A unit
 * with n = lengths[u] tokens and a budget B = budgets[u] (device int32 [units of the cache]) with 0 <= B < n keeps B
 * tokens: those whose position is at least next_position[b] - min(recent, B), then those of the greatest weight;
 * of equal weights the lower slots stay.  Not-a-number ranks above +inf.  (If more tokens than B are that recent, which takes repeated
 * positions, the lower slots of them stay.)  The others leave, and the holes they leave in slots [0, B) are filled from
 * behind: the j-th evicted slot below B receives row, weight and position of the j-th kept slot at or above B.  Slots
 * from B on keep what they hold.  lengths_out[u] (may be `lengths`, not `budgets`; the entries of other layers are left alone) becomes B.
 * A unit with n <= B, a negative length or a negative budget stays as it is, lengths_out[u] = lengths[u]; so does one with
 * n > max_length or beyond its pages (COMPACTOR_STATUS_CAPACITY) and one with a page that is none (COMPACTOR_STATUS_PAGE;
 * with B = 0 no page is looked at and the length becomes 0).
 *   next_position  device int32 [batch]; may be NULL when recent = 0.
 *   max_length     the most tokens a unit may have, at most 393216 (COMPACTOR_E_TOO_LARGE beyond).  It decides how the work is laid
 *                  out (what lies beyond the table's pages does not count): keep it close to what the units hold, and below 66048 where
 *                  none needs more.  256 units of 2459 tokens take 9 us, 14 with a bound of 66048 and 50 with one of 131072.
 * cache->mass is required, cache->positions when recent > 0.  No workspace.
 */
int compactor_paged_evict(const compactor_paged_cache* cache, int32_t first_layer, int32_t layers, const int32_t* lengths,
                          const int32_t* budgets, const int32_t* next_position, int32_t recent, int32_t max_length,
                          int32_t* lengths_out, int32_t* status, void* stream);

/*
 * The same cache with rows held in 4 bits.  A row of 128 channels takes 80 bytes instead of 256: 64 bytes of codes (channel 2 j in the low
 * half of byte j, 2 j + 1 in the high half), then for each group of 32 channels, in order, two bf16: a step s and the least value lo.  A
 * channel of code c stands for lo + s c.  With `least` and `greatest` of the group's 32 values
 *   s = (greatest - least) / 15 rounded up to four significant bits (0 if that is below 2^-120),  lo = least,
 *   c = ceil((x - lo) / s - 1/2), 0 where s is 0: the nearest code, the lower of two as near, at most s / 2 off (the differences are fp32's);
 * a group with a value that is not finite, or whose step exceeds 2^120, is held as not a number throughout.
 * The compactor_paged4_ calls take a compactor_paged_cache whose pools are such rows: k_pages and v_pages 16-byte aligned,
 * stride_token = 80 (the rows of a page lie back to back) and stride_page, both in BYTES, stride_page a multiple of 16 and at least 80 page_tokens.
 * A cache of one kind is refused by the calls for the other.  Everything else is as in the calls without the 4:
 *   paged4_fill       holds the rows as above instead of copying them;
 *   paged4_attention  attends to the values that the rows stand for.  The new token's row is held in 4 bits first and attended to as it is
 *                     held, so that later steps see the same.  Its products are exact before they are summed in fp32, but for two: weights enter
 *                     the product with V as two bf16 terms (within 2^-16 of the weight), and a query channel below 2^-31 (odd channels: 2^-27) of
 *                     its head's greatest is taken to within 2^-39 (2^-35) of that one.  Values are summed as s (c - 7) and lo + 7 s.  A head with a query
 *                     channel of 2^118 or more, or not finite, gives not-a-number.  Its workspace has a size of its own;
 *   paged4_evict      moves rows as they are.
 */
int compactor_paged4_fill(const compactor_paged_cache* cache, int32_t first_layer, const compactor_shape* shape,
                          compactor_mat k_cache, compactor_mat v_cache, const int32_t* idx,
                          const int32_t* head_offsets, const int32_t* keep_counts, const float* mass_in,
                          const int32_t* first_position, const int32_t* lengths, int32_t* lengths_out,
                          int32_t* status, void* stream);
size_t compactor_paged4_attention_workspace_bytes(const compactor_paged_cache* cache, const compactor_decode_options* options);
int compactor_paged4_attention(const compactor_paged_cache* cache, int32_t layer, const compactor_decode_options* options,
                               compactor_rows q, compactor_rows k_new, compactor_rows v_new, const int32_t* new_positions,
                               const int32_t* lengths, compactor_rows out, float* lse_out, int32_t* status,
                               void* workspace, size_t workspace_bytes, void* stream);
int compactor_paged4_evict(const compactor_paged_cache* cache, int32_t first_layer, int32_t layers, const int32_t* lengths,
                           const int32_t* budgets, const int32_t* next_position, int32_t recent, int32_t max_length,
                           int32_t* lengths_out, int32_t* status, void* stream);

/*
 * Rows out of the pages into dense tensors, the counterpart of the fill: row cu_seqlens[b] + j of (layer, head) becomes token
 * first[u] + j of its unit, for 0 <= j < length of sequence b in `shape` and first[u] + j < lengths[u].  Other rows keep what they hold.
 *   shape          the dense tensors' (heads and batch those of the cache); its layers are the cache's from first_layer on.  m is not used.
 *   first          device int32 [units of the cache] or NULL (0); a unit with a negative entry is left out.
 *   lengths        device int32 [units of the cache]; a unit with a negative length, or one beyond its pages (COMPACTOR_STATUS_CAPACITY), is left out.
 *   k_out, v_out   bf16 [layers][heads][total tokens][d], strides as for inputs, rows that do not overlap.  From a cache in 4 bits come the
 *                  nearest bf16 to the values that the rows stand for.
 * Rows on a page that is none are left alone (COMPACTOR_STATUS_PAGE).  No workspace.
 */
int compactor_paged_read(const compactor_paged_cache* cache, int32_t first_layer, const compactor_shape* shape, const int32_t* first,
                         const int32_t* lengths, compactor_mat k_out, compactor_mat v_out, int32_t* status, void* stream);
int compactor_paged4_read(const compactor_paged_cache* cache, int32_t first_layer, const compactor_shape* shape, const int32_t* first,
                          const int32_t* lengths, compactor_mat k_out, compactor_mat v_out, int32_t* status, void* stream);

/*
 * Attention to a few pages of every unit, chosen for each step's queries: compactor_paged_bounds keeps the least and the greatest key of every
 * page, channel by channel; compactor_paged_select scores the pages by them and writes the best as a page table of one layer, which the
 * attention calls take in the place of the cache's own (layers = 1, max_pages = pages, layer 0, the lengths written here).
 * (A cache with positions then wants new_positions: without them the attention would write the token's place in the chosen pages.)
 *   bounds         device bf16 [n_pages][2][d], 16-byte aligned: least values, then greatest, of the keys of the page's tokens (of a cache in 4 bits:
 *                  of what they stand for, rounded to bf16).  Not-a-number in a channel gives not-a-number.
 *
 * compactor_paged_bounds brings the entries of the units' pages up to date, for `layers` layers from first_layer on: after a fill, and
 * after an eviction, which moves rows between pages.
 *   first          device int32 [units of the cache] or NULL (0): pages before the one that holds this token stay as they are (after a fill
 *                  behind `lengths`: the lengths before it).
 *   max_length     the most tokens a unit may have (what lies beyond the table's pages does not count).
 * A unit with a negative length or more than max_length tokens (COMPACTOR_STATUS_CAPACITY) is left out, a page that is none (COMPACTOR_STATUS_PAGE) too.
 *
 * compactor_paged_select, of a cache of either kind (it reads no rows): a unit with t tokens, the one that the step is going to append
 * included, has P = ceil(t / page_tokens) pages.  If P <= pages all are taken.  Otherwise the first `first_pages`, the last `last_pages`
 * and of the others those of the greatest
 *   score = max over the KV head's query heads of sum_c q_c (q_c > 0 ? greatest_c : least_c)
 * (summed in 64 bits, rounded to fp32; of equal scores the lower page; not-a-number ranks above +inf, a page that is none below all), `pages` in all.
 *   q              rows [batch][heads * q_per_kv] of the layer's queries, as the attention gets them.
 *   k_new          rows [batch][heads] of the token that the attention is going to append, or ptr NULL (nothing will be appended).  It enters the bounds
 *                  of its page (as given, in a cache of either kind), so that they need no other call while a sequence grows.  In 4 bits they
 *                  then differ from bounds made anew, which are those of the rows as they are held, by up to half a step of the new row and
 *                  a rounding to bf16, and a later step may choose other pages by the ones than by the others (compactor_paged4_bounds after a step, `first`
 *                  = the lengths before it, makes them those of the held rows again).
 *   lengths        device int32 [units of the cache], without the new token.
 *   table_out      device int32 [heads * batch][pages]: the pages taken, in the unit's order, and -1 behind them; no part of the cache's table.
 *   lengths_out    device int32 [heads * batch], no part of `lengths`: the unit's length over that table, again without the new token; a
 *                  negative length stays, a unit beyond max_length or its pages (COMPACTOR_STATUS_CAPACITY) gets -1.
 *   options (HOST): 1 <= q_per_kv <= 64; max_length, the most tokens a unit may have, the new one included; first_pages >= 0, last_pages
 *                  >= 1 (a unit's last page is filled only in part, and takes the new token), first_pages + last_pages <= pages.
 * Pages that are taken and are none are reported (COMPACTOR_STATUS_PAGE) and left to the attention.
 * At most 49152 pages per unit, and no more in `pages` than a table may have (COMPACTOR_E_TOO_LARGE).  Workspace: compactor_paged_select_workspace_bytes(), 256-byte aligned, contents
 * not preserved; 0 = bad arguments.  `bounds` is written (one page per unit): calls that share it are ordered by the caller.
 */
typedef struct compactor_select_options {
    int32_t q_per_kv;
    int32_t max_length;
    int32_t pages;
    int32_t first_pages;
    int32_t last_pages;
} compactor_select_options;
int compactor_paged_bounds(const compactor_paged_cache* cache, int32_t first_layer, int32_t layers, const int32_t* first,
                           const int32_t* lengths, int32_t max_length, void* bounds, int32_t* status, void* stream);
int compactor_paged4_bounds(const compactor_paged_cache* cache, int32_t first_layer, int32_t layers, const int32_t* first,
                            const int32_t* lengths, int32_t max_length, void* bounds, int32_t* status, void* stream);
size_t compactor_paged_select_workspace_bytes(const compactor_paged_cache* cache, int32_t max_length);
int compactor_paged_select(const compactor_paged_cache* cache, int32_t layer, const compactor_select_options* options,
                           compactor_rows q, compactor_rows k_new, const int32_t* lengths, void* bounds, int32_t* table_out,
                           int32_t* lengths_out, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Norms of queries and keys for each head and the rotation by position, in one pass: what makes the keys that a prefill is scored by
 * (k_plain_out), the keys it is held and attended to as (k_out) and the queries (q_out), and the rows of a decoding step.
 *   y = x * weight / sqrt(mean(x^2) + eps) in fp32, or y = x where the weight is NULL;
 *   angle_i = position * inv_freq[i] (taken in 64 bits), i < rotary / 2; with (j, k) = (i, i + rotary / 2), or (2 i, 2 i + 1) when interleaved,
 *   (y_j, y_k) becomes (y_j cos - y_k sin, y_k cos + y_j sin); channels from `rotary` on stay.  Each output is rounded once.
 *   q, k           rows [tokens][q_heads] and [tokens][k_heads] (stride_seq: between tokens); either number of heads may be 0.
 *   q_weight, k_weight  device bf16 [d], 16-byte aligned, or NULL: no norm.
 *   positions      device int32 [tokens];  inv_freq  device fp32 [rotary / 2]; not used (may be NULL) when rotary = 0.
 *   q_out, k_out   rows as above.  They may be the rows of q and k themselves; other than that outputs overlap neither inputs nor each other.
 *   k_plain_out    rows of y of the keys, or ptr NULL.
 *   options (HOST): d = 128, rotary a multiple of 16 up to d, eps >= 0, interleaved 0 or 1.
 * No workspace.
 */
typedef struct compactor_norm_rope_options {
    int32_t q_heads;
    int32_t k_heads;
    int32_t d;
    int32_t rotary;
    int32_t interleaved;
    float   eps;
} compactor_norm_rope_options;
int compactor_norm_rope(const compactor_norm_rope_options* options, int64_t tokens, compactor_rows q, compactor_rows k,
                        const void* q_weight, const void* k_weight, const int32_t* positions, const float* inv_freq,
                        compactor_rows q_out, compactor_rows k_out, compactor_rows k_plain_out, void* stream);

/*
 * compactor_score for callers that cannot allocate device memory (the paper has no counterpart;
 * this is a deployment convenience).  Same inputs, outputs and results as compactor_score, but
 * no workspace argument: the scratch is a fixed array of compactor_builtin_scratch_bytes()
 * (32 MiB) inside the library, resident on every device the process uses from the first use of
 * the library on that device until the process exits.  The call allocates and frees nothing.
 *   - Size limit: the scratch must hold 16*(batch+1) bytes of tables, about 72 KiB per unit
 *     (at m = 48) and 128 KiB per Gram block (blocks are lengthened up to 65536 tokens to make it
 *     fit, i.e. down to 2 bytes per token per (layer, head)).  A larger problem is refused with
 *     COMPACTOR_E_TOO_LARGE before anything is enqueued; split it by layers or use
 *     compactor_score.
 *   - The first call on each device looks up the array's device address; make that first call
 *     outside any stream capture.
 *   - All calls share the one array and it keeps whatever the previous call left there (nothing
 *     in it needs clearing: every call rewrites what it reads).  Two calls whose device work
 *     can overlap - different streams, or different host threads on the same device - race on
 *     it; order them on one stream or with events.
 */
size_t compactor_builtin_scratch_bytes(void);
int compactor_score_builtin_scratch(const compactor_shape* shape, compactor_mat k_score, const float* phi,
                                    const float* attn_scores, float lambda, float* scores_out,
                                    int32_t* status, void* stream);

/*
 * Self-test of the bounded device-side waits (no counterpart in the paper).  Enqueues a one-warp
 * kernel that waits, with a limit of about a millisecond, once on a barrier that completes and
 * once on a barrier that nothing completes, through the same wait routine the streaming kernels
 * use.  status_out (device int32[1]) receives COMPACTOR_STATUS_TIMEOUT (4) when the first wait
 * succeeded and the second gave up as designed; any other value is a defect.  The context stays
 * usable: nothing traps or hangs.
 */
int compactor_wait_selftest(int32_t* status_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* COMPACTOR_H_ */
