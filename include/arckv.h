/*
 * arckv.h -- C ABI of the MI355X (gfx950) ARC-KV per-context compaction library.
 *
 * ARC-KV (arXiv 2609.36835) replaces a long key/value cache block (K, V, T rows
 * of head dimension d) of one layer-KV-head pair by t << T compact entries
 * (C_k, beta, C_v) so that softmax(q C_k^T + beta) C_v approximates full
 * attention softmax(q K^T) V and the block's attention mass (Section 3.1,
 * eq. compact_attention and eq. block_attention_mass).  Per context, four
 * stages run (Section 3.2):
 *   1. score every cached token and take the top-t tokens as anchors (Section 3.3);
 *   2. assign every key to the anchor with the most similar normalised
 *      attention-response profile and merge each group into one compact key
 *      inside the group's convex hull (Section 3.4);
 *   3. fit the mass bias beta by projected least squares (Appendix A.9, eq. mass_fit;
 *      optionally by exact non-negative least squares);
 *   4. fit the compact values C_v by ridge least squares (Appendix A.9, eq. value_lstsq).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - A call processes B independent pairs (flattened [layer][kv_head]).
 *  - All array arguments are DEVICE pointers owned by the caller, row-major and
 *    contiguous: K, V [B][T][d]; Q_ref [B][n][d] (each pair's n rows ordered
 *    [query head][position]); per-pair vectors [B][len].  Inputs are read-only.
 *    K, V, Q_ref, Y, W1 and C_k move in 16-byte vectors and must be 16-byte
 *    aligned (ARCKV_ERR_INVALID_ARG otherwise).
 *  - K, V and Q_ref share one element type (arckv_problem.dtype): float32 or
 *    bfloat16.  Only d = 128 is supported.  Outputs are float32 (indices int32).
 *  - The library never allocates device memory.  Entry points that need scratch
 *    take a caller-owned device workspace (ws, ws_bytes) of at least
 *    arckv_workspace_size() bytes, 256-byte aligned.  Its contents are
 *    undefined on entry and exit (apart from the counters arckv_assign_stats
 *    reads); it must not be shared by calls that may overlap in time.
 *  - All device work is enqueued on the caller's stream.  The host is
 *    synchronised only where the next launches depend on a device result: the
 *    fits read back the number of pairs to refactor (a failed Cholesky pivot;
 *    in the mass fit also a cut-off refinement) before each possible
 *    ridge-escalation round (not with max_escalations = 0), and the
 *    exact non-negative mass fit (bias_mode = 1) reads two integers back once
 *    per pivoting iteration, to size the next iteration's system and to stop
 *    when every pair has settled.  Results are valid once the stream reaches
 *    them.
 *  - Argument errors are returned synchronously BEFORE any HIP call, so they can
 *    be checked on a machine without a GPU.  A failed kernel launch returns
 *    ARCKV_ERR_HIP.  Numerical failures are reported asynchronously in the
 *    per-pair `info` arrays.  No C++ exception crosses this interface.
 *  - The logit scale s multiplies q.k everywhere (the paper omits 1/sqrt(d) by
 *    convention, Section 3.1); scale <= 0 selects 1/sqrt(d).
 */
#ifndef ARCKV_H
#define ARCKV_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ARCKV_OK = 0,
  ARCKV_ERR_INVALID_ARG = 1,   /* null pointer, bad size, t outside [1, T], ... */
  ARCKV_ERR_UNSUPPORTED = 2,   /* d != 128, unknown dtype, bias_mode outside {0, 1}, ... */
  ARCKV_ERR_WORKSPACE = 3,     /* ws too small or misaligned */
  ARCKV_ERR_HIP = 4            /* a HIP launch or runtime call failed */
} arckv_status;

typedef enum { ARCKV_F32 = 0, ARCKV_BF16 = 1 } arckv_dtype;

typedef struct {
  int32_t B;       /* pairs in the call, >= 1 */
  int32_t T;       /* cached tokens per pair, >= 1 */
  int32_t n;       /* reference queries per pair, >= 1 */
  int32_t d;       /* head dimension; must be 128 */
  int32_t dtype;   /* arckv_dtype of K, V, Q_ref */
  float scale;     /* logit scale s; <= 0 selects 1/sqrt(d) */
} arckv_problem;

/* The token scorer: a 2-layer MLP on concat(k_j, v_j),
 * I_j = w2 . GELU(W1 [k_j; v_j] + b1) + b2, GELU(x) = x Phi(x) (erf form).
 * The bfloat16 path evaluates erfc with the rational approximation of
 * Abramowitz & Stegun 7.1.26 (absolute error <= 1.5e-7), so each GELU is
 * within about 3.3e-7 of the exact one for |x| <= 4 (about 1e-7 relative
 * beyond); the float32 path calls erff.
 * It is query-independent, so the root-mean-square pooling of eq.
 * indexer_pooling reduces to softmax(I), and ranking by I ranks by the pooled
 * score (Section 3.3). */
typedef struct {
  int32_t hidden;     /* hidden width; must be 64 */
  int32_t w1_dtype;   /* arckv_dtype of W1 */
  const void *W1;     /* [B][hidden][2d], input order [k ; v] */
  const float *b1;    /* [B][hidden] */
  const float *w2;    /* [B][hidden] */
  const float *b2;    /* [B] */
} arckv_indexer;

/* Fit parameters (Section 3.4 and Appendix A.9).  The paper gives lambda_m;
 * the remaining values are this library's readings. */
typedef struct {
  float lambda_m;        /* key-merge coefficient in [0, 1]; default 0.25 */
  float delta_beta;      /* relative ridge of the mass fit: G + delta_beta*tr(G)/t*I; default 1e-6 */
  float delta_v;         /* relative ridge of the value fit: lambda_v = delta_v*tr(A)/t; default 1e-3 */
  float eps_w;           /* epsilon_w of eq. mass_fit; default 1e-12 */
  float b_min, b_max;    /* clip range of beta; default [-30, 30] */
  int32_t bias_mode;     /* 0 = projected least squares (eq. mass_fit, the paper's: w* = max(w~, 0));
                          * 1 = exact non-negative least squares on the same ridged system, by block
                          * principal pivoting; other values unsupported */
  int32_t max_escalations; /* ridge x10 retries (from 1e-7 when the ridge is 0) after a failed
                            * Cholesky pivot or a cut-off mass-fit refinement, 0..6; default 6 */
  int32_t refine_steps;  /* iterative-refinement steps after each mass-fit Cholesky solve, 0..4;
                          * default 2.  Each step recomputes the residual from the data
                          * (Phi_C; P_hat for the value fit), not from the float32 Gram, so
                          * the solves converge to the least-squares solutions of the exact
                          * normal equations.  With refine_steps >= 2 a correction (above 1e-10 |w|) that
                          * is not at most half the previous one is undone and ends the
                          * refinement; the pair is then refactored with the ridge raised
                          * tenfold, as after a failed pivot (a ridge small next to the
                          * float32 rounding of a rank-deficient Gram, t > n, makes the
                          * steps diverge). */
  int32_t pair_chunk;    /* pairs processed together by arckv_compact (0 = all B); sizes the workspace,
                          * results do not depend on it */
  int32_t select_chunk;  /* 0 = global top-t (default).  L > 0: when T > 10,000, anchors are the union of
                          * each L-position chunk's local top-t_c (Appendix A.3), so arckv_compact keeps
                          * arckv_select_count(T, t, L) anchors; merge and fits stay global. */
  int32_t nnls_max_iter; /* bias_mode 1: pivoting iterations (one masked Cholesky solve each), 1..256;
                          * default 32.  A pair not settled by then reports info = -2. */
  int32_t value_refine_steps; /* refinement steps after the value-fit solve, 0..4; default 1 (its ridge
                               * keeps the system well conditioned: one step reaches the float32
                               * floor of its residual) */
} arckv_fit_params;

/* Fill *p with the defaults listed above.  Returns ARCKV_ERR_INVALID_ARG on NULL. */
arckv_status arckv_default_params(arckv_fit_params *p);

/* Budget t = clip_[1,T](floor(rho*T + 1/2)), computed in double (the paper
 * rounds the budget by ceil in training, floor per head and round per chunk,
 * Section 3.5 and Appendix A.2-A.3; round-half-up is this library's reading).
 * Errors: T < 1, rho not finite or rho < 0, t == NULL. */
arckv_status arckv_budget(int64_t T, double rho, int32_t *t);

/* Bytes of workspace needed by every entry point below for this problem and
 * budget (the maximum over stages; arckv_compact with p->pair_chunk pairs in
 * flight).  p may be NULL (defaults). */
arckv_status arckv_workspace_size(const arckv_problem *prob, int32_t t,
                                  const arckv_fit_params *p, size_t *bytes);

/* Stage 1a: token scores I [B][T] (float32), Section 3.3 with the MLP scorer.
 * No workspace. */
arckv_status arckv_score(const arckv_problem *prob, const void *K, const void *V,
                         const arckv_indexer *ix, float *scores, hipStream_t stream);

/* The value-aware indexer of Appendix A.1 (eq. value_context,
 * indexer_projection, pairwise_index_score) with H_I = 8 index heads of width
 * d_I = 128 and a value head of width d_A = 128.  All matrices bfloat16,
 * row-major, per pair (B pairs in a call):
 *   L_q, L_k, L_c, L_v [B][1024][128];  U_q, U_k, U_v [B][128][128];
 *   L_x [B][8][d_x];  b_x [B][8] float32;
 *   X_ref [ceil(B / x_group)][n_pos][d_x]: the activation x_r of reference position r,
 *   shared by the query heads of a position and by the x_group consecutive
 *   pairs of one layer (its KV heads).
 * Q_ref rows are ordered [query head][position], so row i uses x_{i mod n_pos}. */
typedef struct {
  int32_t n_pos;      /* reference positions; n must be a multiple of n_pos */
  int32_t d_x;        /* activation width, >= 1 */
  int32_t x_group;    /* pairs sharing one X_ref block, >= 1 */
  float scale_a;      /* logit scale of the value head; <= 0 selects 1/sqrt(d_A) */
  const void *X_ref;
  const void *L_q, *L_k, *L_x;
  const float *b_x;
  const void *U_q, *U_k, *U_v;
  const void *L_c, *L_v;
} arckv_dsa_indexer;

/* Workspace for arckv_score_dsa with pair_chunk pairs in flight (0 = all B). */
arckv_status arckv_dsa_workspace_size(const arckv_problem *prob, int32_t pair_chunk, size_t *bytes);

/* Stage 1a with the value-aware indexer: pooled scores s_j of eq.
 * indexer_pooling, s_j = sqrt(mean_i softmax_j(I_i,:)_j^2), for every cached
 * token of every pair -> scores [B][T] float32 (rank them with arckv_select).
 * K, V, Q_ref bfloat16 only.  Intermediates (the value head's projections and
 * context, qbar, kbar) are stored in bfloat16; accumulation is float32. */
arckv_status arckv_score_dsa(const arckv_problem *prob, const void *K, const void *V,
                             const void *Q_ref, const arckv_dsa_indexer *ix, float *scores,
                             void *ws, size_t ws_bytes, hipStream_t stream);

/* Stage 1b: anchors S = TopK(scores, t) per pair (Section 3.3, eq.
 * persistent_support), written ascending to anchors [B][t].  Order: larger
 * score first, ties to the lower index, -0 equal to +0, NaN below every number.
 * Bit-exact by construction.  Needs 1 <= t <= T. */
arckv_status arckv_select(const arckv_problem *prob, const float *scores, int32_t t,
                          int32_t *anchors, void *ws, size_t ws_bytes, hipStream_t stream);

/* Per-pair budgets of eq. per_head_budget (host only, no GPU work):
 * t_out[i] = clip_[1,T](floor(a_i / sum(a) * P * t)) for P pairs with weights
 * a (host array, finite, >= 0, not all zero) and nominal per-pair budget t. */
arckv_status arckv_budgets(int32_t P, const double *a, int32_t t, int64_t T, int32_t *t_out);

/* Realised anchor count of chunked selection (Appendix A.3; host only):
 * sum over chunks c of length T_c of clip_[1,T_c](round(t T_c / T)) (rounded
 * half up) when chunk_len > 0 and T > 10,000, otherwise t. */
arckv_status arckv_select_count(int64_t T, int32_t t, int32_t chunk_len, int32_t *t_real);

/* Stage 1b, general form: per-pair budgets and/or chunked selection.
 *   t_pair     [B] device array of per-pair budgets (e.g. from arckv_budgets),
 *              or NULL for the uniform budget t; entries are clipped to [1, T].
 *   chunk_len  0 = global top-t; L > 0 = Appendix A.3 chunking when T > 10,000.
 *   anchors    [B][t_stride] output: each row holds the pair's anchors ascending,
 *              then -1 up to t_stride.  t_stride must cover every pair's realised
 *              count (arckv_select_count of its budget); rows are truncated, never
 *              overrun, if it does not.  With t_pair NULL a short t_stride is
 *              rejected (ARCKV_ERR_INVALID_ARG).
 * The order of S and the tie rules are those of arckv_select. */
arckv_status arckv_select_ex(const arckv_problem *prob, const float *scores, int32_t t,
                             const int32_t *t_pair, int32_t chunk_len, int32_t t_stride,
                             int32_t *anchors, hipStream_t stream);

/* Full-cache row statistics (Appendix A.9): with l_ij = s q_i.k_j,
 *   z [B][n]     z_i = max_j l_ij over the whole cache,
 *   m [B][n]     m_i = sum_j exp(l_ij - z_i)            (the mass targets Phi_K 1),
 *   Y [B][n][d]  Y_i = sum_j exp(l_ij - z_i) v_j / m_i   (full attention outputs).
 * No workspace. */
arckv_status arckv_rowstats(const arckv_problem *prob, const void *K, const void *V,
                            const void *Q_ref, float *z, float *m, float *Y, hipStream_t stream);

/* Stage 2: response-profile assignment and convex key merge (Section 3.4,
 * eq. response_profile, anchor_assignment, mass_centroid, key_merge).
 *   z        [B][n] row maxima from arckv_rowstats; max_i z_i is z_merge.
 *   anchors  [B][t] ascending anchor positions.
 *   C_k      [B][t][d] output; row r is the compact key of anchors[r], a convex
 *            combination of its group's keys with weights >= 0 summing to 1.
 *   assign   [B][T] output (may be NULL): the group r of every position;
 *            anchors are assigned to themselves, ties go to the lowest r.
 *   phi      [B][T] output (may be NULL): query-averaged mass exp(l - z_merge). */
arckv_status arckv_merge(const arckv_problem *prob, const void *K, const void *Q_ref,
                         const float *z, const int32_t *anchors, int32_t t, float lambda_m,
                         float *C_k, int32_t *assign, float *phi,
                         void *ws, size_t ws_bytes, hipStream_t stream);

/* Stage 3: mass bias (Appendix A.9, eq. mass_fit).  With
 * Phi_C = exp(s Q C_k^T - z 1^T): w~ solves (G + delta_beta tr(G)/t I) w = h,
 * G = Phi_C^T Phi_C, h = Phi_C^T m, by Cholesky (float32) plus refinement;
 * beta = clip(log max(max(w~, 0), eps_w), b_min, b_max).
 * With p->bias_mode = 1, w* instead minimises w^T (G + lam I) w / 2 - h^T w over
 * w >= 0 (lam the ridge settled by the factorisation above), found by block
 * principal pivoting: each iteration refactors the system restricted to the
 * current free set and solves it with refinement against the data.
 *   K, V  [B][T][d] the cache; read only when z or m is NULL.
 *   z, m  [B][n] row maxima and masses from arckv_rowstats, or NULL: both are then
 *         recomputed from K, V and Q_ref (arckv_rowstats) into the workspace.
 *   beta  [B][t] output.
 *   info  [B] output: 0 = ok; k > 0 = Cholesky pivot k failed after all ridge
 *         escalations; -1 = a non-finite value in z, m or C_k (the pair is not
 *         fitted); -2 = bias_mode 1 did not settle within nnls_max_iter
 *         iterations.  beta is NaN whenever info != 0.
 *   delta_used [B] output (may be NULL): the relative ridge actually used.
 * Ridge escalation: a pair whose factorisation fails, or whose refinement is
 * cut off (refine_steps), is refactored with the ridge raised tenfold (from
 * 1e-7 when delta_beta = 0), at most p->max_escalations times in all.  Before
 * each such round the call reads back one integer (the number of pairs to
 * refactor) and synchronises the stream; with max_escalations = 0 it never
 * synchronises. */
arckv_status arckv_fit_bias(const arckv_problem *prob, const void *K, const void *V, const void *Q_ref,
                            const float *C_k, int32_t t, const float *z, const float *m,
                            const arckv_fit_params *p, float *beta, int32_t *info, float *delta_used,
                            void *ws, size_t ws_bytes, hipStream_t stream);

/* Stage 4: compact values (Appendix A.9, eq. value_lstsq).  With
 * P_hat = softmax(s Q C_k^T + 1 beta^T): C_v solves
 * (A + delta_v tr(A)/t I) C_v = P_hat^T Y, A = P_hat^T P_hat.
 *   K, V  [B][T][d] the cache; read only when Y is NULL.
 *   Y     [B][n][d] full-attention outputs from arckv_rowstats, or NULL:
 *         recomputed from K, V and Q_ref into the workspace.
 *   C_v   [B][t][d] output.
 *   info  [B] output: 0 = ok; k > 0 = Cholesky pivot k failed after all ridge
 *         escalations; -1 = a non-finite value in Y, C_k or beta (a failed mass
 *         fit leaves beta NaN, so its pair reports -1 here).  C_v is NaN
 *         whenever info != 0.
 *   delta_used and the escalation rounds as for arckv_fit_bias. */
arckv_status arckv_fit_values(const arckv_problem *prob, const void *K, const void *V, const void *Q_ref,
                              const float *C_k, const float *beta, int32_t t, const float *Y,
                              const arckv_fit_params *p, float *C_v, int32_t *info, float *delta_used,
                              void *ws, size_t ws_bytes, hipStream_t stream);

/* The whole per-context path for B pairs: score, select, row statistics,
 * merge, mass fit, value fit.  t = arckv_budget(T, rho) (or, with
 * p->select_chunk, arckv_select_count of it) is written to *t_out (host
 * pointer) before any device work.  Outputs: anchors [B][t], C_k [B][t][d],
 * beta [B][t], C_v [B][t][d], info [B][2] (mass-fit, value-fit status as above;
 * a non-finite value anywhere in K, V or Q_ref reaches the row statistics and
 * the pair reports -1 in both).
 * Pairs are processed p->pair_chunk at a time (0 = all at once). */
arckv_status arckv_compact(const arckv_problem *prob, const void *K, const void *V,
                           const void *Q_ref, const arckv_indexer *ix, double rho,
                           const arckv_fit_params *p, int32_t *t_out, int32_t *anchors,
                           float *C_k, float *beta, float *C_v, int32_t *info,
                           void *ws, size_t ws_bytes, hipStream_t stream);

/* Decode-time attention over a compacted block followed by an optional
 * uncompressed block (eq. compact_attention; the joint form of Appendix A.7,
 * eq. concatenated_attention_preservation, which appends zero bias for the
 * uncompressed rows).  For each pair p (one sequence and KV head) and each of
 * its G query rows q (the query heads sharing that KV head):
 *   out[p][q] = softmax([s q C_k^T + beta, s q K_f^T]) [C_v; V_f]
 * with s = scale (<= 0 selects 1/sqrt(d)).  The consumer of arckv_compact's
 * output; with beta = NULL, C_k = K, C_v = V and F = 0 it is full-cache
 * attention.
 *   Q        [P][G][d] bfloat16, d = 128; G in {1, 2, 4, 8}.
 *   C_k, C_v [P][t][d] bfloat16 (may be NULL when t = 0).
 *   beta     [P][t] float32, or NULL for zero bias.
 *   K_f, V_f [P][F][d] bfloat16 (may be NULL when F = 0).
 *   out      [P][G][d] float32.
 * Requires t, F >= 0 and t + F >= 1; all arrays 16-byte aligned.  Workspace:
 * arckv_attend_workspace_size(P, G, t, F) bytes (per-chunk partial results).
 * Reads every key and value row once. */
arckv_status arckv_attend_workspace_size(int32_t P, int32_t G, int32_t t, int32_t F, size_t *bytes);
arckv_status arckv_attend(int32_t P, int32_t G, int32_t t, int32_t F, float scale, const void *Q,
                          const void *C_k, const float *beta, const void *C_v, const void *K_f,
                          const void *V_f, float *out, void *ws, size_t ws_bytes, hipStream_t stream);

/* arckv_attend for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation): the
 * same arguments and result, no workspace.  The split-key partials go to a
 * static device array of 64 MiB that the library holds on each GPU it runs
 * on until the process ends; the call itself allocates nothing.  Returns
 * ARCKV_ERR_WORKSPACE when arckv_attend_workspace_size(P, G, t, F) exceeds
 * 64 MiB (for instance P = 512, G = 4 allows t + F up to 16,128; use
 * arckv_attend with a workspace beyond that), ARCKV_ERR_HIP if the array's
 * device address cannot be obtained.  Every call on one GPU shares that GPU's
 * array, so calls that may overlap in time on one GPU (different streams or
 * host threads) race; calls ordered on one stream do not.  Nothing in the
 * array needs to start at zero. */
arckv_status arckv_attend_noalloc(int32_t P, int32_t G, int32_t t, int32_t F, float scale, const void *Q,
                                  const void *C_k, const float *beta, const void *C_v, const void *K_f,
                                  const void *V_f, float *out, hipStream_t stream);

/* arckv_compact with the scoring stage replaced by caller-supplied scores
 * [B][T] float32 (for instance from arckv_score_dsa): select, row statistics,
 * merge and both fits exactly as arckv_compact. */
arckv_status arckv_compact_scored(const arckv_problem *prob, const void *K, const void *V,
                                  const void *Q_ref, const float *scores, double rho,
                                  const arckv_fit_params *p, int32_t *t_out, int32_t *anchors,
                                  float *C_k, float *beta, float *C_v, int32_t *info,
                                  void *ws, size_t ws_bytes, hipStream_t stream);

/* Statistics of the key-to-anchor decision of the most recent arckv_merge,
 * arckv_compact or arckv_compact_scored call that used this workspace with
 * this problem and anchor count t (Section 3.4, eq. anchor_assignment).  The
 * argmax is decided in up to three passes: an fp16 (bf16 inputs) or fp32
 * contraction whose per-similarity rounding error is bounded, so every key
 * with a single anchor inside the bound is decided there; a refine pass over
 * the flagged keys' candidate anchors with logits accurate to about 1e-6; and
 * a float64 pass for the keys the refine pass cannot separate (equal float64
 * similarities go to the lowest r).  Copies [B][8] int32 to the device array
 * stats, per pair: [0] keys flagged after the first pass, [1] keys decided in
 * float64, [2] candidate anchors of the flagged keys (a whole anchor tile
 * counts its 256 (bf16) or 128 (float32) anchors), [3] keys left undecided
 * (no finite similarity reaches the first pass's bound, which takes a
 * non-finite input; such a key keeps the first pass's best), [4] and [5] the
 * undecided ones of the first and of the refine pass ([5] stays 0: the refine
 * pass sends every key's survivors, however many, to the float64 pass, and a
 * key whose candidates overflow the candidate pool goes there with all t
 * anchors), [6] keys sent to the refine pass, [7]
 * flagged keys with a whole anchor tile among their candidates.  Those
 * counters are the only workspace contents that outlive a call. */
arckv_status arckv_assign_stats(const arckv_problem *prob, int32_t t, const void *ws, size_t ws_bytes,
                                int32_t *stats, hipStream_t stream);

/* ------------------------------------------------------------------ 8-bit cache
 * Keys and values of P pairs (one sequence and KV head each) in 8 bits, with a
 * scale for each block of 64 consecutive tokens: a quarter of a float32 cache,
 * half of a bfloat16 one.  For block b, rows 64 b .. 64 b + 63 of a pair, keys
 * and values apart, with A the largest magnitude among the rows it holds:
 *   scale = 2^e, e the smallest whole number >= -100 with A <= M 2^e,
 *           M = 448 (ARCKV_E4M3) or 127 (ARCKV_INT8);
 *   code  = x / scale rounded to the nearest code, ties to even;
 *   the stored value is scale * code.
 * Scales are powers of two, so the codes do not depend on how they are computed,
 * a stored value is exact in bfloat16, and storing it again changes nothing.
 * An error is at most half a step where a block is written once: 2^-4 of the value's
 * magnitude (2^-10 scale for the smallest) in e4m3, scale / 2 in int8, where a scale
 * is below A / 63.5 (or 2^-100).  A row kept in a block whose scale grows is rounded again
 * (a prompt's last block, every block of single tokens).  The halves add up, but to
 * less than a step of the largest scale that the block has had since: scale in int8;
 * 2^-9 scale in e4m3, where values of 2^-6 scale and more keep their 2^-4.  Keys
 * with outlier channels lose less in e4m3, values of one magnitude less in int8.
 * A block that holds a non-finite number has a NaN scale and reads as NaN, and so do
 * rows kept in it when later ones are replaced: writing the block from its first row
 * on makes it whole again.
 * (The largest magnitudes, above 2^127, may round to infinity.)
 *
 * The caller owns every array and the number of rows that each pair holds
 * ("length", an int32 device array where it differs between pairs).  Rows behind
 * a pair's length are never read; they need not be initialised, nor do the
 * scales and bounds of blocks that hold none. */
typedef enum { ARCKV_E4M3 = 0, ARCKV_INT8 = 1 } arckv_qformat;

typedef struct {
  int32_t P;          /* pairs, 1..2^20 */
  int32_t rows;       /* rows that a pair has room for, 1..2^26; any number, the last block may be short */
  int32_t d;          /* head dimension; must be 128 */
  int32_t format;     /* arckv_qformat */
  void *K, *V;        /* codes [P][rows][128], one byte each, 16-byte aligned */
  float *K_scale;     /* [P][ceil(rows / 64)] */
  float *V_scale;
  void *K_bounds;     /* [P][ceil(rows / 64)][2][128]: each key channel's smallest and largest code in the
                       * block, 16-byte aligned; NULL where no arckv_select_blocks call will read them */
} arckv_qcache;

/* Write n rows of keys and values, [P][n][128] float32 or bfloat16 (dtype; 16-byte
 * aligned), into the cache:
 *   start [P] device array: the first row to write, or NULL for 0 (clipped to [0, rows]);
 *   count [P] device array: how many of the pair's n source rows to write, or NULL
 *         for all (clipped to [0, n]); rows that would lie past the cache's end are dropped.
 * The pair then holds start + count rows: rows before start are kept, rows from
 * start on are replaced, what was behind them no longer counts.  A block that is
 * written from its middle on is scaled anew for all it holds: the rows kept in
 * it are rounded again if its scale grows (nothing moves if it does not).
 * Codes behind the written rows stay as they were, as do blocks without new rows.
 * Needs 1 <= n <= rows.  No workspace, no synchronisation. */
arckv_status arckv_qcache_write(const arckv_qcache *c, int32_t n, int32_t dtype, const void *K, const void *V,
                                const int32_t *start, const int32_t *count, hipStream_t stream);

/* Read rows first .. first + n - 1 of every pair, as float32 or bfloat16 (dtype;
 * both exact), into K and V [P][n][128], 16-byte aligned.  Rows at or past the
 * pair's length ([P] device array, or NULL: all rows are held) come back as
 * zeros.  Needs first >= 0, n >= 1, first + n <= rows. */
arckv_status arckv_qcache_read(const arckv_qcache *c, int32_t first, int32_t n, int32_t dtype, const int32_t *length,
                               void *K, void *V, hipStream_t stream);

/* The k blocks of each pair that its G query rows can give the largest logits to.
 * With lo, hi the block's bounds times its scale, the block's score is
 *   max_g [ s sum_d max(q_gd lo_d, q_gd hi_d) ] + max_j beta_j  (j over the block's rows),
 * which no logit of a stored key of the block exceeds by more than the roundings
 * below; -inf for a block that holds no row, or none with a bias above -inf; NaN for
 * one with a NaN scale or a query with a non-finite channel.  The sum over channels
 * is formed in float64 from exact parts, in one order whatever the call, and the
 * score rounded to float32 at the end: to the nearest, by up to 2^-24 of it either way.
 * Query channels of at least 2^-24 of the row's largest magnitude A enter whole; of
 * smaller ones what lies below 2^-31 A may be cut off, which takes at most
 * 2^-24 s A max_d(|lo_d|, |hi_d|) from a score.
 *   Q      [P][G][128] bfloat16, 16-byte aligned, G in 1..16;
 *   beta   [P][rows] float32, or NULL;
 *   length [P] device array of rows held (clipped to [0, rows]), or NULL: all;
 *   scores [P][ceil(rows / 64)] float32 output;
 *   blocks [P][k] int32 output: the chosen blocks, ascending, in arckv_select's
 *          order of scores (ties to the lower block), 1 <= k <= ceil(rows / 64).
 * Reads scales and bounds, not the codes (c->K, V and V_scale may be NULL).  A
 * pair with fewer than k blocks in use gets unused ones too, which
 * arckv_attend_qcache passes over. */
arckv_status arckv_select_blocks(const arckv_qcache *c, int32_t G, float scale, const void *Q, const float *beta,
                                 const int32_t *length, int32_t k, float *scores, int32_t *blocks,
                                 hipStream_t stream);

/* Decode attention over the 8-bit cache, or over listed blocks of it only,
 * followed by an optional uncompressed block: for each pair and each of its G
 * query rows,
 *   out = softmax([s q K^T + beta, s q K_f^T]) [V; V_f]
 * with K, V the stored values.  arckv_attend's counterpart; over
 * (C_k, beta, C_v) written by arckv_qcache_write it is the consumer of a
 * compaction in 8 bits.
 *   Q        [P][G][128] bfloat16, G in 1..16.
 *   beta     [P][rows] float32, or NULL for zero bias.  A row with beta = -inf is
 *            left out, whatever its key and value hold.
 *   length   [P] device array of rows held (clipped to [0, rows]), or NULL: all.
 *   blocks   [P][nsel] device array of blocks to attend to, or NULL with nsel = 0
 *            for all.  Entries outside [0, ceil(rows / 64)) are passed over (a
 *            list may be padded with -1); a block that is listed twice counts twice.
 *   K_f, V_f [P][F][128] bfloat16 (may be NULL when F = 0).
 *   length_f [P] device array of rows held in K_f, V_f (clipped to [0, F]), or NULL: F.
 *   out      [P][G][128] float32; zeros for a pair without any row to attend to.
 * All tensors 16-byte aligned (per-pair int32 and float32 arrays by element).
 * Workspace: arckv_attend_qcache_workspace_size bytes; 0 where a pair's rows are one
 * workgroup's work, ws may then be NULL.  Reads every code once. */
arckv_status arckv_attend_qcache_workspace_size(int32_t P, int32_t rows, int32_t G, int32_t nsel, int32_t F,
                                                size_t *bytes);
arckv_status arckv_attend_qcache(const arckv_qcache *c, int32_t G, int32_t nsel, int32_t F, float scale, const void *Q,
                                 const float *beta, const int32_t *length, const int32_t *blocks, const void *K_f,
                                 const void *V_f, const int32_t *length_f, float *out, void *ws, size_t ws_bytes,
                                 hipStream_t stream);

/* ------------------------------------------------------------------ 4-bit cache
 * Keys and values of P pairs in 4 bits (two codes, nibbles, to a byte: "ncache"), every row on its own: 128 codes of a row
 * in 64 bytes and a scale for each group of 32 consecutive channels in a byte, 68
 * bytes against the 256 of bfloat16 (136 a token with its value).
 *   code   e2m1: sign, two exponent bits, one mantissa bit; the magnitudes 0, 0.5,
 *          1, 1.5, 2, 3, 4, 6 in the order of the codes 0..7, negatives 8..15.
 *          Channel 2 j is the low half of byte j of the row, channel 2 j + 1 the high.
 *   scale  2^e, e the smallest whole number in [-100, 125] with A <= 6 * 2^e (125
 *          where there is none), A the largest magnitude of the group; held as e + 127.
 *   code = x / scale rounded to the nearest code, ties to even (an even code); the
 *   stored value is scale * code.  A zero keeps its sign.
 * Scales are powers of two, so the codes do not depend on how they are computed, a
 * stored value is exact in bfloat16, and storing it again gives the same values.  An
 * error is at most half a step: a quarter of the value's magnitude from one scale
 * on, a quarter of the scale below it (magnitudes above 7 * 2^125 become 6 * 2^125).
 * A group with a non-finite number has the scale byte 255 and codes of 0, and reads
 * as NaN.  Rows do not depend on each other: a write changes the rows it
 * writes and nothing else.
 *
 * The caller owns the arrays and the number of rows that each pair holds.  Rows
 * behind a pair's length are never read and need not be initialised. */
typedef struct {
  int32_t P;              /* pairs, 1..2^20 */
  int32_t rows;           /* rows that a pair has room for, 1..2^26 */
  int32_t d;              /* head dimension; must be 128 */
  void *K, *V;            /* codes [P][rows][64] bytes, 16-byte aligned */
  void *K_scale, *V_scale;  /* [P][rows][4] bytes, 4-byte aligned */
} arckv_ncache;

/* Write n rows of keys and values, [P][n][128] float32 or bfloat16 (dtype; 16-byte
 * aligned), into the cache, as arckv_qcache_write does:
 *   start [P] device array: the first row to write, or NULL for 0 (clipped to [0, rows]);
 *   count [P] device array: how many of the pair's n source rows to write, or NULL
 *         for all (clipped to [0, n]); rows that would lie past the cache's end are dropped.
 * Needs 1 <= n <= rows.  No workspace, no synchronisation. */
arckv_status arckv_ncache_write(const arckv_ncache *c, int32_t n, int32_t dtype, const void *K, const void *V,
                                const int32_t *start, const int32_t *count, hipStream_t stream);

/* Read rows first .. first + n - 1 of every pair, as float32 or bfloat16 (dtype;
 * both exact), into K and V [P][n][128], 16-byte aligned.  Rows at or past the
 * pair's length ([P] device array, or NULL: all rows are held) come back as
 * zeros.  Needs first >= 0, n >= 1, first + n <= rows. */
arckv_status arckv_ncache_read(const arckv_ncache *c, int32_t first, int32_t n, int32_t dtype, const int32_t *length,
                               void *K, void *V, hipStream_t stream);

/* Decode attention over the 4-bit cache followed by an optional uncompressed block:
 * for each pair and each of its G query rows,
 *   out = softmax([s q K^T + beta, s q K_f^T]) [V; V_f]
 * with K, V the stored values: arckv_attend_qcache's counterpart without lists of
 * blocks; over (C_k, beta, C_v) written by arckv_ncache_write it is the consumer of
 * a compaction in 4 bits.
 *   Q        [P][G][128] bfloat16, G in 1..16.
 *   beta     [P][rows] float32, or NULL for zero bias.  A row with beta = -inf is
 *            left out, whatever its key and value hold.
 *   length   [P] device array of rows held (clipped to [0, rows]), or NULL: all.
 *   K_f, V_f [P][F][128] bfloat16 (may be NULL when F = 0).
 *   length_f [P] device array of rows held in K_f, V_f (clipped to [0, F]), or NULL: F.
 *   out      [P][G][128] float32; zeros for a pair without any row to attend to, NaN
 *            for a query row with a non-finite channel where there is one.
 * A mean of finite values is finite, however large they are and however many; for it sums
 * are held in units in which up to (rows + F)^2 2^-114 of a result may be lost, whatever
 * its size.  A logit of -inf in float32 counts as a row left out.
 * Tensors 16-byte aligned (per-pair int32 and float32 arrays by element).  Workspace:
 * arckv_attend_ncache_workspace_size bytes; 0 where a pair's rows are one
 * workgroup's work, ws may then be NULL.  Reads every code once. */
arckv_status arckv_attend_ncache_workspace_size(int32_t P, int32_t rows, int32_t G, int32_t F, size_t *bytes);
arckv_status arckv_attend_ncache(const arckv_ncache *c, int32_t G, int32_t F, float scale, const void *Q,
                                 const float *beta, const int32_t *length, const void *K_f, const void *V_f,
                                 const int32_t *length_f, float *out, void *ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------ rotary positions
 * Turn rows of queries and keys by their positions.  With h = d_rot / 2, pair i < h of a row
 * is its channels (i, i + h) (ARCKV_ROTARY_HALVES) or (2 i, 2 i + 1)
 * (ARCKV_ROTARY_NEIGHBOURS), and for a token at position p, a = p * freq[i]:
 *   (u, v) -> factor (u cos a - v sin a, u sin a + v cos a);
 * channels from d_rot on are copied.  With transpose the turn is by -a: the transposed
 * of that map, which takes the gradient of y to that of x (and, with factor 1, undoes it).
 * Turning by a difference of positions moves keys that have been turned already.
 * The angle is formed in float64 and reduced to one turn there, so that far positions
 * keep their precision; its sine and cosine and the products are float32, and a
 * bfloat16 result is rounded once. */
typedef enum { ARCKV_ROTARY_HALVES = 0, ARCKV_ROTARY_NEIGHBOURS = 1 } arckv_rotary_layout;

typedef struct {
  int32_t N;          /* tokens, 1..2^26 */
  int32_t d;          /* head dimension; must be 128 */
  int32_t d_rot;      /* leading channels that are turned, even, 2..128 */
  int32_t layout;     /* arckv_rotary_layout */
  int32_t dtype;      /* arckv_dtype of x and y */
  int32_t transpose;  /* 0 or 1 */
  float factor;       /* finite; multiplies the turned channels */
} arckv_rotary_params;

/* Rows of one tensor: element (n, h, c) at x[n * x_token + h * x_head + c].  Strides in
 * elements, >= 0, multiples of 16 bytes; x may repeat rows (stride 0), those of y must
 * not overlap: its larger stride covers all that its smaller one spans.  y may be x with
 * the same strides; it must share no row with x otherwise, nor with rows of a call's
 * other tensor. */
typedef struct {
  int32_t heads;      /* 1..2^20 */
  const void *x;
  int64_t x_token, x_head;
  void *y;
  int64_t y_token, y_head;
} arckv_rotary_rows;

/*   positions [N] int32 device array, any sign, or NULL: token n is at position n;
 *   freq      [d_rot / 2] float64 device array, radians per position;
 *   a, b      rows that share the positions (a layer's queries and keys); b may be NULL.
 * Tensors 16-byte aligned, at most 2^30 rows in all.  No workspace, no synchronisation. */
arckv_status arckv_rotary(const arckv_rotary_params *p, const int32_t *positions, const double *freq,
                          const arckv_rotary_rows *a, const arckv_rotary_rows *b, hipStream_t stream);

/* Frequencies of the pairs (host only, no GPU work), with f_i = base^(-2 i / d_rot) and the
 * context stretched to s = stretch times the `length` positions of training:
 *   ARCKV_STRETCH_NONE    f_i
 *   ARCKV_STRETCH_LINEAR  f_i / s (position interpolation)
 *   ARCKV_STRETCH_BASE    f_i of the base  base * s^(d_rot / (d_rot - 2))  (d_rot > 2)
 *   ARCKV_STRETCH_TURNS   g_i f_i + (1 - g_i) f_i / s by the turns r_i = length f_i / (2 pi) that a pair makes in
 *                         training, g_i = clip_[0,1]((r_i - few) / (many - few))
 *   ARCKV_STRETCH_INDEX   the same with g_i falling along i instead, from 1 at floor(c(many)) to 0 at ceil(c(few)),
 *                         c(r) = d_rot log(length / (2 pi r)) / (2 log base), both clipped to [0, d_rot - 1]
 *                         (their difference taken as 0.001 where they meet)
 * freq: host array [d_rot / 2] output.  Needs a finite base > 1, and where they are used stretch >= 1,
 * length > 0 and 0 < few < many, all finite. */
typedef enum {
  ARCKV_STRETCH_NONE = 0, ARCKV_STRETCH_LINEAR = 1, ARCKV_STRETCH_BASE = 2, ARCKV_STRETCH_TURNS = 3,
  ARCKV_STRETCH_INDEX = 4
} arckv_stretch;

arckv_status arckv_rotary_frequencies(int32_t d_rot, double base, int32_t mode, double stretch, double length,
                                      double few, double many, double *freq);

/* Human-readable name of a status code (static string). */
const char *arckv_status_string(arckv_status s);

/* Instrumentation.  When enabled (non-zero), entry points record HIP events
 * around each internal kernel stage on the call's stream; arckv_stage_times
 * then synchronises those events and returns per-stage milliseconds of the
 * most recent call, accumulated over calls since the last reset.
 *   names   receives up to max_stages static stage names (may be NULL),
 *   ms      receives the accumulated milliseconds,
 *   counts  receives how many launches were timed per stage (may be NULL).
 * Returns the number of stages via *n_stages.  Not thread-safe. */
arckv_status arckv_set_timing(int32_t enable);
arckv_status arckv_stage_times(int32_t max_stages, const char **names, double *ms,
                               int32_t *counts, int32_t *n_stages);
arckv_status arckv_reset_timing(void);

#ifdef __cplusplus
}
#endif
#endif /* ARCKV_H */
