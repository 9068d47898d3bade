/*
 * osscar.h -- C interface of the MI355X (gfx950) per-layer structured-pruning solver of OSSCAR
 * (arxiv 2403.12983).
 *
 * Problem (Section 3, eq. (MIQP); Section 4.1, eq. (struc)): the rows of the dense weight matrix
 * W (d1 x m) are split into p contiguous groups of q rows (d1 = p*q: FFN neurons q = 1, conv input
 * channels q = k_H*k_W, attention heads q = D_head).  Keep k groups K, zero the other rows and refit
 * the kept rows so that
 *        obj(What) = || X W - X What ||_F^2 + lambda || W - What ||_F^2
 * is as small as the local search of Section 4.2 can make it.  With H = X^T X + lambda I, G = H W this
 * is c0 + 2 L(What), L the quadratic of eq. (MIQP), c0 = Tr(W^T H W).
 *
 * Naming: this interface uses K for the KEPT groups (the paper's S is the pruned set, K its
 * complement), W for the given dense weights (the paper's W-hat) and What for the solved weights.
 *
 * Conventions for every call
 *   - "dev" pointers are device (HBM) addresses on the current HIP device, "host" pointers are host
 *     addresses.  All matrices are row-major; leading dimensions are in elements.
 *   - The library allocates no device memory.  The caller hands one workspace (256-byte aligned), of
 *     osscar_workspace_bytes() bytes or somewhat less, to osscar_create and owns it, X, W and What.
 *     The context keeps pointers into the workspace only; W is read only during osscar_gram.
 *   - All work is ordered on the stream given to osscar_create.  Calls that return host values
 *     synchronise that stream; osscar_gram without finalize does not (bf16 chunks on the matrix-core path; other chunks
 *     may).  The context owns one more stream (default
 *     priority) for a product of the search that overlaps with others; it forks from and joins the caller's stream
 *     through events inside a call, so the caller sees the ordering of a single stream.
 *   - Every call returns an osscar_status.  No exception crosses this boundary and nothing aborts.
 *     After a failure other than OSSCAR_EINVAL the context refuses further compute calls
 *     (OSSCAR_ESTATE) until it is destroyed and re-created.  osscar_last_error() describes the failure.
 *   - Groups are equal-sized and contiguous (the three cases of Section 3; Prop. 4.2 assumes equal size).  There is no
 *     group map argument: a caller whose groups are scattered permutes the rows of W (and the columns of X) first.
 *   - Precision.  H, G and the search state are stored in float32 (products accumulated in float64 where it matters).
 *     Choices, kept sets, final weights and final objective follow a float64 evaluation of the same method for any H the
 *     inverse converges on.  Quantities tracked through many updates (the objective trace of a search) follow it to about
 *     1e-5 relative while the diagonally scaled H restricted to the kept rows has a condition number below about 1e4; above
 *     that the float32 rounding of H alone moves them by up to 6e-8 * cond, and refresh_every (a rebuild from H and G every so
 *     many swaps) bounds the drift.
 *   - Calls on one context must not overlap; contexts sharing a workspace must not be used concurrently.
 */
#ifndef OSSCAR_H
#define OSSCAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct osscar_ctx osscar_ctx; /* opaque; host memory owned by the library */

typedef enum {
  OSSCAR_OK = 0,
  OSSCAR_EINVAL = 1, /* bad argument (shape, k > p, NULL pointer, misaligned buffer, ...) */
  OSSCAR_ENOMEM = 2, /* workspace too small */
  OSSCAR_ENOTPD = 3, /* H_KK (or a q x q pivot block) is not positive definite to working precision */
  OSSCAR_EHIP = 4,   /* a HIP runtime call failed */
  OSSCAR_ESTATE = 5  /* call order violated, or the context is poisoned by an earlier failure */
} osscar_status;

typedef enum { OSSCAR_F32 = 0, OSSCAR_BF16 = 1, OSSCAR_I8 = 2 /* activations of osscar_int_product only */ } osscar_dtype;

/* Problem description (Section 3: d1 x m weights, p groups of q rows; Section 4.1: keep k = p - p'). */
typedef struct {
  int64_t d1;        /* rows of W = columns of X; must equal p*q */
  int64_t m;         /* columns of W */
  int32_t p;         /* number of groups */
  int32_t q;         /* rows per group, 1 <= q <= 64 */
  int32_t k;         /* groups to keep, 1 <= k <= p */
  int32_t max_swaps; /* upper bound on the swap budget of any osscar_local_search call (sizes the trace) */
  int32_t x_dtype;   /* osscar_dtype of X */
  int32_t w_dtype;   /* osscar_dtype of W */
  int32_t from_dense; /* nonzero: size the workspace for osscar_init_greedy too (it inverts all of H) */
  int32_t target_output; /* nonzero: size the workspace for osscar_gram_target too */
} osscar_desc;

/* Bytes of device workspace with which every phase of this description runs at its best (0 if the description is invalid).
 * Small layers use two to four times what their arrays need (288 x 64 float32: 48 MB against 14.5; 8192 x 2048: 2.06 GB
 * against 2.02): copies of the float64 accumulators and partial tiles, which let the ranges of a contraction run side by side. */
size_t osscar_workspace_bytes(const osscar_desc* desc);

/* Creates a context.  workspace_dev: device, 256-byte aligned.  With fewer than osscar_workspace_bytes(desc) bytes the context does
 * without those copies and partial tiles (the same results, sums in another order; small layers are slower); OSSCAR_ENOMEM
 * if the arrays themselves do not fit.
 * hip_stream: a hipStream_t (NULL = the default stream).  *out receives the context. */
osscar_status osscar_create(osscar_ctx** out, const osscar_desc* desc, void* workspace_dev, size_t workspace_bytes,
                            void* hip_stream);
osscar_status osscar_destroy(osscar_ctx* ctx);

/* Quadratic-form construction (Section 3, dense-layer paragraph: H = X^T X, G = X^T X W; the ridge is
 * this build's addition).  Each call adds one chunk of calibration rows: H += Xc^T Xc with
 * Xc dev, row-major n_c x d1 (leading dimension ldx >= d1), dtype desc.x_dtype.  Any number of chunks,
 * any n_c >= 0; products are accumulated in float64 across chunks.
 * finalize != 0 (after adding Xc, which may be NULL with n_c = 0): lambda = lambda_abs + lambda_rel *
 * mean(diag(X^T X)); H += lambda I (stored float32); G = H W (float32); c0 = Tr(W^T G); the group norms
 * ||W_{Q^j}||_F are recorded for osscar_init_support.  W_dev: dev, row-major d1 x m, leading dimension
 * ldw, dtype desc.w_dtype (ignored unless finalize).  A new first chunk after finalize starts a new layer. */
osscar_status osscar_gram(osscar_ctx* ctx, const void* Xc_dev, int64_t n_c, int64_t ldx, int finalize,
                          const void* W_dev, int64_t ldw, double lambda_abs, double lambda_rel);

/* Convolutional layers (Section 3, "Structured pruning in convolutional layers": W is (C_in * k_H * k_W) x C_out and
 * the rows of X are the k_H x k_W patches of the layer's input).  Same as osscar_gram, but takes the input feature map
 * itself and forms the patches on the fly, so that the caller never holds the k_H * k_W times larger patch matrix.
 * F_dev: dev, contiguous (batch, channels, h_in, w_in), dtype desc.x_dtype, zero padding `pad` on every side.  The
 * patch at output position (b, oy, ox) is the row (b * h_out + oy) * w_out + ox, and input channel c, kernel offset
 * (dy, dx) is the column (c * kh + dy) * kw + dx: the rows of W acting on channel c form the group of kh * kw rows c.
 * channels * kh * kw must equal desc.d1.  Chunks (batches of feature maps) may be mixed with osscar_gram chunks. */
osscar_status osscar_gram_conv(osscar_ctx* ctx, const void* F_dev, int32_t batch, int32_t channels, int32_t h_in, int32_t w_in,
                               int32_t kh, int32_t kw, int32_t stride, int32_t pad, int finalize, const void* W_dev,
                               int64_t ldw, double lambda_abs, double lambda_rel);

/* Sequential-pipeline variant of osscar_gram (Appendix B.1, "Pruning strategies": the layer is asked to reproduce
 * the DENSE model's output from the PRUNED model's input).  Yc_dev: dev, row-major n_c x m, leading dimension
 * ldy >= m, dtype desc.x_dtype: the dense model's output of this layer for the same calibration rows as Xc.
 * Accumulates H += Xc^T Xc and X^T Y += Xc^T Yc (float64 across chunks) and ||Y||_F^2.  finalize: lambda as in
 * osscar_gram; H += lambda I; G = X^T Y + lambda W; c0 = ||Y||_F^2 + lambda ||W||_F^2, so that
 * obj(What) = ||Y - X What||_F^2 + lambda ||W - What||_F^2 = c0 - 2 Tr(G^T What) + Tr(What^T H What) and every later
 * call works unchanged.  Needs desc.target_output != 0.  A layer takes all its chunks through this call or all
 * through osscar_gram (OSSCAR_ESTATE otherwise). */
osscar_status osscar_gram_target(osscar_ctx* ctx, const void* Xc_dev, const void* Yc_dev, int64_t n_c, int64_t ldx,
                                 int64_t ldy, int finalize, const void* W_dev, int64_t ldw, double lambda_abs,
                                 double lambda_rel);

/* Alternative to osscar_gram for callers that already hold the quadratic form: copies H (d1 x d1,
 * symmetric positive definite, ridge included) and G (d1 x m), both dev float32 row-major and dense
 * (ld = d1, m), and takes c0 and the p group norms (host float64) used by the magnitude mode. */
osscar_status osscar_set_quadratic(osscar_ctx* ctx, const float* H_dev, const float* G_dev, double c0,
                                   const double* group_norms_host);

/* Support initialisation.  OSSCAR_INIT_MAGNITUDE: keep the k groups of largest Frobenius norm
 * (Appendix B.1, "MP"; equal norms: the lower group index stays).  OSSCAR_INIT_GIVEN: keep
 * groups_host[0..k) (distinct, any order).  Then builds the state Proposition 4.1 assumes -- the
 * inverse P of H on the kept rows, the optimal kept weights B = P G_K (eq. (optf)) -- plus the
 * candidate-side quantities V = P H_{K,Kc} and R = G_Kc - V^T G_K used by the impact scores
 * (eq. (impact)), and returns obj(K) = c0 - Tr(G_K^T B) in *obj_host (may be NULL). */
enum { OSSCAR_INIT_MAGNITUDE = 0, OSSCAR_INIT_GIVEN = 1 };
osscar_status osscar_init_support(osscar_ctx* ctx, int mode, const int32_t* groups_host, double* obj_host);

/* Nested schedule of Algorithm 1 from the dense layer (S_0 empty and t_i = p_i = t_hat for every iteration:
 * Section 4.2; Appendix B.1 takes t_hat = 2 for channels and attention heads and 10 for the intermediate
 * dimension of feed-forward layers).  Starts with every group kept (P = H^-1, B = H^-1 G; obj = 0 after
 * osscar_gram, c0 - Tr(G^T B) otherwise); each
 * iteration scores every kept group by the cost of removing it (eq. (impact), closed form of
 * Proposition 4.1 Case 1) at the state the iteration starts from, removes the t_hat cheapest (lowest group
 * index on ties; the last iteration takes what is left to reach k) and updates inverse, weights and objective
 * by Case 1.  Leaves the context as osscar_init_support does, so osscar_local_search and osscar_backsolve
 * can follow.  Needs desc.from_dense != 0.  1 <= t_hat <= 64.
 * refresh_every > 0 rebuilds the state from H and G after that many removals (at iteration boundaries).
 * flags: 0, or OSSCAR_SEARCH_EAGER to update the state in place after every removal also for q = 1, or
 * OSSCAR_SEARCH_NO_LOOKAHEAD (see osscar_local_search).
 * removed_host (host, optional): p - k group ids in the order removed (within an iteration: cheapest first).
 * gaps_host (host, optional): one float per iteration, ceil((p - k) / t_hat) of them: relative gap between the
 * costliest removal chosen and the cheapest kept group left out (inf if none was left out).
 * obj_host (host, optional): the tracked objective of the resulting kept set. */
osscar_status osscar_init_greedy(osscar_ctx* ctx, int32_t t_hat, int32_t refresh_every, uint32_t flags,
                                 int32_t* removed_host, float* gaps_host, double* obj_host);

/* Local search (Section 4.2 and Algorithm 1 with t-hat = 2, p-hat = 0: one group leaves, one enters).
 * Each iteration scores every kept group by the cost of removing it and every outside group by the
 * gain of adding it (eq. (impact), via the closed forms of Proposition 4.1, Cases 1 and 2), picks the
 * cheapest removal and the largest gain (ties: lowest group index), evaluates the pair's exact effect
 * (Case 3) and applies it by low-rank up/downdates if obj drops by more than rel_tol*obj; otherwise
 * the search stops.  At most max_swaps (<= desc.max_swaps) iterations.
 * flags: OSSCAR_SEARCH_ALWAYS_ACCEPT applies every selected pair (Algorithm 1 as printed).
 * OSSCAR_SEARCH_EAGER applies every swap to the whole state at once (one pass over HBM per swap); by
 * default, layers with q = 1 keep up to 64 swaps pending as a small low-rank correction and apply them
 * together on the matrix cores -- the same swaps, with less traffic.  In that mode the products of Z with the
 * rows most likely to be swapped next are computed ahead by one matrix product per flush;
 * OSSCAR_SEARCH_NO_LOOKAHEAD turns that off (every swap then reads Z once).
 * OSSCAR_SEARCH_EXACT_IN (a stronger rule than the separable scores of eq. (impact), not in the paper): with the
 * leaving group fixed as above, the entering group is the one with the largest exact gain of the pair, i.e. every
 * candidate is scored at the state without the leaving group (Case 1 applied to the blocks its score needs); costs one
 * more pass over Z per iteration and runs on the in-place path; trace_gap[2i+1] then refers to these scores.
 * Such swaps are made many to a launch where all workgroups fit the GPU at once; OSSCAR_SEARCH_LAUNCH_PER_SWAP makes
 * every swap a launch of its own (the same swaps).  A launch whose workgroups wait for one another longer than 2 ms, because
 * other work keeps some of them from starting, is given up without effect, the launches enqueued behind it are idle, and the rest of the call
 * goes a launch per swap.  For tests: OSSCAR_SEARCH_IMPATIENT gives up the first launch of many swaps, OSSCAR_SEARCH_IMPATIENT_LATER
 * the first one that goes on behind fetched products with swaps pending, with another one enqueued behind it.
 * refresh_every > 0 recomputes V, R and B from P, H, G by GEMM after that many accepted swaps.
 * Optional host outputs of length max_swaps (entry i describes iteration i, including a final rejected
 * one): trace_out / trace_in = group leaving / entering; trace_gap[2i], trace_gap[2i+1] = relative gap
 * between best and second-best removal cost / addition gain; trace_obj[i] = obj after the iteration. */
enum { OSSCAR_SEARCH_ALWAYS_ACCEPT = 1u, OSSCAR_SEARCH_EAGER = 2u, OSSCAR_SEARCH_NO_LOOKAHEAD = 4u, OSSCAR_SEARCH_EXACT_IN = 8u,
       OSSCAR_SEARCH_LAUNCH_PER_SWAP = 16u, OSSCAR_SEARCH_IMPATIENT = 32u, OSSCAR_SEARCH_IMPATIENT_LATER = 64u };
typedef struct {
  int32_t iters;     /* iterations run (accepted swaps + at most one rejected) */
  int32_t accepted;  /* swaps applied */
  double obj_initial;
  double obj_final;  /* tracked through the updates */
} osscar_search_result;
osscar_status osscar_local_search(osscar_ctx* ctx, int32_t max_swaps, double rel_tol, uint32_t flags,
                                  int32_t refresh_every, osscar_search_result* res_host, int32_t* trace_out_host,
                                  int32_t* trace_in_host, float* trace_gap_host, double* trace_obj_host);

/* Block moves (Section 4.2 with t-hat = 2 * block, p-hat = 0: s1 = s2 = block).  Each iteration scores every group
 * at the current state (eq. (impact)), takes the `block` kept groups that are cheapest to remove and the `block`
 * outside groups with the largest gain (lowest index on ties; cut to min(block, k, p - k)), applies the whole move
 * by the low-rank updates of Proposition 4.1 and keeps it if obj dropped by more than rel_tol*obj; otherwise the
 * move is taken back and the search stops.  block = 1 is osscar_local_search's move.  1 <= block <= 64.
 * flags as for osscar_local_search.  Optional host outputs: trace_out / trace_in, max_iters * block entries each
 * (iteration i at [i*block, (i+1)*block), cheapest removal / largest gain first, -1 padding); trace_gap[2i],
 * trace_gap[2i+1] = relative gap between the last group chosen and the first left out on either side;
 * trace_obj[i] = obj after iteration i.  res->iters counts iterations, res->accepted the moves kept. */
osscar_status osscar_block_search(osscar_ctx* ctx, int32_t max_iters, int32_t block, double rel_tol, uint32_t flags,
                                  osscar_search_result* res_host, int32_t* trace_out_host, int32_t* trace_in_host,
                                  float* trace_gap_host, double* trace_obj_host);

/* Test hook: applies the swap (group g_out leaves, g_in enters) unconditionally (Case 3). */
osscar_status osscar_apply_swap(osscar_ctx* ctx, int32_t g_out, int32_t g_in);

/* Final weights (closed-form optimum for the final kept set, Appendix A.1): What_K = (H_KK)^-1 G_K, other
 * rows zero.  The maintained weights are refined by float64-residual correction steps B += P (G_K - H_KK B)
 * until the correction is below float32 resolution; if the maintained inverse P has drifted too far for
 * that, H_KK is inverted afresh.
 * What_dev: dev, row-major d1 x m, leading dimension ldw_hat, dtype out_dtype.  support_host (may be
 * NULL): the k kept groups, ascending.  *obj_host (may be NULL): c0 - Tr(G_K^T What_K). */
osscar_status osscar_backsolve(osscar_ctx* ctx, void* What_dev, int64_t ldw_hat, int32_t out_dtype,
                               int32_t* support_host, double* obj_host);

/* Inspection hook: copies an internal array to dst_dev (dev, dense row-major).  float32: H d1 x d1;
 * G d1 x m; P kr x kr; B kr x m; V kr x cr; R cr x m (kr = k*q, cr = d1 - kr; rows / columns follow the
 * kept groups, resp. the other groups, in ascending group order).  float64: REM, ADD: length p, indexed
 * by group id (+inf / -inf where not applicable).  int32: KEPT_SLOTS / CAND_SLOTS: the kept / other
 * group ids, ascending. */
enum { OSSCAR_T_H = 0, OSSCAR_T_G = 1, OSSCAR_T_P = 2, OSSCAR_T_B = 3, OSSCAR_T_V = 4, OSSCAR_T_R = 5,
       OSSCAR_T_REM = 6, OSSCAR_T_ADD = 7, OSSCAR_T_KEPT_SLOTS = 8, OSSCAR_T_CAND_SLOTS = 9 };
osscar_status osscar_get_tensor(osscar_ctx* ctx, int which, void* dst_dev, size_t dst_bytes);

/* Scalars of the last finalize: lambda, c0 (host float64). */
osscar_status osscar_get_scalars(osscar_ctx* ctx, double* lambda_host, double* c0_host);

/* Device times of the last call of each kind, in milliseconds (HIP events on the context's stream):
 * [0] the Gram accumulation of the chunk passed together with finalize, with the products of earlier calls' rows that were
 * still waiting for theirs (these alone if the finalizing call has no rows), [1] finalize, [2] init_support,
 * [3] local_search, [4] backsolve, [6] total time of the search's refreshes and flushes.  Sampled once
 * per batch of iterations: eager search [5] mean duration of one bulk update of N, [7] of one update of Z (groups of
 * more than one row: [5] of both, which share a launch);
 * delayed-update search [5] and [7] mean duration of a swap's launch (the first of a batch, also where that one fetches the
 * products of a pivot that were not computed ahead and makes no swap).
 * [8] the product G = H W inside finalize (one GEMM launch, or the three bf16 products and their repacking when W is
 * bf16).  [9] the inverse of H on the kept rows in the last state build: the blocked sweep on a float64 copy of H_KK
 * (about 2 kr^3 flops on the float64 matrix cores).  [10] zero.  [11] not a time: the largest P_ii H_ii over the kept rows
 * (the variance inflation factor 1 / (1 - R_i^2): how much of a kept row the other kept rows explain), a
 * measure of the conditioning of H_KK.  [12] the candidate-side products V, S, R of the last state build together.
 * [13] mean duration of one launch of the bf16 Gram kernel (one launch per 16384 calibration rows) in the last
 * osscar_gram call that added rows on that path before the last finalize, [14] the number of launches averaged, [15] the rows
 * of these launches (they include rows of earlier calls that were still waiting for their product).  out_host: 16 doubles. */
osscar_status osscar_get_timers(osscar_ctx* ctx, double* out_host);

/* Diagnostics of the last osscar_local_search call on the delayed-update path (all zero otherwise), 8 values:
 * [0] flushes (the pending low-rank correction applied to the stored state by matrix products), [1] how many of them the
 * kernels asked for by stopping early (a selected group was still pending, or the spare slots for products not computed
 * ahead ran out), [2] pivots whose products with Z had not been computed ahead (each costs one pass over Z), [3] iterations
 * run; [4] launches that could make several swaps, [5] whether one of them was given up; [6..7] reserved (zero).  out_host: 8 int64. */
osscar_status osscar_get_counters(osscar_ctx* ctx, int64_t* out_host);

/* Diagnostic log of the library's general matrix-product launches (all contexts of the process; not thread-safe).
 * osscar_debug_gemm_log(1) clears the log and starts recording: every launch is bracketed by two events on its stream.
 * osscar_debug_gemm_log(0) stops and clears.  osscar_debug_gemm_log_read waits for the recorded launches and writes up to
 * `capacity` rows of five float64 {M, N, K, kind, milliseconds} (kind: 1 = float32 accumulation, + 2 = float64 output,
 * + 4 = lower-triangle tiles only, + 8 = second operand transposed, 16 = int8-digit product, packing included; a Gram
 * product X^T X is a lower triangle with the second operand transposed) to out_host; returns the number of rows, -1 on a bad
 * argument.  At most 16384 launches are kept. */
osscar_status osscar_debug_gemm_log(int32_t enable);
int32_t osscar_debug_gemm_log_read(double* out_host, int32_t capacity);

/* The large products that define the state of a support (every dimension >= 1024: B = P G_K, V = P H_{K,Kc}, the Schur
 * complement S and R of Proposition 4.1's closed forms) run on the int8 matrix cores from five 7-bit digits per float32
 * operand, with exact integer sums (kind 16 in the log above), and so does the residual of the back-solve; smaller ones, and
 * the residuals that involve the inverse, on the float64-accumulating kernel.  So does X^T X of rows that the bf16 kernel does not
 * take (float32, or bf16 at other alignments) from 256 tiles of 128 x 128 and 1024 rows per call on, except for columns with
 * rare large values.  osscar_debug_int_products(0) sends all of them to the float64-accumulating kernels,
 * osscar_debug_int_products(1) restores the default.  Process-wide, for tests that hold the two
 * against each other. */
osscar_status osscar_debug_int_products(int32_t enable);

/* The inverse of H on the kept rows (P of Proposition 4.1) is computed by a blocked sweep on a float64 copy of H_KK and
 * rounded to float32 once.  osscar_debug_refined_inverse(1) switches to the other route - the sweep in float32 storage,
 * then Newton-Schulz steps P <- P + P (I - H_KK P) with a float64-accumulated residual - and (0) back.  Process-wide, for
 * tests that hold the two against each other.  Timer slot 9 is the duration of the float64 sweep (of the residual product
 * on the other route), slot 11 the largest P_ii H_ii (the residual |I - H_KK P| before the last step on the other route). */
osscar_status osscar_debug_refined_inverse(int32_t enable);

/* The library overlaps independent parts of two phases on a second stream of its own: in the inverse of H_KK the bulk of
 * each panel's update beside the next panel's small kernels, in the flush of the delayed-update search (Proposition 4.1
 * applied to 64 pending swaps at once) the update of N beside that of Z and the products computed ahead.
 * osscar_debug_side_stream(0) runs everything in order on the context's stream, (1) (the default) restores the overlap.
 * Process-wide.  The inverse is bit-identical either way (every tile sees the same operations in the same order); the
 * search may differ in the last digits of the row norms, because the candidates for the products computed ahead are then
 * picked after the score refresh instead of before it. */
osscar_status osscar_debug_side_stream(int32_t enable);

/* Host-only inspection of the Gram kernel's tile schedule (no device is touched): writes up to `capacity` (row, column)
 * pairs of 128 x 128 tiles, in workgroup order, to out_host (2 ints each; (-1, -1) = padding) and returns the length of
 * the schedule, or -1 for a bad d1.  Workgroup i runs on XCD i % 8. */
int32_t osscar_debug_tile_schedule(int64_t d1, int32_t* out_host, int32_t capacity);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the quadratic form of one small layer in one call, with no context and no workspace.  Same result
 * as osscar_gram(ctx, X, n, ldx, finalize = 1, W, ...) followed by reading H, G, lambda and c0 back:
 *   H = X^T X + lambda I (float32, d1 x d1, both triangles), lambda = lambda_abs + lambda_rel * mean(diag(X^T X)),
 *   G = H W (float32, d1 x m), c0 = Tr(W^T G); products accumulated in float64.
 * X_dev: dev, row-major n x d1 (leading dimension ldx), dtype x_dtype; W_dev: dev, d1 x m (ldw), dtype w_dtype;
 * H_dev, G_dev: dev outputs, dense (leading dimensions d1 and m), G_dev may lie where W_dev does; scalars_dev: dev, 2 float64 = {lambda, c0}.
 * Everything is enqueued on hip_stream (a hipStream_t, NULL = default stream); the call does not wait for it and
 * calls no hipMalloc, hipFree or other allocating routine.  What osscar_gram keeps in the caller's workspace meanwhile
 * (float64 accumulator, partial tiles, scalars) lives in a device array of OSSCAR_STATIC_SCRATCH_BYTES that
 * every GPU the library runs on holds until the process ends.  Limits: d1, m <= OSSCAR_STATIC_MAX_DIM, any n >= 0;
 * larger sizes return OSSCAR_ENOMEM.  All calls on one GPU share that array: calls that overlap in time on one GPU
 * (different streams or host threads) race and must be serialised by the caller.  After a failure
 * osscar_last_error(NULL) describes it (per host thread). */
#define OSSCAR_STATIC_MAX_DIM 1024
#define OSSCAR_STATIC_SCRATCH_BYTES 21037056
osscar_status osscar_gram_static(const void* X_dev, int64_t n, int64_t ldx, int32_t x_dtype, const void* W_dev, int64_t ldw,
                                 int32_t w_dtype, int64_t d1, int64_t m, double lambda_abs, double lambda_rel, float* H_dev,
                                 float* G_dev, double* scalars_dev, void* hip_stream);

/* ----------------------------------------------------------------------------------------------------------------------
 * Running, serving, scoring and training a pruned layer.  These calls take no context.  Everything is enqueued on
 * hip_stream (a hipStream_t, NULL = default stream) and may be captured into a graph; no call waits for it, allocates or keeps
 * anything.  A workspace is device memory of the size that the query beside the call names, at a 256-byte boundary, with any
 * contents; two calls may use the same one if they are ordered.  Buffers of one call must not overlap unless said.  dtypes are
 * OSSCAR_F32 or OSSCAR_BF16 unless said.  No size may exceed 2^30, and no product what a launch takes (of 16 rows or fewer: 2^27 columns and more).  After a failure
 * osscar_last_error(NULL) describes it (per host thread).
 * ---------------------------------------------------------------------------------------------------------------------- */

/* Gated feed-forward layer (the other common form of the layers whose neurons Section 3 prunes; its output is the X of the
 * down projection's Gram, osscar_gram):
 *   g = X Wg,  u = X Wu,  H = act(g) * u  (element by element),   X n x d, Wg and Wu d x f, H n x f.
 * Sums are float32; H is rounded once.  float32 operands of up to 16 tokens (32, where d f <= 2^25) are multiplied as they are; of more tokens, and in every product of
 * the backward pass, as three bf16 pieces each, which leaves the error of a float32 product, but an infinity makes its row or column of the product NaN, and operands
 * below 1e-34 lose bits (relative error of the product 3e-6 at 1e-35, 3e-4 at 1e-37).
 * bf16 takes d up to 4194296 (backward: f too) and f up to 16777208, but for 16 rows or fewer of small or unaligned f x d weights, which have no such limit. */
enum { OSSCAR_ACT_SILU = 0, OSSCAR_ACT_GELU = 1 /* 0.5 g (1 + erf(g / sqrt 2)) */, OSSCAR_ACT_GELU_TANH = 2, OSSCAR_ACT_RELU = 3 };
typedef struct {
  int64_t n, d, f;    /* tokens (n = 0: nothing to do), inputs, neurons */
  int64_t ldx;        /* leading dimension of X */
  int64_t ldw;        /* leading dimension of Wg and Wu */
  int64_t ldh;        /* leading dimension of H and dH */
  int32_t dtype;      /* of X, Wg, Wu, H, dH, dX */
  int32_t act;
  int32_t rows_out;   /* 0: Wg, Wu are d x f in memory (as W of this interface); nonzero: f x d, a neuron's weights side by side */
  int32_t unaligned;  /* nonzero: X, Wg or Wu may begin at any element; zero: at a 16-byte boundary (bf16) */
} osscar_gated_desc;
/* Workspace of a forward call (backward = 0), of a backward call with G and U (1) or without (2); 0 if the description is invalid.  A
 * forward call takes: none, where its tiles fill the chip; where they leave part of it idle, the sums of the parts that a contraction is dealt out in (1 x 2048 x 4096 bf16 17 MB,
 * float32 64 x 7168 x 14336 66 MB, 202 MB at most); and copies of bf16 operands whose rows do not begin at 16-byte boundaries or are not a multiple of 8 long. */
size_t osscar_gated_workspace_bytes(const osscar_gated_desc* desc, int32_t backward);
/* G_dev, U_dev (both or neither): dense n x f float32 outputs, g and u for osscar_gated_backward. */
osscar_status osscar_gated_forward(const osscar_gated_desc* desc, const void* X_dev, const void* Wg_dev, const void* Wu_dev, void* H_dev,
                                   float* G_dev, float* U_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream);
/* Gradients, given dH (n x f, leading dimension ldh):  dg = dH u act'(g), du = dH act(g) (both rounded to the dtype before the
 * products), dX = dg Wg^T + du Wu^T, dWg = X^T dg, dWu = X^T du.  G_dev, U_dev: what forward left there, or NULL: g and u are computed
 * again.  dX_dev (may be NULL): leading dimension lddx.  dWg_dev, dWu_dev (both or neither): layout of Wg, leading dimension lddw, dtype
 * dw_dtype; they are written, not added to.  act' is 0 at the corner of ReLU. */
osscar_status osscar_gated_backward(const osscar_gated_desc* desc, const void* X_dev, const void* Wg_dev, const void* Wu_dev, const void* dH_dev,
                                    const float* G_dev, const float* U_dev, void* dX_dev, int64_t lddx, void* dWg_dev, void* dWu_dev, int64_t lddw,
                                    int32_t dw_dtype, void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* Products in 8-bit integers, for serving kept rows: with a scale per token and one per output channel
 *   s_i = max_k |X_ik| / 127,  q_ik = X_ik / s_i to the nearest integer (halves to even),  Y_ij = s_i w_j sum_k q_ik Wq_jk + bias_j.
 * The sum is exact (int32; d1 <= OSSCAR_INT_MAX_DIM).  A row of zeros has scale 0 and gives bias; a row with an infinity or NaN gives NaN, and
 * so does a channel.
 * osscar_int_weights: W_dev is d1 x m (rows_out = 0) or m x d1 (nonzero) in memory, leading dimension ldw; Wq_dev is m x d1 with leading
 * dimension ldq (a multiple of 16, at a 16-byte boundary; zeros from column d1 on), w_scale_dev m float32.
 * osscar_int_rows: the same of the n rows of X, for several products with the same X. */
#define OSSCAR_INT_MAX_DIM 131071
osscar_status osscar_int_weights(const void* W_dev, int64_t d1, int64_t m, int64_t ldw, int32_t w_dtype, int32_t rows_out, int8_t* Wq_dev, int64_t ldq,
                                 float* w_scale_dev, void* hip_stream);
osscar_status osscar_int_rows(const void* X_dev, int64_t n, int64_t d1, int64_t ldx, int32_t x_dtype, int8_t* Xq_dev, int64_t ldq, float* x_scale_dev,
                              void* hip_stream);
/* Workspace of osscar_int_product; 0 if the sizes are invalid. */
size_t osscar_int_workspace_bytes(int64_t n, int64_t d1, int64_t m);
/* x_dtype OSSCAR_F32 or OSSCAR_BF16: X is quantised here, x_scale_dev must be NULL; OSSCAR_I8: X_dev is Xq with x_scale_dev (n float32).
 * Wq_dev as osscar_int_weights leaves it (what lies in a row from column d1 on does not matter).  bias_dev: m float32, or NULL.  Y_dev: n x m,
 * leading dimension ldy, dtype y_dtype. */
osscar_status osscar_int_product(const void* X_dev, int64_t n, int64_t d1, int64_t ldx, int32_t x_dtype, const float* x_scale_dev, const int8_t* Wq_dev,
                                 int64_t ldq, const float* w_scale_dev, int64_t m, const float* bias_dev, void* Y_dev, int64_t ldy, int32_t y_dtype,
                                 void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* What a model answers with, from its logits (n x vocab, leading dimension ld, the paper's perplexities are the exponential of the mean of -logp;
 * Section 5): with z = scale * logits and 0 < scale < 2.3e38,
 *   logp_i = z_{i,t_i} - lse_i,  entropy_i = -sum_v p_iv log p_iv,  lse_i = log sum_v exp z_iv,
 * and the `top` (<= OSSCAR_TOP_MAX, <= vocab) largest logits of each row, largest first, equal ones by index, NaN before all others.
 * targets_dev: n int64; negative: the row has no target, logp_i = 0; vocab or more: logp_i = NaN.
 * logp_dev, entropy_dev: n float32 (entropy may be NULL).  lse_dev: n x 2 float32 (may be NULL), the largest logit m of the row and
 * log sum_v exp(scale (l_v - m)): lse_i = scale m + that, in two parts for osscar_logprobs_backward.  top_index_dev, top_logp_dev: n x top int64 and float32
 * (ignored with top = 0).  A logit of minus infinity has probability 0.  A row of nothing else has lse minus infinity, entropy 0, and logp minus infinity
 * for its target and its alternatives; a row with NaN or plus infinity has NaN. */
#define OSSCAR_TOP_MAX 64
size_t osscar_logprobs_workspace_bytes(int64_t n, int64_t vocab, int32_t top);
osscar_status osscar_logprobs(const void* logits_dev, int64_t n, int64_t vocab, int64_t ld, int32_t dtype, const int64_t* targets_dev, float scale,
                              int32_t top, float* logp_dev, float* entropy_dev, float* lse_dev, int64_t* top_index_dev, float* top_logp_dev,
                              void* workspace_dev, size_t workspace_bytes, void* hip_stream);
/* Gradient of sum_i (dlogp_i logp_i + dentropy_i entropy_i + sum_j dtop_ij top_logp_ij) with respect to the logits:
 *   scale [ dlogp (1{v = t} - p_v) - dentropy p_v (log p_v + entropy) + sum_j dtop_j (1{v = top_index_j} - p_v) ].
 * Any of dlogp_dev, dentropy_dev and dtop_dev may be NULL; entropy_dev goes with dentropy_dev, top_index_dev with dtop_dev.  A row without a target ignores
 * dlogp_i; with dlogp_dev a target of vocab or more makes the row NaN; a row of minus infinities alone has gradient 0 whatever its target.  dlogits_dev: leading
 * dimension ldd, dtype as logits; it may be logits_dev itself (with ldd = ld). */
osscar_status osscar_logprobs_backward(const void* logits_dev, int64_t n, int64_t vocab, int64_t ld, int32_t dtype, const int64_t* targets_dev, float scale,
                                       const float* lse_dev, const float* dlogp_dev, const float* entropy_dev, const float* dentropy_dev, int32_t top,
                                       const int64_t* top_index_dev, const float* dtop_dev, void* dlogits_dev, int64_t ldd, void* hip_stream);

/* Layer norm of the rows of X (n x d), in front of the projections that a pruned layer is made of:
 *   mu = mean x,  r = 1 / sqrt(mean (x - mu)^2 + eps),  Y = (x - mu) r w + b.
 * w_dev, b_dev: d of w_dtype; either may be NULL (1 and 0).  stats_dev: n x 2 float32 (may be NULL), mu and r of each row for osscar_layernorm_backward.  Sums are
 * float32; a row whose squares sum to no float32 (values of 1e18 and beyond) or that holds an infinity or NaN is NaN.  Y_dev may be X_dev (ldy = ldx).  X and Y have
 * one dtype; eps must be a positive float32. */
osscar_status osscar_layernorm_forward(const void* X_dev, int64_t n, int64_t d, int64_t ldx, int32_t dtype, const void* w_dev, const void* b_dev, int32_t w_dtype, float eps,
                                       void* Y_dev, int64_t ldy, float* stats_dev, void* hip_stream);
/* Gradients, given dY (dtype as X): with h = (x - mu) r and g = dY w,  dX = r (g - mean g - h mean(g h)),  dw = sum over rows of dY h,  db = sum of dY.  dX_dev, dw_dev and
 * db_dev: any may be NULL; dX_dev may be dY_dev or X_dev (of one leading dimension).  dw and db: dw_dtype, written, not added to, in an order that does not change from call
 * to call.  A call that wants neither takes no workspace; osscar_layernorm_workspace_bytes is 0 if the sizes are invalid. */
size_t osscar_layernorm_workspace_bytes(int64_t n, int64_t d);
osscar_status osscar_layernorm_backward(const void* X_dev, int64_t n, int64_t d, int64_t ldx, int32_t dtype, const void* w_dev, int32_t w_dtype, const void* dY_dev, int64_t lddy,
                                        const float* stats_dev, void* dX_dev, int64_t lddx, void* dw_dev, void* db_dev, int32_t dw_dtype, void* workspace_dev,
                                        size_t workspace_bytes, void* hip_stream);

/* Low-rank adapters of many requests beside a shared projection (one that osscar_int_product serves, or any other), each row with its own:
 *   T_i = A_e x_i,  y_i = base_i + s_e B_e^T T_i,   e = index_i,   X n x d, Y and base n x m, T n x rank.
 * A is count x rank x d and B count x rank x m in memory: a component's numbers side by side in both (B of a layer m x rank is stored transposed, once).  index: n int64; a row with a
 * negative one has no adapter (y = base), one with `count` or more is NaN.  Without an index every row has the first adapter.  scale: count float32 (NULL: 1).  ranks: count int32 (NULL: all of
 * `rank`), the components of each adapter that count, from the first on; the others are not read.  base may be NULL (zeros) or Y itself.  Products of bf16 are summed in float32, T is float32 and goes
 * into the second product as two bf16 pieces (16 bits; an infinity there makes its row NaN), y is rounded once.  Rows of one adapter next to each other are fastest: 32 neighbouring rows
 * are read once for each adapter that they have; from 512 rows and 8 adapters on (backward with dA and dB: from 257 rows on) the rows are put in that order first. */
#define OSSCAR_ADAPTERS_MAX 4096
#define OSSCAR_ADAPTER_MAX_RANK 1024
typedef struct {
  int64_t n, d, m;            /* rows (n = 0: nothing to do; at most 2^22), inputs, outputs */
  int64_t ldx;                /* leading dimension of X */
  int64_t lda, next_a;        /* elements from one component of A to the next, from one adapter to the next */
  int64_t ldb, next_b;        /* the same of B */
  int32_t count, rank;        /* at most OSSCAR_ADAPTERS_MAX, OSSCAR_ADAPTER_MAX_RANK */
  int32_t dtype;              /* of X, A, B, base, Y, dY, dX */
  int32_t index;              /* nonzero: the calls are given an index */
} osscar_adapters_desc;
/* Workspace of a forward call (backward = 0), of a backward call (1), or of one without dA and dB (2); 0 if the description is invalid (for 1: also if
 * d and m have 2^24 blocks of 128 columns together). */
size_t osscar_adapters_workspace_bytes(const osscar_adapters_desc* desc, int32_t backward);
/* T_dev: dense n x rank float32 output for osscar_adapters_backward (zeros where there is no adapter or component), or NULL. */
osscar_status osscar_adapters_forward(const osscar_adapters_desc* desc, const void* X_dev, const void* A_dev, const void* B_dev, const int64_t* index_dev,
                                      const float* scale_dev, const int32_t* ranks_dev, const void* base_dev, int64_t ldbase, void* Y_dev, int64_t ldy, float* T_dev,
                                      void* workspace_dev, size_t workspace_bytes, void* hip_stream);
/* Gradients, given dY (n x m, leading dimension lddy):  dT_i = s_e B_e dY_i,  dX_i = base_i + A_e^T dT_i,  dA_e = sum of dT_i x_i^T and dB_e = s_e sum of T_i dY_i^T over the rows of
 * e.  T_dev: what forward left there, or NULL: computed again.  base_dev: n x d, leading dimension ldbase, NULL (zeros) or dX itself (the gradient that came through the
 * shared projection).  dX_dev may be NULL, or dY_dev or X_dev, which are read first (and base too: around a square projection they may be one).  dA_dev and dB_dev may be NULL (both or
 * neither): dense, of the shapes of A and B, dw_dtype, written, not added to, zeros for adapters and components without
 * rows, in an order that does not change from call to call.  A row whose index is `count` or more has dX of NaN and no part in dA and dB. */
osscar_status osscar_adapters_backward(const osscar_adapters_desc* desc, const void* X_dev, const void* A_dev, const void* B_dev, const int64_t* index_dev,
                                       const float* scale_dev, const int32_t* ranks_dev, const void* dY_dev, int64_t lddy, const float* T_dev, const void* base_dev, int64_t ldbase,
                                       void* dX_dev, int64_t lddx, void* dA_dev, void* dB_dev, int32_t dw_dtype, void* workspace_dev, size_t workspace_bytes,
                                       void* hip_stream);

/* AdamW, one step over many tensors: with t = step counted from 1, and float32 factors rounded once from float64, every operation below rounded by itself,
 *   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) (g g),  p = p (1 - lr weight_decay) - lr / (1 - b1^t) (m / (sqrt v / sqrt(1 - b2^t) + eps)).
 * A tensor is n contiguous elements of any shape (n = 0: nothing to do).  p: float32, or bf16, rounded to the nearest, with a float32 copy `master` that holds the
 * parameters (p is then written, not read), or without.  Nothing may overlap, within a tensor or between tensors.
 * bits 32: m and v are float32.  bits 8: m and v are codes of 8 bits, m_scale and v_scale a power of two (float32) for each OSSCAR_ADAMW_BLOCK elements of a tensor (the last block may be shorter):
 *   m = m_scale * the 8-bit float e4m3 (sign, 4 bits of exponent with bias 7, 3 of mantissa, subnormal numbers);
 *   sqrt v = v_scale * (c < 16 ? c : (16 + c % 16) 2^(c / 16 - 1)), c a byte: whole numbers to 32, then 16 steps an octave, to 31 * 2^14.
 * The scales put the largest power of two of a block at 2^7 and 2^17 (never below 2^-126); numbers are rounded to the nearest code (halves to even), but a v above zero keeps a code above
 * zero.  All codes and scales 0 is a state of zeros.  A state that is not finite makes its block's scale NaN, and so the whole block from the next step on.
 * stochastic: codes, and bf16 parameters without a master, are rounded up with the probability that their part of a step is, so that changes smaller than a step (0.001 of v) are not lost
 * on average: bits r of the hash h below are added to the float32 number under its last kept bit and the rest cut off; for m the low 20 of h, for sqrt v the high 19 of the
 * low 32 of 0x9E3779B9 h, for p the high 16 of h (numbers below the smallest normal one first have it added).  h = mix(low 32 bits of i ^ mix(high 32 bits of i ^ mix(seed))), i the number of
 * the element in the call, each tensor before it counting as whole blocks; mix(x): x = (x ^ x >> 16) * 0x9E3779B9, x = (x ^ x >> 15) * 0xB7E15163, x ^ x >> 16 in 32 bits.  A seed of its own for each step;
 * with step_dev the low 32 bits of the step are added to it, so that each replay of a captured step has one.
 * lr_dev, step_dev (may be NULL): one float32, one int64 on the device that take the place of lr and step (below 1: 1), for steps that are captured once and replayed.  grad_scale_dev (may be NULL): one float32 that
 * every gradient is multiplied by first; if it is not finite the call changes nothing. */
#define OSSCAR_ADAMW_BLOCK 256
typedef struct {
  int64_t n;
  void* p;
  float* master;               /* or NULL */
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;    /* bits 8; else not looked at */
  int32_t p_dtype, g_dtype;    /* OSSCAR_F32 or OSSCAR_BF16, each of its own */
} osscar_adamw_tensor;
typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  int64_t step;
  const float* lr_dev;
  const int64_t* step_dev;
  const float* grad_scale_dev;
  uint32_t seed;
  int32_t stochastic;
  int32_t bits;
} osscar_adamw_desc;
/* tensors: host array, read during the call. */
osscar_status osscar_adamw(const osscar_adamw_tensor* tensors, int64_t count, const osscar_adamw_desc* desc, void* hip_stream);
/* What 8-bit states stand for: m and sqrt v of each tensor in bf16, which holds them exactly but for m of scales below 2^-124 (m reaches 2^-9 scales, bf16's steps end at 2^-133:
 * rounded to the nearest of them, halves to even); n elements at m_out[k] and root_out[k] (host arrays of device pointers).  Of the tensors n, m, v, m_scale and v_scale are looked at. */
osscar_status osscar_adamw_values(const osscar_adamw_tensor* tensors, int64_t count, void* const* m_out, void* const* root_out, void* hip_stream);

/* Description of the last failure: of a context, or (ctx == NULL) of the last failed call on this host thread that takes
 * no context. */
const char* osscar_last_error(const osscar_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* OSSCAR_H */
