/*
 * fmm8 -- Strassen-type rank-7 bilinear matrix multiplication under a
 * block-scaled e4m3 model, with an fp64 error measurement, on AMD MI355X
 * (gfx950).
 *
 * The operation (Section 2.1 and Section 2.2 of "Fast Matrix Multiplication
 * in fp8: Certified Coefficient Optimization and Measured Error"):
 *
 *   A (M x K) and B (K x N) are split into a 2^l x 2^l grid of sub-blocks.
 *   For every term r of the depth-l flattened realization (U, V, w)
 *     x_r = sum_b U[r,b] A_b   (fp32)          -- encoded combinations,
 *     y_r = sum_b V[r,b] B_b   (fp32)
 *   are formed from the unquantized operands, quantized to e4m3 with one
 *   scale per block of `block` consecutive elements along the contracted
 *   axis (Assumption 1; Appendix E.2), multiplied with fp32 accumulation,
 *   and decoded:  C_(I,K) = sum_r w[r, K 2^l + I] P_r.
 *
 * Coefficient conventions (Appendix A, eq. A.1): rv(A) = (a11,a12,a21,a22);
 * U_r is indexed by 2i+j for A-block (i,j), V_r by 2j+k, and the third factor
 * is cyclic, w_r = rv(W_r^T), indexed by 2k+i.  A depth-l table (Section 3.2,
 * Kronecker powers; Section 4.3, flattened realizations) has T = R^l terms
 * r = sum_t r_t R^(l-t) and 4^l columns, sub-block (P,Q) at column P 2^l + Q;
 * each entry is the product of the l base coefficients, multiplied left to
 * right in binary64 and rounded once to binary32.
 *
 * Memory and ownership.  Every device buffer is allocated and owned by the
 * caller; matrices are row-major and contiguous, batch-major.  Opaque host
 * handles (fmm_real, fmm_plan) are owned by the library and released with
 * their _destroy call.  fmm_encode, fmm_multiply and fmm_matmul never
 * allocate; fmm_plan_create uploads the plan's coefficient tables to the
 * device that is current at the time of the call, and the plan may only be
 * used with that device.
 *
 * Execution.  Device calls are asynchronous on `stream` (a hipStream_t
 * passed as void*; NULL is the null stream) and never synchronize the host.
 * A plan is immutable: one plan may be used concurrently on several streams
 * with distinct workspaces.
 *
 * Errors.  Every call returns an int status: FMM_OK (0) or a negative code.
 * No exception crosses the boundary.  Device-side problems (a failed launch)
 * are reported as FMM_ERR_HIP; fmm_status_string() names any code, and
 * fmm_last_error_detail() returns the last HIP error string of the calling
 * thread.  Non-finite inputs are undefined behaviour.
 */
#ifndef FMM8_H
#define FMM8_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------ */
enum {
  FMM_OK = 0,
  FMM_ERR_ARG = -1,          /* null pointer, out-of-range enum, bad tolerance */
  FMM_ERR_SHAPE = -2,        /* dimensions not divisible as required */
  FMM_ERR_UNSUPPORTED = -3,  /* a shape/rule/block/depth the library does not run */
  FMM_ERR_NOT_EXACT = -4,    /* Brent residual above the tolerance */
  FMM_ERR_SINGULAR = -5,     /* a basis change with |det| < 1e-12 */
  FMM_ERR_HIP = -6,          /* a HIP runtime call or a kernel launch failed */
  FMM_ERR_DEVICE = -7,       /* the device is not gfx950 */
  FMM_ERR_WORKSPACE = -8,    /* workspace too small or misaligned */
  FMM_ERR_NOMEM = -9         /* host allocation failed */
};

/* ---- named realizations ------------------------------------------------ */
enum {
  FMM_CUBIC8 = 0,            /* the cubic <2,2,2;8> algorithm, Phi = 8 (Section 3.2) */
  FMM_STRASSEN = 1,          /* Strassen 1969, M1..M7 in classical order, Phi = 32 */
  FMM_WINOGRAD = 2,          /* Strassen-Winograd variant, raw gauge, Phi = 56 (Table E.2) */
  FMM_TSTAR = 3              /* the Phi-optimal T*, Phi = 200/9 (Theorem 1; eq. A.2) */
};

/* ---- block-scale rules (Appendix E.2; power-of-two variants) ------------ */
enum {
  FMM_RULE_FP32_AMAX = 0,    /* s = fl32(max(amax, fl32(1e-12)) / 448), stored as fp32 */
  FMM_RULE_POW2_CEIL = 1,    /* s = 2^e, e the least integer with a <= 448 2^e; E8M0 byte */
  FMM_RULE_POW2_OCP = 2      /* s = 2^(floor(log2 a) - 8) (OCP MX rule, clips to 448); E8M0 */
};

/* ---- plan flags ---------------------------------------------------------- */
enum {
  /* Sum the products of the dequantized operands at fp32 precision.  The
   * default sub-product path feeds the e4m3 codes and E8M0 scales to the
   * fp8 matrix cores, whose dot product aligns each group of eight products
   * to the group's largest and keeps 13 bits below it (measured on gfx950);
   * with this flag the operands go to the bf16 matrix cores (23 retained
   * bits) exactly: with E8M0 scales each code is converted to bf16 together
   * with its block's power of two (the dequantized value itself, exact for
   * every scale the rules produce), with fp32 scales each block's partial
   * sum of codes is scaled and accumulated in fp32.  Half the peak rate of
   * the default path.  FP32_AMAX scales and block 16 always take this path;
   * tile-aligned plans with FP32_AMAX scales run on FMM_LAYOUT_TILE256x64
   * whatever K. */
  FMM_FLAG_EXACT_DOT = 1,
  /* Weight-side deployment granularity (Appendix E, weight-scale
   * granularity; the real kernel's 128 x 128 weight blocks): one B-side scale
   * covers 128 consecutive columns of B (rows of y_r^T) x `block` positions
   * of the contracted axis, its maximum taken over the encoded combination;
   * the last block of a ragged N / 2 is short.  The stored scales stay one per
   * (row, block), replicated over each 128-row block.  Depth 1 only
   * (FMM_ERR_UNSUPPORTED otherwise). */
  FMM_FLAG_B_BLOCK128 = 2,
  /* Round each encoded B combination to bfloat16 (nearest, ties to even)
   * before its scale and cast (Appendix E: the real path's pre-round of the
   * encoded weights).  Depth 1 only. */
  FMM_FLAG_B_BF16 = 4,
  /* Take the large-tile sub-product path (FMM_LAYOUT_TILE256x64) whenever
   * the shape allows it.  Without the flag, plans with E8M0 scales take that
   * path only where K / 2^l >= 1024, and at depth 1 not where the fused
   * 128 x 128 tiles are estimated the faster (fused_beats_large_tiles in
   * plan.cpp): it writes every fp32 P_r to the workspace and reads it back,
   * which costs more than it saves there (plans with fp32 scales take it
   * whenever the shape allows).  No effect on the result's definition; shapes the path cannot
   * take ignore the flag. */
  FMM_FLAG_LARGE_TILE = 8
};

typedef struct fmm_real fmm_real;   /* a base realization (U, V, w) of <m,k,n;R>, binary64 */
typedef struct fmm_plan fmm_plan;   /* one problem shape bound to a realization */

typedef struct {
  int64_t batch;   /* number of independent products, >= 0 */
  int64_t M, K, N; /* each >= 0 and divisible by 2^depth (by m, k, n for a realization of
                    * another shape <m,k,n;R>); K / 2^depth (K / k) divisible by block */
  int32_t depth;   /* recursion (Kronecker) depth l: 1, 2 or 3 */
  int32_t block;   /* e4m3 block length along the contracted axis: 16, 32 or 128 */
  int32_t rule;    /* FMM_RULE_* */
  int32_t flags;   /* FMM_FLAG_* bits; others must be 0 */
} fmm_plan_desc;

/* Layouts of the quantized operands in a workspace (fmm_view.code_layout). */
enum {
  /* codes [batch][terms][rows][kdim], scales [batch][terms][rows][kblocks] */
  FMM_LAYOUT_ROWS = 0,
  /* codes [batch][terms][rows / 256][kdim / 64][256][64]: 256-row x 64-byte
   * tiles, each contiguous; inside a tile, 16-byte chunk c of tile row t sits
   * at chunk c ^ ((t >> 2) & 3) of that row.
   * scales [batch][terms][kblocks][rows]: for each block of the contracted
   * axis, one scale per row.  E8M0 bytes have the rows of every 256-row tile
   * permuted so that tile row 128 h + 32 i + j (h < 2, i < 4, j < 32) sits at
   * byte 4 (32 h + j) + i; fp32 scales (FMM_RULE_FP32_AMAX) are in row order.
   * Used by plans whose sub-products run on 256-row tiles: depth 1 or 2,
   * M / 2^l and N / 2^l multiples of 256, K / 2^l a multiple of 64 (of 128
   * at block 128), and either fp32 scales (the exact-dot path) or E8M0
   * scales with FMM_FLAG_LARGE_TILE or K / 2^l >= 1024 (see there) (the fp8 matrix cores
   * at blocks 32 and 128, the exact-dot path at block 16 or with
   * FMM_FLAG_EXACT_DOT); and every plan of a
   * realization of another shape (rows M / m and N / n, kdim K / k).  The B
   * side is read as 128-row halves of these tiles. */
  FMM_LAYOUT_TILE256x64 = 1,
  /* codes [batch][terms][rows / 128][kdim / 128][128][128]: 128-row x 128-byte
   * tiles, each contiguous; inside a tile, 16-byte chunk c of tile row t sits
   * at chunk c ^ (t & 7) ^ ((t >> 3) & 1) of that row.
   * scales [batch][terms][rows / 128][kdim / 128][128][4 or 8]: for each tile
   * row and 128-byte step, 4 E8M0 bytes: at block 32 the step's blocks 0, 2,
   * 1, 3 in that order, at block 128 the step's one block repeated 4 times;
   * at block 16, 8 bytes: the step's blocks 0, 2, 4, 6, then 1, 3, 5, 7.
   * Used by the other plans with E8M0 scales (blocks 16, 32 and 128) whose
   * M / 2^l and N / 2^l are multiples of 128 and K / 2^l a multiple of 128. */
  FMM_LAYOUT_TILE128x128 = 2
};

/* Where the quantized operands of one side sit inside a workspace, in layout
 * code_layout (A side: rows = M / 2^l; B side: rows = N / 2^l, i.e. y_r
 * transposed; the contracted axis has kdim = K / 2^l codes in kblocks blocks).
 * codes : uint8 e4m3 codes
 * scales: one per block; uint8 E8M0 (e + 127) when scale_bytes == 1, IEEE
 *         binary32 when scale_bytes == 4. */
typedef struct {
  void *codes;
  void *scales;
  int64_t batch, terms, rows, kdim, kblocks;
  int32_t scale_bytes;
  int32_t code_layout; /* FMM_LAYOUT_* */
} fmm_view;

/* ---- realizations (host only; no device needed) ------------------------ */

/* A named realization.  *out receives a new handle. */
int fmm_realization_builtin(int which, fmm_real **out);

/* A realization of <m,k,n;R> (Section 2.1: R rank-one terms of the matrix
 * multiplication tensor of an m x k by k x n product) from caller arrays U, V,
 * w, each R x (m k), R x (k n), R x (n m) row-major binary64: A is split into
 * an m x k grid of sub-blocks, block (i, j) at index i k + j; B into a k x n
 * grid, block (j, l) at j n + l; C block (i, l) takes w's index l m + i (the
 * cyclic third factor of Appendix A; at <2,2,2> the conventions above).
 * Exact means sum_r U_r[i k + j] V_r[j' n + l] w_r[l' m + i'] =
 * [j = j'][l = l'][i = i'] (the Brent equations); if the largest deviation
 * exceeds tol the call fails with FMM_ERR_NOT_EXACT (tol < 0 is FMM_ERR_ARG).
 * <2,2,2;R> takes 1 <= R <= 8 and runs at depths 1 to 3.  Other shapes (the
 * rows of Table E.1 beyond <2,2,2>) take m k, k n, n m <= 64 and
 * 1 <= R <= 4096 (FMM_ERR_UNSUPPORTED for larger grids; m, k or n < 1 or R
 * out of range: FMM_ERR_ARG) and run at depth 1 only, on the large-tile plans
 * (FMM_LAYOUT_TILE256x64). */
int fmm_realization_create(int m, int k, int n, int R, const double *U, const double *V,
                           const double *w, double tol, fmm_real **out);

/* D . g for g = (X, Y, Z) in GL(2)^3 (eq. A.1):
 *   u -> u (X (x) Y^-T), v -> v (Y (x) Z^-T), w -> w (Z (x) X^-T),
 * each 2x2 factor given row-major (4 doubles).  Evaluated in binary64 in
 * this order: the inverse by the adjugate (det = a d - b c, entries divided
 * by det), then the Kronecker matrix, then u K with each entry summed in
 * ascending index; no fused multiply-add.  |det| < 1e-12 gives
 * FMM_ERR_SINGULAR.
 * Another shape <m,k,n> takes g in GL(m) x GL(k) x GL(n): X m x m, Y k x k,
 * Z n x n row-major, the same formulas (u indexed i k + j, so
 * X (x) Y^-T has entry [i k + j][i' k + j'] = X[i][i'] (Y^-T)[j][j'];
 * likewise v, w), i.e. U_r -> X^T U_r Y^-T, V_r -> Y^T V_r Z^-T,
 * W_r -> Z^T W_r X^-T as matrices; the inverses by Gauss-Jordan elimination
 * with partial pivoting. */
int fmm_realization_transform(const fmm_real *d, const double X[4], const double Y[4],
                              const double Z[4], fmm_real **out);

/* The canonical rebalanced gauge (Appendix E.2):
 * (U_r, V_r, W_r) -> (U_r / s_r, s_r V_r, W_r), s_r = sqrt(|U_r| / |V_r|)
 * (terms with a zero U_r or V_r unchanged); any shape. */
int fmm_realization_rebalance(const fmm_real *d, fmm_real **out);

/* Re-basing (Section 3.1; the protocol of Appendix E.2): minimize Phi over
 * the change-of-basis orbit D . g, g = (X, Y, Z) in GL(2)^3 (eq. A.1), or in
 * GL(m) x GL(k) x GL(n) for another shape (fmm_realization_transform's
 * action; P = m^2 + k^2 + n^2 entries, 12 at <2,2,2>).
 * Starts: g = (I, I, I) (the realization itself) and, for s < nstarts, the
 * caller's triple starts[P s .. P s + P - 1] = (X, Y, Z), each row-major
 * (the paper draws X, Y, Z as I + 0.45 N(0,1) and rejects |det| < 1e-3; the
 * caller does the drawing).  Each start runs limited-memory BFGS (memory 10)
 * with a strong-Wolfe line search (c1 = 1e-4, c2 = 0.9) in binary64 over the
 * P entries of g, with the exact gradient, until the largest gradient entry
 * is at most gtol * max(1, Phi), progress falls below rounding, or max_iter
 * iterations.  The terminal g gives D . g by fmm_realization_transform's
 * arithmetic; among the terminal realizations with a finite Phi and a Brent
 * residual <= tol, the one with the least Phi (the earliest start on ties)
 * is returned in *out (a new handle), its Phi in *phi (may be NULL).
 * start_phi (may be NULL; 1 + nstarts entries) receives each start's terminal
 * Phi, NaN where it was singular or failed the exactness check.
 * Errors: FMM_ERR_ARG (null d or out; nstarts < 0; starts NULL while
 * nstarts > 0; max_iter < 1; gtol <= 0; tol < 0 or NaN); FMM_ERR_NOT_EXACT
 * if no start ends exact within tol.  Host only. */
int fmm_realization_optimize(const fmm_real *d, int nstarts, const double *starts, int max_iter,
                             double gtol, double tol, fmm_real **out, double *phi, double *start_phi);

/* Phi(D . g) for g = (X, Y, Z) = g[0..3], g[4..7], g[8..11] (row-major 2x2
 * each; eq. A.1) and its gradient with respect to those 12 entries, the
 * objective fmm_realization_optimize minimizes (another shape: X, Y, Z of
 * m^2, k^2, n^2 entries in that order, P in all, and grad of P entries).
 * phi may be NULL.  Errors: FMM_ERR_ARG (null d, g or grad).  A singular g
 * gives non-finite values. */
int fmm_realization_phi_gradient(const fmm_real *d, const double *g, double *phi, double *grad);

/* Phi = sum_r |U_r|^2 |V_r|^2 |W_r|^2 and Gamma = sum_r |U_r||V_r||W_r|
 * (Section 2.1) of the depth-l flattening (Phi^l, Gamma^l), and the Brent
 * residual of the base realization.  Any output pointer may be NULL.  Other
 * shapes than <2,2,2>: depth 1 only (FMM_ERR_UNSUPPORTED otherwise). */
int fmm_realization_metrics(const fmm_real *d, int depth, double *phi, double *gamma,
                            double *brent_resid);

/* R (base rank) and T = R^depth (other shapes: depth 1 only, as above). */
int fmm_realization_terms(const fmm_real *d, int depth, int64_t *rank, int64_t *terms);

/* The shape <m,k,n> and rank R of a realization (any pointer may be NULL). */
int fmm_realization_shape(const fmm_real *d, int *m, int *k, int *n, int *R);

/* The base coefficients, R x (m k), R x (k n), R x (n m) binary64 (R x 4 each
 * at <2,2,2>; any pointer may be NULL). */
int fmm_realization_coefficients(const fmm_real *d, double *U, double *V, double *w);

/* The exact fp32 depth-l tables the kernels use, T x 4^l each (other shapes:
 * depth 1, R x (m k), R x (k n), R x (n m), each entry rounded once). */
int fmm_realization_tables(const fmm_real *d, int depth, float *U, float *V, float *w);

void fmm_realization_destroy(fmm_real *d);

/* ---- plans and the product --------------------------------------------- */

/* Validates desc (FMM_ERR_ARG / FMM_ERR_SHAPE / FMM_ERR_UNSUPPORTED are
 * returned before any device call), then uploads the coefficient tables to
 * the current device (FMM_ERR_DEVICE if it is not gfx950).
 * A realization of another shape <m,k,n;R> splits A into m x k sub-blocks of
 * M / m x K / k, B into k x n of K / k x N / n, and runs at depth 1 on the
 * large-tile path only: M / m and N / n multiples of 256 and K / k a multiple
 * of 64 (of 128 at block 128), with no flags but FMM_FLAG_EXACT_DOT and
 * FMM_FLAG_LARGE_TILE; anything else is FMM_ERR_UNSUPPORTED (dimensions not
 * divisible by m, k, n or K / k by block: FMM_ERR_SHAPE).  Such plans have
 * no operand-noise or cross-term pass (FMM_ERR_UNSUPPORTED). */
int fmm_plan_create(const fmm_real *d, const fmm_plan_desc *desc, fmm_plan **out);

/* Bytes of device workspace fmm_encode/fmm_multiply/fmm_matmul need: the
 * codes and scales of both operands, plus, for large-tile plans the fp32
 * sub-products P_r, and for the others at depth >= 2 the inner-level partial
 * products.
 * The workspace must be 256-byte aligned. */
int fmm_plan_workspace_size(const fmm_plan *p, size_t *bytes);

/* Steps "encode + quantize" of both operands (device pointers dA: batch x M x K,
 * dB: batch x K x N, fp32, each 16-byte aligned) into the workspace. */
int fmm_encode(const fmm_plan *p, const float *dA, const float *dB, void *dWs, void *stream);

/* Pointers and extents of the quantized operands inside dWs (host call). */
int fmm_operand_views(const fmm_plan *p, void *dWs, fmm_view *a, fmm_view *b);

/* Steps "fp8 sub-products + W-combine" (Algorithm 1, the products P_r of the
 * quantized operands and C = sum_r w_r (x) P_r): reads the encoded workspace
 * and writes C (batch x M x N fp32, 4-byte aligned).  Equal to fmm_products
 * followed by fmm_combine on the same stream. */
int fmm_multiply(const fmm_plan *p, void *dWs, float *dC, void *stream);

/* The first half of fmm_multiply: the T block-scaled fp8 sub-products with
 * fp32 accumulation.  Plans with the large-tile layout (fmm_view.code_layout
 * == FMM_LAYOUT_TILE256x64) write every P_r, fp32, to the workspace (and
 * fmm_combine forms C = sum_r w_r (x) P_r over all T terms in one pass, in
 * ascending r with one fused multiply-add per nonzero weight); the others
 * fold the base-level w into the sub-product kernel and write C (depth 1) or
 * the per-outer-term partial sums (depth >= 2, workspace). */
int fmm_products(const fmm_plan *p, void *dWs, float *dC, void *stream);

/* The second half of fmm_multiply: what remains of the W-combine after
 * fmm_products (reads the workspace, writes C); nothing for the plans that
 * fold it into the sub-product kernel at depth 1. */
int fmm_combine(const fmm_plan *p, void *dWs, float *dC, void *stream);

/* The kernel that fmm_products launches for this plan, with its tile of a
 * sub-product's rows and columns, e.g. "gemm_tile256x256_kernel 256x256"
 * (a static string; NULL for a NULL plan). */
const char *fmm_products_kernel(const fmm_plan *p);

/* fmm_encode followed by fmm_multiply. */
int fmm_matmul(const fmm_plan *p, const float *dA, const float *dB, float *dC, void *dWs,
               void *stream);

void fmm_plan_destroy(fmm_plan *p);

/* ---- error measurement (Appendix E.2: relative error against an fp64 product) */

/* dCref = A B in binary64 (batch x M x N), from the fp32 operands. */
int fmm_reference_f64(int64_t batch, int64_t M, int64_t K, int64_t N, const float *dA,
                      const float *dB, double *dCref, void *stream);

/* Device scratch the reduction below needs (bytes; the scratch passed must
 * hold at least that many and be 8-byte aligned, else FMM_ERR_WORKSPACE). */
int fmm_error_stats_scratch_size(int64_t batch, int64_t M, int64_t N, size_t *bytes);

/* Per product b: dOut[2b] = sum (C - Cref)^2, dOut[2b+1] = sum Cref^2, binary64,
 * by a fixed-order two-pass reduction (identical results run to run).
 * dOut is a device pointer to 2*batch doubles. */
int fmm_error_stats(int64_t batch, int64_t M, int64_t N, const float *dC, const double *dCref,
                    double *dOut, void *dScratch, size_t scratch_bytes, void *stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * fmm_error_stats without the scratch argument.  The reduction's partials
 * live in a static device array of the library (8 MiB on every device the
 * library runs on, held until the process ends), so at most
 * FMM_ERROR_STATS_NOALLOC_MAX_BATCH products per call; a larger batch fails
 * with FMM_ERR_WORKSPACE (fmm_last_error_detail() says why) before any device
 * call.  Same kernels, same fixed order and results as fmm_error_stats.  The
 * call itself allocates nothing; its first call on a device looks up the
 * array's device address there.  Calls on one device share the array: calls
 * that overlap in time on one device (other streams, other threads) race and
 * must be serialized by the caller.  Every partial is written before it is
 * read, so a call does not depend on what an earlier call left there. */
#define FMM_ERROR_STATS_NOALLOC_MAX_BATCH 1024
int fmm_error_stats_noalloc(int64_t batch, int64_t M, int64_t N, const float *dC, const double *dCref,
                            double *dOut, void *stream);

/* ---- the codec alone --------------------------------------------------- */

/* Operand-side rounding energy of the encoding in dWs (Appendix D,
 * eq. D.1: the noise coefficient s^2 = sum (xhat - x)^2 / sum x^2 of the
 * model of Section 2.2).  Call after fmm_encode with the same dA, dB and
 * workspace: the combinations x_r are formed again with the encoder's
 * arithmetic, the stored codes and scales are decoded to xhat_r (exact in
 * binary64), and dOut (device, [batch][2][T][2] binary64; side 0 = A, 1 = B)
 * receives, for every batch element, side and flattened term, the sums of
 * (xhat - x)^2 and of x^2 over the term's positions (binary64, a fixed
 * summation order, so repeated calls agree bit for bit).  With
 * FMM_FLAG_B_BF16, x is the combination before the bfloat16 rounding.
 * dScratch: device, 8-byte aligned, at least fmm_encode_noise_scratch_size
 * bytes (FMM_ERR_WORKSPACE otherwise).  Depths 1 and 2 (FMM_ERR_UNSUPPORTED
 * at depth 3).  Asynchronous on stream. */
int fmm_encode_noise_scratch_size(const fmm_plan *p, size_t *bytes);
int fmm_encode_noise(const fmm_plan *p, const float *dA, const float *dB, const void *dWs, double *dOut,
                     void *dScratch, size_t scratch_bytes, void *stream);

/* The cross-term diagnostic of the error model (Appendix D: the share of
 * the error's linear part that the diagonal sum defining Phi leaves out).
 * Call after fmm_encode with the same dA, dB and workspace; depth-1 plans
 * only (FMM_ERR_UNSUPPORTED otherwise), any layout, rule and block.  With
 * X_r, Y_r the fp32 combinations (the encoder's arithmetic), dX_r, dY_r their
 * rounding residuals against the stored codes times their scales, t_r =
 * dX_r Y_r + X_r dY_r (m' x n', binary64) and L_q = sum_r w[r, q] t_r, dOut
 * (device, [batch][2] binary64) receives for every batch element
 * |L|^2 = sum_q |L_q|^2 and diag = sum_{r, q} w[r, q]^2 |t_r|^2, each by a
 * fixed summation order (repeated calls agree bit for bit); the residual
 * fraction is (|L|^2 - diag) / |L|^2.  dScratch: device, 256-byte aligned, at
 * least fmm_cross_terms_scratch_size bytes (16 (M + N) K / 2 + 8 M N / 4
 * bytes per term and product, FMM_ERR_WORKSPACE otherwise).  With
 * FMM_FLAG_B_BF16, Y_r is the combination before the bfloat16 rounding.
 * Asynchronous on stream; measurement, not on the timed path. */
int fmm_cross_terms_scratch_size(const fmm_plan *p, size_t *bytes);
int fmm_cross_terms(const fmm_plan *p, const float *dA, const float *dB, const void *dWs, double *dOut,
                    void *dScratch, size_t scratch_bytes, void *stream);

/* dOut[i] = e4m3 code of dIn[i] at unit scale: round to nearest, ties to the
 * even mantissa field, saturate to +-448, keep the sign (the cast the
 * quantizer applies after dividing by the block scale).  n >= 0; dIn must be
 * 16-byte and dOut 4-byte aligned. */
int fmm_e4m3_quantize(const float *dIn, uint8_t *dOut, int64_t n, void *stream);

/* dOut[i] = e4m3 code of dIn[i] / 2^e: the cast the power-of-two scale rules
 * (FMM_RULE_POW2_CEIL, FMM_RULE_POW2_OCP; E8M0 byte e + 127) apply to every
 * element of a block, through the same device routine as the encoder.  The
 * quotient is the binary32 value fl32(x / 2^e), then cast as above: round to
 * nearest, ties to the even mantissa field, saturate to +-448 (a quotient
 * beyond the binary32 range included), keep the sign.  e in [-126, 127] (the
 * rules produce -48 .. 120; FMM_ERR_ARG otherwise); n >= 0; dIn 16-byte and
 * dOut 4-byte aligned.  Asynchronous on stream. */
int fmm_e4m3_quantize_pow2(const float *dIn, uint8_t *dOut, int64_t n, int32_t e, void *stream);

/* ---- an 8-bit linear layer ------------------------------------------------
 *
 * The products above quantize both of their operands inside the call.  A
 * layer's weights, and activations that a norm has just written, are
 * quantized once and then multiplied, or kept, as they are; the calls below
 * make such operands, multiply them, and give the gradients of what they
 * stand for.
 *
 * Codes.  A matrix of `rows` x `cols` values is held as int8 codes q
 * [rows][fmm_q8_pitch(cols)] and fp32 scales s [rows]; the values are q s.  The
 * pitch is cols rounded up to 128, and codes past cols are zero: the calls that
 * write codes write those zeros, the ones that read codes rely on them.
 * Quantizing a row: a = max(amax |x|, 1e-12), q = the integer nearest
 * fl32(x fl32(127 / a)), ties to even, in [-127, 127]; s = fl32(a / 127).  A row
 * that holds a NaN or an infinity gets scale NaN and zero codes, so that what
 * is computed from it is NaN.  Codes written by the caller may also be -128.
 *
 * Checkpoint.  The same rule over each group of 128 columns of a row: codes as
 * above, scales [rows][pitch / 128].
 *
 * Types.  `type` names the activations' element type (FMM_F32, FMM_BF16,
 * FMM_F16).  Every sum, statistic and scale is fp32 (products of codes: int32,
 * exact), and a result is rounded once, to nearest even, when it is stored.
 *
 * Matrices are row-major and contiguous.  Codes must be 16-byte aligned, scales,
 * bias and other fp32 arrays 4-byte, activations aligned to their element
 * unless a call says more (FMM_ERR_ARG otherwise).  Unlike the calls above these
 * define the result for NaN and infinities: they propagate as in the formulas.
 * Asynchronous on `stream`; nothing is allocated or synchronized, so calls may
 * be captured into a graph. */
enum {
  FMM_F32 = 0,
  FMM_BF16 = 1,
  FMM_F16 = 2
};

/* Bytes (= codes) of one row of codes: cols rounded up to 128 (-1 if cols < 0). */
int64_t fmm_q8_pitch(int64_t cols);

/* dCodes, dScales = the codes of dX (rows x cols).  rows, cols >= 0; more than
 * 2^30 rows or 2^24 columns: FMM_ERR_UNSUPPORTED, as in the calls below. */
int fmm_q8_quantize(int type, int64_t rows, int64_t cols, const void *dX, int8_t *dCodes, float *dScales, void *stream);

/* dOut (rows x cols, `type`) = the values that codes stand for: group 0, one
 * scale per row; group 128, one per row and group (a checkpoint).  FMM_ERR_ARG
 * for another group. */
int fmm_q8_dequantize(int type, int64_t rows, int64_t cols, int group, const int8_t *dCodes, const float *dScales,
                      void *dOut, void *stream);

typedef struct {
  int64_t rows, cols;   /* rows >= 0, cols >= 1 */
  int32_t type;         /* FMM_F32, FMM_BF16 or FMM_F16: x, residual, h, gain and their gradients */
  float eps;            /* >= 0, finite */
} fmm_norm_desc;

/* The RMS norm with the residual's addition and an 8-bit output:
 *   h = x + residual (in fp32), rstd = (mean_j h_j^2 + eps)^-1/2, y = h rstd gain.
 * dH (may be NULL) receives h rounded to the type, dCodes / dScales the codes of
 * y, dRstd [rows] rstd, and dSaved / dSavedScales (both NULL or neither) the
 * checkpoint of h.  The codes are those of the row h gain (the factor rstd is
 * common to the row, and multiplies the scale only).  There and in the checkpoint
 * 2^-118 takes the place of 1e-12, but for rows and groups that are zero: where eps is
 * small, y is of order 1 however small h is.  (Squares are fp32: rows with magnitudes
 * past 1e17 may have rstd 0, and ones below 1e-18 with eps = 0 lose digits of it.)
 * dResidual and dGain may be NULL (0 and 1).  dH may be dX or dResidual
 * (FMM_ERR_UNSUPPORTED for rows of more than 32768 columns, which are read twice). */
int fmm_rmsnorm_q8(const fmm_norm_desc *desc, const void *dX, const void *dResidual, const void *dGain, void *dH,
                   int8_t *dCodes, float *dScales, int8_t *dSaved, float *dSavedScales, float *dRstd, void *stream);

/* Its gradient, from dY = d loss / d y (through the rounding to codes as if it
 * were the identity) and, where h was also used by others, dDh = d loss / d h:
 *   xh = h rstd, c = mean_j(dY_j gain_j xh_j),
 *   dDx = rstd (dY gain - xh c) + dDh   (the gradient of x and of the residual),
 *   dDgain_j = sum over rows of dY_j xh_j   (fp32 [cols]; NULL: not wanted).
 * h comes from dH, or, with dH NULL, from the checkpoint dSaved / dSavedScales.
 * dDh and dGain may be NULL.  dDx may be dDh, and must not overlap the other
 * inputs.  The sums over rows go through dScratch (16-byte aligned, at least
 * the size below; FMM_ERR_WORKSPACE) in a fixed order: repeated calls agree bit
 * for bit. */
int fmm_rmsnorm_q8_backward_scratch_size(const fmm_norm_desc *desc, size_t *bytes);
int fmm_rmsnorm_q8_backward(const fmm_norm_desc *desc, const void *dDy, const void *dDh, const void *dH,
                            const int8_t *dSaved, const float *dSavedScales, const float *dRstd, const void *dGain,
                            void *dDx, float *dDgain, void *dScratch, size_t scratch_bytes, void *stream);

typedef struct {
  /* tokens, output channels, input channels; each >= 0.  K <= 131071, M and N at
   * most 2^30, M N at most 2^37 (FMM_ERR_UNSUPPORTED) */
  int64_t M, N, K;
  int32_t type;      /* FMM_F32, FMM_BF16 or FMM_F16: the output, or its gradient and the gradients from it */
} fmm_q8_desc;

/* dC (M x N, `type`) = dSa[m] dSw[n] sum_k qa[m][k] qw[n][k] + dBias[n]: the codes
 * dA of the activations (M rows, a scale for each token) against the codes dW of
 * the weights (N rows, a scale for each output channel); dBias (fp32 [N]) may be
 * NULL.  The sum over k is exact. */
int fmm_q8_matmul(const fmm_q8_desc *desc, const int8_t *dA, const float *dSa, const int8_t *dW, const float *dSw,
                  const float *dBias, void *dC, void *stream);

/* The kernel that fmm_q8_matmul launches for these sizes on the current device, with
 * its tile, e.g. "matmul_kernel 256x256" ("ahead": the 128 tile with a longer ring).  A
 * static string; NULL for sizes that the call refuses. */
const char *fmm_q8_matmul_kernel(const fmm_q8_desc *desc);

/* The gradients of that product from dDy = d loss / d C (M x N, 16-byte aligned)
 * and the layer's 8-bit operands, the checkpoint of its input among them:
 *   dDx (M x K) = (dDy * sw) qw,  dDw (N x K) = (dDy * sa)^T qa,
 *   dDbias[n] = sum_m dDy[m][n] (fp32).
 * Any of the three may be NULL (not wanted), and the operands that only it needs
 * (dW, dSw; dA, dSa) with it.  The products run on the bf16 matrix cores with
 * fp32 sums.  FMM_BF16 rounds the values q s to bf16, its dY being exact; FMM_F16
 * carries dY s to 16 bits and FMM_F32 to 24, the codes being exact, at two and
 * three times the matrix work.  Where bf16 would round a finite value to infinity,
 * it is bf16's largest number (FMM_BF16), or parts of one sign that add up to it (the
 * others).  M and N at most 2^22, and M N, M K and N K at
 * most 2^34 (FMM_ERR_UNSUPPORTED).  dScratch: 256-byte aligned, at least the
 * size below (FMM_ERR_WORKSPACE). */
int fmm_q8_linear_backward_scratch_size(const fmm_q8_desc *desc, size_t *bytes);
int fmm_q8_linear_backward(const fmm_q8_desc *desc, const void *dDy, const int8_t *dA, const float *dSa,
                           const int8_t *dW, const float *dSw, void *dDx, void *dDw, float *dDbias, void *dScratch,
                           size_t scratch_bytes, void *stream);

/* The kernel of its products, as above, with the tiles of dDx and dDw, e.g.
 * "grad_kernel 64x64 128x128"; runs (may be NULL) receives how many runs the
 * contracted axis of each is split into.  want_dx, want_dw: which of them are wanted. */
const char *fmm_q8_linear_backward_kernel(const fmm_q8_desc *desc, int want_dx, int want_dw, int32_t runs[2]);

/* ---- linear layers on e4m3 blocks ------------------------------------------
 *
 * Linear layers on e4m3 operands as they are stored, by expert or not, with 8-bit
 * gradients; and the clipping of many gradients by their global norm.
 *
 * Codes.  A block is 128 columns of a row (activations, gradients) or 128 x 128 (a
 * weight); those past the last whole block are part of one.  Its scale is
 * 2^e, e the least integer >= -126 with a <= 448 2^e, a the largest magnitude of the
 * block's finite values (e = 0 where a = 0); the code of x is the e4m3 number nearest
 * x 2^-e, ties to even, and a code for NaN (0x7f, 0xff) for NaN and infinities.  Codes are one byte
 * each, rows padded with zeros to fmm_q8_pitch(cols); scales are the bytes e + 127
 * (E8M0), [rows][fmm_f8_scale_pitch(cols)] or, of a weight, [ceil(rows / 128)][...].  A
 * layer of experts has its weights and their scales one after the other.  Codes from
 * elsewhere may be used: scale bytes 1 to 254, zeros in the padding of codes, and
 * values (code times scale) that fp32 holds.
 *
 * Sums.  fp32 outputs: codes and scales as bf16 on the bf16 matrix cores, fp32 sums (values
 * below 2^-126 keep bf16's digits there).  16-bit outputs: the fp8 matrix cores, which
 * keep 13 bits below the largest product of each group of eight, and fp32 sums (on normal values off by 1.5e-5 of
 * the results' root mean square, whatever K is; rounding to fp16 is 2.1e-4, to bf16 1.7e-3).  Each result
 * is rounded once, to nearest even.
 *
 * Alignment: codes and scales 16 bytes, scratch 256, others their element
 * (FMM_ERR_ARG).  Asynchronous on `stream`; nothing is allocated on the device or
 * synchronized, so calls may be captured into a graph; repeated calls agree bit for bit. */

/* Bytes of one row of scales: ceil(cols / 128) rounded up to 16 (-1 if cols < 0). */
int64_t fmm_f8_scale_pitch(int64_t cols);

/* dCodes, dScales = the codes of the rows of dX (rows x cols, `type`), a scale for each
 * 128 columns; of `count` weights (rows x cols each), a scale for each 128 x 128.  At most
 * 2^30 rows, 2^22 columns and weights and, padded, 2^34 elements (FMM_ERR_UNSUPPORTED). */
int fmm_f8_quantize(int type, int64_t rows, int64_t cols, const void *dX, uint8_t *dCodes, uint8_t *dScales, void *stream);
int fmm_f8_quantize_weight(int type, int64_t count, int64_t rows, int64_t cols, const void *dX, uint8_t *dCodes,
                           uint8_t *dScales, void *stream);

/* dOut (count x rows x cols, `type`) = the values that codes stand for, a scale for each
 * 1 x 128 (block_rows 1) or 128 x 128 (block_rows 128; FMM_ERR_ARG for others). */
int fmm_f8_dequantize(int type, int64_t count, int64_t rows, int64_t cols, int block_rows, const uint8_t *dCodes,
                      const uint8_t *dScales, void *dOut, void *stream);

typedef struct {
  /* tokens, experts (>= 1), output channels, input channels.  Each at most 2^22, 4096
   * experts, and every matrix padded to 128 (rows for each expert) at most 2^34
   * elements (FMM_ERR_UNSUPPORTED) */
  int64_t rows, experts, N, K;
  int32_t type;      /* FMM_F32, FMM_BF16 or FMM_F16: the output, or its gradient and the gradients from it */
} fmm_f8_desc;

/* dC[m] (rows x N, `type`) = A[m] W[e]^T + dBias[e], e the expert of row m: the values of
 * the codes dA (rows x K) and dW (experts x N x K).  dOffsets (int32 [experts + 1], on the
 * device): expert e has the rows dOffsets[e] .. dOffsets[e + 1] - 1; NULL: there is
 * one expert, with every row.  Rows of no expert are left as they were.  Offsets count as raised to the
 * largest before them and cut to 0 .. rows, so whatever they hold nothing outside
 * the matrices is touched.  dBias (fp32 [experts][N]) may be NULL. */
int fmm_f8_matmul(const fmm_f8_desc *desc, const uint8_t *dA, const uint8_t *dSa, const uint8_t *dW, const uint8_t *dSw,
                  const int32_t *dOffsets, const float *dBias, void *dC, void *stream);

/* The kernel that fmm_f8_matmul launches for these sizes on the current device, with its
 * tile.  A static string; NULL for sizes that the call refuses. */
const char *fmm_f8_matmul_kernel(const fmm_f8_desc *desc);

/* The gradients of that product from dDy = d loss / d C (rows x N) and the operands of
 * the forward pass, on 8-bit operands again:
 *   dDx[m] (rows x K) = Q(dDy)[m] W[e], codes of 128 columns of a row of dDy;
 *   dDw[e] (experts x N x K) = Q(dDy)^T Q(A) over the expert's rows, codes of 128 rows of a
 *   column counted from the expert's first row, of dDy and of the values of dA;
 *   dDbias[e] (fp32, experts x N) = sums of dDy's columns over the expert's rows.
 * Experts without rows get zeros.  Any of the three may be NULL (not wanted), and the
 * operands that only it needs with it.  dScratch: at least the size below
 * (FMM_ERR_WORKSPACE). */
int fmm_f8_linear_backward_scratch_size(const fmm_f8_desc *desc, size_t *bytes);
int fmm_f8_linear_backward(const fmm_f8_desc *desc, const void *dDy, const uint8_t *dA, const uint8_t *dSa,
                           const uint8_t *dW, const uint8_t *dSw, const int32_t *dOffsets, void *dDx, void *dDw,
                           float *dDbias, void *dScratch, size_t scratch_bytes, void *stream);

/* The kernel of its products, with the tiles of dDx and dDw; want_dx, want_dw: which are wanted. */
const char *fmm_f8_linear_backward_kernel(const fmm_f8_desc *desc, int want_dx, int want_dw);

/* Clipping by the global norm of `count` tensors (host arrays: element type, number of elements
 * >= 0, device addresses of each, read before the call returns):
 *   dNorm (fp32, one) = sqrt(sum of the squares of all elements), summed in binary64,
 *   dOut[i] = dIn[i] min(1, most / (norm + 1e-6)).
 * most >= 0.  dOut[i] may be dIn[i]; else outputs must not overlap inputs or one another.  A
 * norm of infinity gives the factor 0, whatever most is (and NaN where the element is infinite itself), NaN gives
 * NaN everywhere.  A finite norm past fp32's largest number is infinity in dNorm alone.  At most 122880 tensors
 * and 2^42 elements (FMM_ERR_UNSUPPORTED).  dScratch: 8-byte aligned, at least the size below
 * (FMM_ERR_WORKSPACE). */
size_t fmm_clip_scratch_size(void);
int fmm_clip(const int32_t *types, const int64_t *sizes, void *const *dIn, void *const *dOut, int64_t count, float most,
             float *dNorm, void *dScratch, size_t scratch_bytes, void *stream);

/* ---- misc ---------------------------------------------------------------- */

const char *fmm_status_string(int status);
const char *fmm_last_error_detail(void);
/* FMM_OK if device `device` is a gfx950, FMM_ERR_DEVICE if not, FMM_ERR_HIP
 * if it cannot be queried. */
int fmm_device_check(int device);

#ifdef __cplusplus
}
#endif

#endif /* FMM8_H */
