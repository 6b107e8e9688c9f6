/*
 * optima.h -- C ABI of the OPTIMA weight-update hot path on AMD MI355X (gfx950).
 *
 * OPTIMA (arXiv 2512.13886) rewrites the layer-wise weight reconstruction that
 * follows mask selection as one quadratic program per output column (Eq. (3)-(6)):
 *
 *     minimise  (w_j - w0_j)^T H (w_j - w0_j)   subject to  w_j[i] = 0 for every
 *     pruned entry i (mask[j][i] == 0),
 *
 * with one Hessian H = X^T X shared by all columns of the layer. The library
 * computes H from calibration tokens, damps it, estimates its spectral norm and
 * solves all column QPs together with a batched restarted accelerated
 * primal-dual hybrid gradient (rAPDHG) method (Section 3.3-3.4, Algorithm 1).
 *
 * Conventions shared by every call
 *   - Matrices are row-major. The weight and mask are stored [n_cols][d]: row j
 *     holds the QP of output column j (the PyTorch Linear layout; the paper
 *     writes W as d_in x d_out, Eq. (3)).
 *   - Mask bytes: 1 keeps the weight, 0 prunes it (Eq. (1)).
 *   - Every pointer argument is a device pointer owned by the caller unless
 *     stated otherwise; the library keeps no pointer after a call returns and
 *     allocates no device memory. Work buffers come from the caller through a
 *     `ws` argument sized by the matching *_workspace_bytes query.
 *   - All calls are ordered on `stream` (NULL = the default stream).
 *   - Errors are returned before any kernel is launched when they come from
 *     argument validation. HIP failures map to OPTIMA_E_HIP.
 */
#ifndef OPTIMA_H
#define OPTIMA_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int optima_status;

#define OPTIMA_OK 0
#define OPTIMA_E_INVAL (-1)       /* NULL pointer, bad size, misaligned or aliased buffer */
#define OPTIMA_E_HIP (-2)         /* a HIP runtime call or kernel launch failed */
#define OPTIMA_E_NONFINITE (-3)   /* NaN or Inf in H, W0 or the spectral norm */
#define OPTIMA_E_WORKSPACE (-4)   /* ws NULL or smaller than the size query returned */
#define OPTIMA_E_UNSUPPORTED (-5) /* unsupported dtype, or the device is not gfx950 */

#define OPTIMA_DTYPE_F32 0
#define OPTIMA_DTYPE_BF16 1
#define OPTIMA_DTYPE_F64 2
#define OPTIMA_DTYPE_I8 3 /* 8-bit codes with scales (optima_rms_norm, optima_w4_*) */
#define OPTIMA_DTYPE_MX4 4 /* microscaled 4-bit codes with scales (optima_mx4_linear) */

/* Arithmetic of the solver's per-iteration H-products (optima_solver_opts).
 * FP32: v_mfma_f32_16x16x4_f32, fp32 products and sums.
 * BF16X3: every fp32 operand v is split into bf16 planes hi = rne(v),
 *   lo = rne(v - hi), and a*b is formed as hi*hi + hi*lo + lo*hi on
 *   v_mfma_f32_16x16x32_bf16 with fp32 accumulation; the dropped terms are
 *   below 3 * 2^-16 |a b| per product. The precision applies to every
 *   product of a solve, the setup products H w0 and H x0 included (with at
 *   most 8 active columns the iteration products stream H once per
 *   iteration through a 16-column MFMA kernel, with the same products). BF16X3 is
 *   the default: on the 4096-wide outlier layer its
 *   solutions differ from FP32's by under 1e-5 relative (Frobenius) and it
 *   runs the iteration about 2.5x faster. */
#define OPTIMA_PREC_FP32 0
#define OPTIMA_PREC_BF16X3 1

/* Solve method (optima_solver_opts.method).
 * RAPDHG: the paper's batched restarted accelerated method on the constrained
 *   form, Eq. (6) (described with optima_qp_solve_batched below).
 * CG: the unconstrained form of Eq. (7)-(11). With the pruned entries fixed
 *   at zero the optimum solves H_KK x_K = (H w0)_K for every column, which
 *   conjugate gradients reach without restarts or a step size: from
 *   x = sel(mask, w0, +0), r = P (H w0 - H x), p = r, each iteration forms
 *   q = H p (one batched product), alpha = r.r / p.q_K, x += alpha p,
 *   r -= alpha q_K, beta = r'.r' / r.r, p = r' + beta p, with x, r and p exactly
 *   zero off K. Columns are tested every check_every iterations with the same
 *   rule as RAPDHG, evaluated from the recurrence residual (r_d = 2 ||r_K||,
 *   gap = 2 |x.r|); lambda_max, the beta_* constants, step_safety and
 *   restarts are unused (lambda_max may be NULL). */
#define OPTIMA_METHOD_RAPDHG 0
#define OPTIMA_METHOD_CG 1

/* Human-readable name of a status code (static string, never NULL). */
const char* optima_status_string(optima_status status);

/* Library ABI version (increments on any signature change). */
int optima_abi_version(void);

/* ---------------------------------------------------------------------------
 * Hessian accumulation -- Section 3.4 "Hessian calculation", Algorithm 1.
 *
 * H[d][d] (fp32) = (accumulate ? H : 0) + X^T X, where X[n_tok][d] holds n_tok
 * calibration tokens (one or many 2048-token sequences; the paper sums
 * y_i^T y_i sequence by sequence, which gives the same matrix as stacking).
 * X is fp32 (dtype OPTIMA_DTYPE_F32) or bf16 (OPTIMA_DTYPE_BF16); products are
 * formed exactly and summed in fp32. Both triangles of H are written and the
 * result is exactly symmetric; with accumulate = 1 the lower triangle of the
 * incoming H is read and taken as the whole matrix. n_tok = 0 leaves H as it is
 * (accumulate = 1) or zeroes it. X must be 16-byte aligned (OPTIMA_E_INVAL
 * otherwise); H may alias nothing else. ws must hold
 * optima_hessian_workspace_bytes(n_tok, d, dtype) bytes: split-K partial sums,
 * plus a token-slab transpose buffer unless X is bf16 with d % 256 == 0 (then
 * token rows are read in place and only a 64-row tail buffer is needed). The size
 * for more tokens is never smaller.
 * ------------------------------------------------------------------------- */
size_t optima_hessian_workspace_bytes(int64_t n_tok, int64_t d, int dtype);
optima_status optima_hessian_accumulate(const void* X, int dtype, int64_t n_tok,
                                        int64_t d, float* H, int accumulate,
                                        void* ws, size_t ws_bytes,
                                        hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Damping. The paper's H = X^T X is only positive semi-definite (Eq. (6));
 * this call adds lambda * I with lambda = rel_damp * trace(H) / d, which makes
 * every column QP strictly convex so its optimum (Eq. (10)-(11)) is unique.
 * The trace is summed in fp64 on the device. lambda_out (device, one float,
 * required) receives lambda; if the trace is not finite, H is left unchanged
 * and lambda_out receives NaN (the solve then reports OPTIMA_E_NONFINITE).
 * ------------------------------------------------------------------------- */
optima_status optima_hessian_damp(float* H, int64_t d, float rel_damp,
                                  float* lambda_out, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Shared diagonal preconditioning (Jacobi). Not in the paper; a reading usual
 * for PDLP-family first-order solvers. One scaling serves all columns, so the
 * batching of Algorithm 1 is unchanged.
 *
 * H[d][d] fp32 (symmetric, damped) is replaced in place by D H D with
 * D_i = H_ii^(-1/2) (computed in fp64, rounded to fp32; 1 where H_ii is not
 * positive and finite), and scale_out[d] (device) receives D. The factor of
 * entry (i, j) is the fp32 product D_i D_j, so exact symmetry is kept. In the
 * coordinates y = D^-1 w every column QP of Eq. (6) keeps its zero pattern and
 * objective values, and its optimum is D^-1 w*. The outlier channels of
 * transformer layers make H badly scaled (condition numbers of 10^3 - 10^4);
 * D H D is well conditioned and the solvers need far fewer iterations.
 * Workflow: damp, optima_hessian_jacobi, optima_spectral_norm on the scaled H,
 * then optima_qp_solve_batched with opts.col_scale = scale_out: the solver
 * iterates on the scaled problem, tests termination with the gradient in the
 * original coordinates and writes W_out in the original coordinates.
 * ------------------------------------------------------------------------- */
optima_status optima_hessian_jacobi(float* H, int64_t d, float* scale_out,
                                    hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Spectral norm of H for the solver's step size (Section 3.3: the first-order
 * method's bottleneck is products with H; its step needs ||Q|| = 2 lambda_max).
 * H must be symmetric positive semi-definite (X^T X + lambda I is), [d][d]
 * fp32, 4-byte aligned (16-byte alignment and d % 4 == 0 enable vector loads).
 *
 * V0: [block][d] fp32 device array of start vectors (row a is vector a), not
 * modified; 1 <= block <= OPTIMA_SPECTRAL_MAX_BLOCK.
 *   block == 1: power iteration. Iteration i forms y = H v with v of unit
 *     length, rho_i = v^T y and v <- y / ||y||.
 *   block >= 2: subspace (orthogonal) iteration with Rayleigh-Ritz.
 *     Iteration i multiplies an orthonormal basis Q of the current block by
 *     H (Y = H Q, one pass over H) and takes rho_i = the largest Ritz value
 *     of span(Q), i.e. the largest eigenvalue of Q^T H Q; the next basis spans
 *     Y (Cholesky QR in fp64). Convergence goes as lambda_{block+1} /
 *     lambda_1 instead of lambda_2 / lambda_1, so Hessians whose top
 *     eigenvalues cluster (outlier channels) need a handful of passes. The
 *     b x b eigenvalue is found by repeated squaring, within 1e-8 relative.
 *     Directions that become numerically dependent (Cholesky pivot below
 *     1e-14 of the diagonal) are dropped.
 * Both stop once |rho_i - rho_{i-1}| <= tol * rho_i, or after max_iters
 * iterations. lambda_max (device, one float) receives the last rho (NaN if H
 * holds NaN/Inf and block >= 2); iters (device int32, may be NULL) the
 * iteration count. Blocking: the call synchronises `stream` a few times to
 * test convergence. ws: optima_spectral_norm_workspace_bytes(d, block) bytes.
 * ------------------------------------------------------------------------- */
#define OPTIMA_SPECTRAL_MAX_BLOCK 16
size_t optima_spectral_norm_workspace_bytes(int64_t d, int block);
optima_status optima_spectral_norm(const float* H, int64_t d, const float* V0,
                                   int block, int max_iters, float tol,
                                   void* ws, size_t ws_bytes, float* lambda_max,
                                   int32_t* iters, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * optima_spectral_norm for callers that cannot allocate memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, iterations, results and blocking behaviour as
 * optima_spectral_norm, without `ws`: the work buffer is a fixed array of
 * OPTIMA_SPECTRAL_NOALLOC_SCRATCH_BYTES inside the library, one copy per
 * device, held from the library's load until the process ends. It covers
 * every block size for d <= OPTIMA_SPECTRAL_NOALLOC_MAX_DIM; a larger d
 * returns OPTIMA_E_WORKSPACE before any launch. The call allocates nothing
 * (no device memory, no pinned host memory): its convergence polls copy into
 * host stack memory and synchronise `stream`. The first call on a device
 * looks up the array's device address once (hipGetSymbolAddress).
 * Every call on a device shares that device's array and leaves its contents
 * there: calls that overlap on one device (two streams, or two host threads)
 * race on it and must be serialised by the caller. Calls on different
 * devices are independent.
 * ------------------------------------------------------------------------- */
#define OPTIMA_SPECTRAL_NOALLOC_MAX_DIM 16384
#define OPTIMA_SPECTRAL_NOALLOC_SCRATCH_BYTES (8454144)
optima_status optima_spectral_norm_noalloc(const float* H, int64_t d, const float* V0,
                                           int block, int max_iters, float tol,
                                           float* lambda_max, int32_t* iters,
                                           hipStream_t stream);

/* ---------------------------------------------------------------------------
 * The same lambda_max (the step size of Section 3.3's first-order solver) by
 * the symmetric Lanczos process with full reorthogonalisation. Step j builds
 * q_j of an orthonormal basis of the Krylov space span{v0, H v0, ...,
 * H^(j-1) v0} from one product with H:
 *   w = H q_j, alpha_j = q_j^T w, w <- w - alpha_j q_j - beta_(j-1) q_(j-1),
 *   w <- w - Q (Q^T w), beta_j = ||w||, q_(j+1) = w / beta_j,
 * and rho_j = the largest eigenvalue of the j x j tridiagonal matrix
 * T = tridiag(beta; alpha; beta) = Q^T H Q (the largest Ritz value of the
 * Krylov space; never above lambda_max(H), non-decreasing in j). Its
 * convergence goes as a Chebyshev polynomial of the step count, so spectra
 * whose top has no gap (near-isotropic inputs, or H after diagonal scaling)
 * need far fewer passes over H than the subspace iteration of
 * optima_spectral_norm. The basis is fp32, all sums fp64; the eigenvalue of
 * T comes from Sturm-count bisection in fp64 (relative width 1e-15).
 *
 * H: [d][d] fp32, symmetric, 4-byte aligned (16-byte alignment and d % 4 ==
 * 0 enable vector loads). v0: [d] fp32 device start vector, not modified.
 * It stops once |rho_j - rho_(j-1)| <= tol * rho_j, once beta_j <= 1e-6 *
 * rho_j (the Krylov space is invariant: rho_j is an eigenvalue), or after
 * min(max_steps, d) steps, 1 <= max_steps <= OPTIMA_LANCZOS_MAX_STEPS.
 * Without a gap at the top of the spectrum the Ritz value rises by small
 * amounts long before it converges: there tol = 1e-7 stops within about
 * 1e-6 of lambda_max where 1e-6 can stop 3e-4 short.
 * lambda_max (device, one float) receives the last rho (0 for a zero v0, NaN
 * if H or v0 holds NaN/Inf); steps (device int32, may be NULL) the step
 * count. Blocking: the call synchronises `stream` every 8 steps to test
 * convergence. ws: optima_spectral_lanczos_workspace_bytes(d, max_steps)
 * bytes (about max_steps * d * 4 for the basis).
 * ------------------------------------------------------------------------- */
#define OPTIMA_LANCZOS_MAX_STEPS 256
size_t optima_spectral_lanczos_workspace_bytes(int64_t d, int max_steps);
optima_status optima_spectral_lanczos(const float* H, int64_t d, const float* v0,
                                      int max_steps, float tol, void* ws,
                                      size_t ws_bytes, float* lambda_max,
                                      int32_t* steps, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Wanda mask selection -- the mask M that the weight update starts from
 * (Algorithm 1 takes it from a selector; the configurations use the Wanda
 * saliency cited in Section 2, with the 2:4 pattern of Section 4).
 *
 * W0: [n_cols][d] fp32 (row j = column QP j), 4-byte aligned. col_sq: the
 * squared input norms c[i] = sum_t X[t][i]^2, element i at col_sq[i * stride],
 * fp32 (OPTIMA_DTYPE_F32) or fp64 (OPTIMA_DTYPE_F64); e.g. the diagonal of the
 * undamped Hessian is H with stride d + 1. mask: [n_cols][d] uint8 output
 * (1 keeps), 4-byte aligned, overlapping neither input.
 * score[j][i] = W0[j][i]^2 * c[i] in fp64 (the square of the saliency
 * |W0[j][i]| sqrt(c[i]), same order; exact square, one rounded product).
 * pattern OPTIMA_MASK_UNSTRUCTURED keeps the d - floor(sparsity * d) highest
 * scores of every row (0 <= sparsity <= 1); OPTIMA_MASK_2TO4 keeps the two
 * highest of every group [4g, 4g + 4) of a row (d % 4 == 0). Equal scores go
 * to the lower index; NaN scores rank below all others; -0 equals +0. The
 * result is a pure function of the input values: bit-exact against any IEEE
 * implementation of the same rule. Asynchronous on `stream`.
 * ------------------------------------------------------------------------- */
#define OPTIMA_MASK_UNSTRUCTURED 0
#define OPTIMA_MASK_2TO4 1
optima_status optima_wanda_mask(const float* W0, int64_t n_cols, int64_t d,
                                const void* col_sq, int col_sq_dtype,
                                int64_t col_sq_stride, int pattern,
                                double sparsity, uint8_t* mask,
                                hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Layer forward pass -- Algorithm 1: the layer outputs y = L(x) on the
 * calibration tokens, and the activations X <- L(X) handed to the next layer
 * once L is pruned. Also the squared output error between two weight sets.
 * The layer-wise error of Section 4 (MSE against the dense layer's outputs,
 * OPTIMA's over another method's) is a ratio of two such errors.
 *
 * Z[n_tok][d_out] = X W^T with X [n_tok][d_in] bf16 (row-major, 16-byte
 * aligned, d_in a multiple of 64) and W [d_out][d_in] fp32 rounded to bf16
 * on the device (round to nearest even), products exact, sums in fp32.
 * d_out must be a multiple of 4.
 * Y (nullable): act(Z), act OPTIMA_ACT_NONE or OPTIMA_ACT_SILU (z / (1 +
 *   e^-z) in fp32), stored as y_dtype OPTIMA_DTYPE_BF16 (round to nearest
 *   even, 8-byte aligned) or OPTIMA_DTYPE_F32 (16-byte aligned).
 * err_out (nullable, device double): receives the sum over all outputs of
 *   (Z - Y_ref)^2, accumulated in fp64 in a fixed order; Y_ref (fp32
 *   [n_tok][d_out], 16-byte aligned) is then required when n_tok > 0: a
 *   reference Z, e.g. the dense layer's from an earlier call with act NONE
 *   and fp32 Y. Y_ref without err_out, or neither Y nor err_out, is
 *   OPTIMA_E_INVAL. With n_tok = 0, X, Y and Y_ref are not read and
 *   err_out receives 0.
 * ws: optima_linear_forward_workspace_bytes(n_tok, d_in, d_out) bytes
 * (the bf16 weights and per-tile partial sums). The call synchronises the
 * stream once. It returns OPTIMA_E_NONFINITE if W holds a NaN or Inf.
 * ------------------------------------------------------------------------- */
#define OPTIMA_ACT_NONE 0
#define OPTIMA_ACT_SILU 1
size_t optima_linear_forward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_out);
optima_status optima_linear_forward(const void* X, int64_t n_tok, int64_t d_in,
                                    const float* W, int64_t d_out, int act, void* Y,
                                    int y_dtype, const float* Y_ref, double* err_out,
                                    void* ws, size_t ws_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Batched column-QP solve -- Eq. (6), Algorithm 1, Section 3.3-3.4.
 *
 * For every row j < n_cols of W0 (fp32 values) and mask (uint8), writes
 *   W_out[j] = argmin (w - W0[j])^T H (w - W0[j])  s.t. w[i] = +0.0 where
 *              mask[j][i] == 0,
 * reached with the batched rAPDHG iteration. The pruned entries are fixed
 * through equal lower and upper bounds (Section 3.4), i.e. the projection
 * keeps them at exactly +0.0 (bit pattern 0). Per column j, with
 * alpha_k = 2/(k+2), eta_k = (k+1)/(2L), L = 2 lambda_max (1 + step_safety):
 *   x_md = (1-alpha) x_ag + alpha x;  g = 2 H (x_md - w0);
 *   x = sel(mask, x - eta g, +0);     x_ag = (1-alpha) x_ag + alpha x,
 * starting from x = x_ag = sel(mask, w0, +0). Every check_every iterations
 * (and at max_iters) x and x_ag are scored by r_d = ||g restricted to kept
 * entries||, gap = |z^T g|, KKT = sqrt(r_d^2 + gap^2); the lower-KKT one is the
 * candidate (ties: x_ag). A column terminates (unless fixed_iters) when
 * r_d <= eps_abs + eps_rel ||2 H w0|| and gap <= eps_abs + eps_rel (|P| + |D|)
 * with P = f(cand), D = w0^T H w0 - cand^T H cand (Appendix D tolerances). It
 * restarts to the candidate on KKT decay by beta_sufficient, on decay by
 * beta_necessary without progress since the last check, or when the iterations
 * since the last restart reach beta_artificial times the total; a restart is
 * accepted only if it does not raise the objective above the previous restart
 * point's. Columns are fully independent: the result for a column does not
 * depend on the others in the batch (Algorithm 1 batching).
 *
 * H: [d][d] fp32, symmetric, 16-byte aligned. lambda_max: device float (from
 * optima_spectral_norm, optima_spectral_lanczos or the caller). W_out: [n_cols][d] fp32, must not
 * overlap W0. stats (host struct of device arrays, may be NULL; each array may
 * be NULL): per column iterations run, accepted restarts, convergence flag,
 * objective at the start point sel(mask, w0, 0), objective and KKT of W_out
 * (computed on the device from the maintained products). info (host, may be
 * NULL) receives run totals (for CG the timed window of each run of
 * iterations also covers their CG update kernels). ws:
 * optima_qp_workspace_bytes(d, n_cols) bytes.
 * Blocking: the call synchronises `stream` once per check to learn how many
 * columns are still active (RAPDHG with fixed_iters, where all are, once
 * every 32 checks and at the end). Non-convergence is not an error; it is
 * reported per column. Returns OPTIMA_E_NONFINITE if H or W0 holds NaN/Inf,
 * lambda_max is not a positive finite number, or opts.col_scale holds an
 * entry that is not positive and finite.
 * ------------------------------------------------------------------------- */
typedef struct {
  int64_t max_iters;      /* >= 0; the paper uses 100000 (Table 8) */
  int32_t check_every;    /* >= 1; default 64 */
  int32_t fixed_iters;    /* 1: run exactly max_iters, checks only restart */
  float eps_rel;          /* default 0.01 (Table 8) */
  float eps_abs;          /* default 0.01 (Table 8) */
  float beta_sufficient;  /* default 0.2 */
  float beta_necessary;   /* default 0.8 */
  float beta_artificial;  /* default 0.36 */
  float step_safety;      /* default 1e-3 */
  int32_t restarts;       /* 0 disables restarts; default 1 */
  int32_t precision;      /* OPTIMA_PREC_BF16X3 (default) or OPTIMA_PREC_FP32 */
  int32_t method;         /* OPTIMA_METHOD_RAPDHG (default) or OPTIMA_METHOD_CG */
  const float* col_scale; /* NULL (default), or the [d] device diagonal D of a
                             preconditioned H = D H0 D (optima_hessian_jacobi);
                             see "Shared diagonal preconditioning" */
  int32_t sparse;         /* 1 (default): when precision is BF16X3, method is
                             RAPDHG and no mask row keeps more than 2 entries
                             of any group of 4 consecutive columns (a 2:4 mask,
                             Section 4), the iteration products take x
                             2:4-compressed and multiply on the sparse MFMA
                             (v_smfmac_f32_16x16x64_bf16), skipping the pruned
                             entries; the same products are formed, summed in
                             another order. 0: dense products always. */
  int32_t cooperative;    /* 1 (default): when at most 8 columns are still active
                             and d <= 4096, the iterations between two checks
                             run as one cooperative launch (hipLaunchCooperativeKernel)
                             that keeps H's split planes in registers and meets
                             at a grid barrier between iterations; the same
                             products and updates, bit for bit, as one launch
                             per iteration. 0: one launch per iteration (for
                             callers whose streams cannot take cooperative
                             launches). Falls back to per-iteration launches
                             by itself when the device refuses them. Dense
                             solves with d <= 256 run those iterations in one
                             ordinary launch whatever this says and for any
                             number of columns. */
} optima_solver_opts;

typedef struct {
  int32_t* iters;
  int32_t* restarts;
  uint8_t* converged;
  float* f_initial;
  float* f_final;
  float* kkt_final;
} optima_solve_stats;

typedef struct {
  int64_t iterations;         /* iterations run by the longest-running column */
  int64_t gemm_calls;         /* H-product launches (including the two at setup) */
  int64_t row_products;       /* sum over those launches of the columns multiplied */
  int64_t checks;             /* check passes */
  int64_t timed_launches;     /* H-product launches between checks (the iteration loop) */
  int64_t timed_row_products; /* columns multiplied by those launches */
  double timed_product_ms;    /* their device time, from HIP events recorded on `stream`
                                 around each run of back-to-back product launches */
  int64_t sparse_products;    /* 1 if the iteration products ran 2:4-sparse (opts.sparse) */
  int64_t few_launches;       /* the timed launches that ran the few-column kernel (at most 8
                                 active columns with split planes: H streamed once per launch;
                                 not the one-launch blocks of dense solves with d <= 256) */
  int64_t few_row_products;   /* columns multiplied by those launches */
  double few_product_ms;      /* their device time (included in timed_product_ms) */
  int64_t persistent_launches; /* blocks of few-column iterations (the iterations between two
                                  checks) that ran as one cooperative launch keeping H's planes
                                  in registers (d <= 4096); each counts all of its iterations in
                                  few_launches */
} optima_solve_info;

void optima_solver_opts_default(optima_solver_opts* opts);
size_t optima_qp_workspace_bytes(int64_t d, int64_t n_cols);
optima_status optima_qp_solve_batched(const float* H, int64_t d,
                                      const float* lambda_max, const float* W0,
                                      const uint8_t* mask, int64_t n_cols,
                                      const optima_solver_opts* opts, void* ws,
                                      size_t ws_bytes, float* W_out,
                                      const optima_solve_stats* stats,
                                      optima_solve_info* info,
                                      hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Feed-forward half of a decoder block.
 *
 * The inputs of the gate and up projections are the RMS norm of the residual
 * stream, those of the down projection the gated product of the two: the X whose
 * Hessians the calls above form (Algorithm 1; the paper prunes every linear layer
 * of a block). The calls below compute both for calibration, their gradients for
 * recovery steps under the masks, and their few-token forms with 4-bit weights
 * for serving the pruned block.
 *
 * Conventions of these calls: token matrices have a row pitch in elements (ldx,
 * ...; at least the row's length) and need only the alignment of an element;
 * weights are contiguous. All are asynchronous on `stream`, record no memset and
 * synchronise nothing, so that they can be captured in a HIP graph. NaN and
 * infinities go through the arithmetic. Every sum is fp32 or wider (whole numbers:
 * int32) and is taken in an order that depends on the sizes and types only. With no tokens
 * nothing is read of token matrices. Outputs share elements with neither inputs nor each
 * other except where stated; rows of one pitch may lie between each other's (halves of one
 * buffer's columns), of different pitches the whole extents count.
 * ------------------------------------------------------------------------- */

/* RMS norm with the residual's addition.
 *   s = x + r (r = 0 where R is NULL), y = s * weight / sqrt(mean(s^2) + eps)
 * over rows of d <= OPTIMA_NORM_MAX_DIM values (larger: OPTIMA_E_UNSUPPORTED).
 * X, R and S are of `dtype` (F32 or BF16), weight of w_dtype. S (nullable)
 * receives s rounded to dtype; the norm is taken of the fp32 s, whose squares overflow (y = 0)
 * where |s| passes about 1e19. S may be X or R
 * themselves (same pointer and pitch), and so may Y if it has their type.
 * Y: y_dtype F32, BF16, or I8: codes q = rne(y * (1 / scale)) within +-127 with
 *   scale = max |y| / 127 (0 below the smallest normal number) over each group of `group` consecutive values (32, 64 or
 *   128; the last group of a row may be shorter) or over the row (group = 0).
 *   scales[n_tok][ceil(d / group)] (one a row for group = 0) is required then. A
 *   group with scale 0 has codes 0; one with a NaN or infinity has codes 0 and a NaN
 *   or infinite scale. For other types scales is NULL and group 0.
 * eps > 0. */
#define OPTIMA_NORM_MAX_DIM 16384
optima_status optima_rms_norm(const void* X, int64_t ldx, const void* R, int64_t ldr, int dtype,
                              int64_t n_tok, int64_t d, const void* weight, int w_dtype,
                              float eps, void* S, int64_t lds, void* Y, int64_t ldy, int y_dtype,
                              float* scales, int64_t group, hipStream_t stream);

/* Gradient of the RMS norm at S, the sum that the forward call stored. With
 * rstd = 1 / sqrt(mean(s^2) + eps), xh = s rstd and p = weight * dy:
 *   dX = dS + rstd (p - xh mean(p xh)),   dweight = sum over tokens of dy xh.
 * dS (nullable) is the gradient that reaches s from the residual stream; dX is the
 * gradient of both x and r, and may be dY or dS themselves. S, dY, dS and dX are of
 * `dtype`. dweight (nullable): fp32 [d], added to what it holds with accumulate = 1.
 * ws: optima_rms_norm_backward_workspace_bytes(n_tok, d) bytes, unless dweight is
 * NULL. */
size_t optima_rms_norm_backward_workspace_bytes(int64_t n_tok, int64_t d);
optima_status optima_rms_norm_backward(const void* S, int64_t lds, const void* weight, int w_dtype,
                                       const void* dY, int64_t lddy, const void* dS, int64_t ldds,
                                       int dtype, int64_t n_tok, int64_t d, float eps, void* dX,
                                       int64_t lddx, float* dweight, int accumulate, void* ws,
                                       size_t ws_bytes, hipStream_t stream);

/* Gated feed-forward product.
 *   G = X Wg^T, U = X Wu^T, H = act(G) * U element by element
 * X: [n_tok][d_in] bf16, any d_in >= 1; Wg, Wu: [d_ff][d_in] bf16 (16-byte aligned
 * where d_in % 8 == 0). H: h_dtype BF16 or F32. G and U (nullable): bf16
 * [n_tok][d_ff], what the gradient takes; H is formed of the unrounded sums.
 * act: OPTIMA_ACT_SILU or OPTIMA_ACT_NONE. The 64 x 64 tiles of [n_tok][max(d_in, d_ff)]
 * and twice those of [d_ff][d_in] stay below 2^23 together, here and in the gradient.
 * ws: optima_gated_forward_workspace_bytes(n_tok, d_in, d_ff) bytes (0 for few tokens,
 * never less for more): copies of operands whose rows do not suit wide loads, and parts
 * of split sums. */
size_t optima_gated_forward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_ff);
optima_status optima_gated_forward(const void* X, int64_t ldx, int64_t n_tok, int64_t d_in,
                                   const void* Wg, const void* Wu, int64_t d_ff, int act, void* H,
                                   int64_t ldh, int h_dtype, void* G, int64_t ldg, void* U,
                                   int64_t ldu, void* ws, size_t ws_bytes, hipStream_t stream);

/* Gradient of the gated product.
 *   dU = dH * act(G), dG = dH * U * act'(G)
 *   dX = dG Wg + dU Wu,  dWg = mask_g * (dG^T X),  dWu = mask_u * (dU^T X)
 * The products take dG and dU in two bf16 parts, within 2^-16 of each value, and round once, to
 * the type of the output.
 * X, Wg, Wu, act as in the forward call, G and U what it stored, dH bf16. dX
 * (nullable): dx_dtype BF16 or F32. dWg and dWu (both or neither): [d_ff][d_in] of
 * dw_dtype, added to what they hold with accumulate = 1. mask_g, mask_u (each
 * nullable): uint8 [d_ff][d_in]; where 0, the weight is pruned and its gradient is
 * exactly 0, so that a step along it keeps the pattern.
 * ws: optima_gated_backward_workspace_bytes(n_tok, d_in, d_ff) bytes. */
size_t optima_gated_backward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_ff);
optima_status optima_gated_backward(const void* X, int64_t ldx, int64_t n_tok, int64_t d_in,
                                    const void* Wg, const void* Wu, int64_t d_ff, int act,
                                    const void* G, int64_t ldg, const void* U, int64_t ldu,
                                    const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                    int dx_dtype, void* dWg, void* dWu, int dw_dtype,
                                    const uint8_t* mask_g, const uint8_t* mask_u, int accumulate,
                                    void* ws, size_t ws_bytes, hipStream_t stream);

/* 4-bit weights with group scales.
 * W: [n][d] F32 or BF16. Groups of `group` (32, 64 or 128) consecutive values of a
 * row have scale = bf16(max |w| * (1 / 7)), the product and 1 / 7 in fp32, and codes
 * clamp(rne(w / scale), -7, 7): a zero weight, as every pruned one is, stays exactly
 * zero. A group with a NaN or infinity has codes 0 and a NaN or infinite scale. The chunks
 * (below), n ceil(d / 128), are at most 2^28 - 16.
 * Q: [n][optima_w4_row_bytes(d)], 16-byte aligned. A chunk of 128 codes takes 64
 *   bytes: dword j of its 16-byte block b holds codes 32 j + 8 b .. + 7, the even ones
 *   in nibbles 0..3 and the odd ones in nibbles 4..7, each as code + 8; rows are
 *   padded to whole chunks with zero codes.
 * scales: bf16 [n][ceil(d / group)]. */
size_t optima_w4_row_bytes(int64_t d);
optima_status optima_w4_pack(const void* W, int dtype, int64_t n, int64_t d, int64_t group,
                             void* Q, void* scales, hipStream_t stream);

/* Y = X deq(Q)^T for the tokens of decoding steps: the weights are streamed once for
 * every 64 tokens.
 * X: [n_tok][d] of x_dtype BF16, or I8 with x_scales: fp32 [n_tok][ceil(d / x_group)]
 * with x_group = group, or one a token with x_group = 0 (as optima_rms_norm writes
 * them). Y: [n_tok][d_out] BF16 or F32. 8-bit codes are multiplied exactly within a
 * group; products of 16-bit tokens with codes are exact and summed in fp32. A zero weight adds
 * exactly nothing, except to an infinite or NaN token (NaN).
 * ws: optima_w4_workspace_bytes(n_tok, d, d_out, n_mats) bytes, with n_mats 1 here and 2
 * for the gated product: 0 up to 16 tokens, and never less for more tokens. */
size_t optima_w4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out, int n_mats);
optima_status optima_w4_linear(const void* X, int64_t ldx, int x_dtype, const float* x_scales,
                               int64_t x_group, int64_t n_tok, int64_t d, const void* Q,
                               const void* scales, int64_t group, int64_t d_out, void* Y,
                               int64_t ldy, int y_dtype, void* ws, size_t ws_bytes,
                               hipStream_t stream);

/* The gated product with 4-bit weights: H = act(X deq(Qg)^T) * (X deq(Qu)^T). */
optima_status optima_w4_gated(const void* X, int64_t ldx, int x_dtype, const float* x_scales,
                              int64_t x_group, int64_t n_tok, int64_t d, const void* Qg,
                              const void* scales_g, const void* Qu, const void* scales_u,
                              int64_t group, int64_t d_ff, int act, void* H, int64_t ldh,
                              int h_dtype, void* ws, size_t ws_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * From packed weights to a model's answers. The conventions are those of the
 * calls above.
 * ------------------------------------------------------------------------- */

/* Microscaled 4-bit floating point: rows of n x d values in blocks of 32.
 * A block has the scale 2^(e - 2), e = floor(log2(max |v|)), not below 2^-127, and the code of a
 * value is v / scale rounded to nearest even among 0, 0.5, 1, 1.5, 2, 3, 4 and 6 (codes 0 .. 7;
 * + 8 for negative ones), at most 6: a zero weight, as every pruned one is, stays exactly zero. A
 * block with a NaN or infinity has scale byte 255 and codes 0: all its values are NaN.
 * X: [n][ldx] of `dtype` F32 or BF16; weights or tokens.
 * Q: [n][optima_mx4_row_bytes(d)], 16-byte aligned. Code k is in byte k / 2 of its row, an even
 *   one in the low half; rows are padded to whole 256 values with zero codes.
 * scales: [n][optima_mx4_scale_bytes(d)], 4-byte aligned: the exponent plus 127, that of block b
 *   (0 .. 3) of the 128 values c at byte 16 (c / 4) + 4 b + c % 4; rows are padded with zeros.
 * The 256-value pieces, n ceil(d / 256), are at most 2^27 - 8, here and in unpack. */
size_t optima_mx4_row_bytes(int64_t d);
size_t optima_mx4_scale_bytes(int64_t d);
optima_status optima_mx4_pack(const void* X, int64_t ldx, int dtype, int64_t n, int64_t d, void* Q,
                              void* scales, hipStream_t stream);

/* The values that codes and scales stand for, Y: [n][ldy] of `dtype` F32 or BF16. Both hold every
 * value of pack exactly. */
optima_status optima_mx4_unpack(const void* Q, const void* scales, int64_t n, int64_t d, void* Y,
                                int64_t ldy, int dtype, hipStream_t stream);

/* Y = X W^T for packed weights W [d_out][d], as optima_mx4_pack lays them out.
 * X: [n_tok][d] of x_dtype BF16 with pitch ldx and x_scales NULL, or of MX4: packed tokens with
 * x_scales (ldx is not used). n_tok <= 2^21, d <= 2^20, d_out <= 2^24, and fewer than 2^24 - 8
 * tiles of 64 x 64 outputs. Y: [n_tok][d_out] BF16 or F32. Products of values are exact, their sums
 * fp32. A zero weight adds exactly nothing, except to an infinite or NaN token (NaN). More than 16
 * packed tokens want both scales 16-byte aligned, as an allocation is: at other multiples of 4 bytes
 * every 16 tokens read all weights again.
 * ws: optima_mx4_workspace_bytes(n_tok, d, d_out) bytes: 0 up to 8 tokens, never less for more. */
size_t optima_mx4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out);
optima_status optima_mx4_linear(const void* X, int64_t ldx, int x_dtype, const void* x_scales,
                                int64_t n_tok, int64_t d, const void* Q, const void* scales,
                                int64_t d_out, void* Y, int64_t ldy, int y_dtype, void* ws,
                                size_t ws_bytes, hipStream_t stream);

/* Log probabilities of given tokens under rows of logits, z = scale * X (scale > 0, as one over a
 * temperature):
 *   lse = log sum exp z,  logp = z[token] - lse,  entropy = - sum p log p,  p = exp(z - lse)
 * and the k most probable alternatives, top_index and top_logp: [n][k], by falling logit, equal
 * ones by rising index (-0 is 0; in a row with NaN they are k different places, no more is said).
 * X: [n][ldx] of `dtype` F32 or BF16, vocab <= 2^20 of them a row. tokens: [n], needed for logp; a
 * negative one is none (logp 0), one of vocab or more gives NaN. logp, lse, entropy: fp32 [n],
 * each nullable; k <= OPTIMA_TOP_MAX and vocab, top_index and top_logp each nullable, one at
 * least with k > 0.
 * Logits of -inf have probability 0 and add nothing to the entropy. A row with nothing else has lse,
 * logp and top_logp -inf and entropy 0; one with NaN or +inf has NaN in all four.
 * ws: optima_token_logprobs_workspace_bytes(n, vocab, k) bytes, 8-byte aligned: never less for
 * more rows. */
#define OPTIMA_TOP_MAX 32
size_t optima_token_logprobs_workspace_bytes(int64_t n, int64_t vocab, int64_t k);
optima_status optima_token_logprobs(const void* X, int64_t ldx, int dtype, int64_t n, int64_t vocab,
                                    const int64_t* tokens, float scale, float* logp, float* lse,
                                    float* entropy, int64_t k, int64_t* top_index, float* top_logp,
                                    void* ws, size_t ws_bytes, hipStream_t stream);

/* Gradient of the log probabilities, the entropy and lse, from what the forward call stored:
 *   dX = scale * (dlogp (onehot(token) - p) - dentropy p (log p + entropy) + dlse p)
 * with p = exp(z - lse). dlogp (with tokens), dentropy (with entropy) and dlse: fp32 [n], each
 * nullable, one at least. A row without a token has no part of dlogp; one whose token is vocab or
 * more is NaN; one whose lse is below -1e30 (nothing but masks) has gradient 0. Where |lse| is more
 * than 256 and the row's own (within |lse| 2^-22), p is worked out from the row itself, so that common
 * offsets, as a mask of -1e9 on all of a row, cost no accuracy; elsewhere it is as exact as lse, within
 * |lse| 2^-24 of itself. dX: [n][lddx] of X's dtype, and may be X itself (same pointer and pitch). */
optima_status optima_token_logprobs_backward(const void* X, int64_t ldx, int dtype, int64_t n,
                                             int64_t vocab, const int64_t* tokens, float scale,
                                             const float* lse, const float* entropy,
                                             const float* dlogp, const float* dentropy,
                                             const float* dlse, void* dX, int64_t lddx,
                                             hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* OPTIMA_H */
