/*
 * soap.h — C ABI of the MI355X (gfx950) SOAP optimizer-step library.
 *
 * The library performs the per-weight-matrix SOAP update of "SOAP, Muon, and
 * Beyond: Pushing LLM Pretraining Scales" (Algorithm 2, KL-SOAP listing, with
 * the plain-EMA Kronecker factors of the Section 2 Shampoo primer, eigenbasis
 * refresh every step (F = 1, hyperparameter table of Section 5.4) and the
 * real-time refresh of Section 5.4.2).  One call of soap_step does, in order:
 *
 *   1. L <- b2 L + (1-b2) G G^T,   R <- b2 R + (1-b2) G^T G          (factor EMA)
 *   2. Q_L <- QR(L Q_L).Q,  Q_R <- QR(R Q_R).Q, diag(R-factor) >= 0  (refresh)
 *   3. M <- b1 M + (1-b1) G;  G' = Q_L^T G Q_R;  M' = Q_L^T M Q_R    (rotate in)
 *   4. V <- b2 V + (1-b2) G'^2;  N = (M'/c1) / (sqrt(V/c2) + eps)    (Adam)
 *   5. W <- (1 - lr wd) W - lr Q_L N Q_R^T                            (rotate out)
 *
 * with c1 = 1 - b1^t and c2 = 1 - b2^t (c1 = c2 = 1 under
 * SOAP_FLAG_NO_BIAS_CORRECTION).  M is the first moment in weight space; by
 * linearity and orthogonality of the Q this equals Algorithm 2's
 * eigenbasis-resident m when the basis is refreshed every step.  V is indexed
 * by (column of Q_L, column of Q_R).
 *
 * Conventions for every entry point:
 *  - All matrices are fp32, row-major and dense: the leading dimension is the
 *    number of columns.  A weight is m x n ("in" x "out" in Algorithm 2):
 *    param, grad, M, V are m x n; L, Q_L are m x m; R, Q_R are n x n.
 *    Batched tensors are contiguous [batch][rows][cols].
 *  - Matrix pointers are DEVICE pointers (hipMalloc or torch device memory),
 *    16-byte aligned.  The caller owns every buffer, including the workspace;
 *    the library never allocates or frees device memory.  It keeps no
 *    optimizer state between calls.  It does keep, until the process ends:
 *    the thread-local error string; per device, three internal streams of
 *    default priority (created on first use: the m x m factor's chain and
 *    the block factorizations of both QRs run on them, forked from and
 *    joined back into the caller's stream with events); per host thread and
 *    device, seven HIP events for the step's forks and joins, and per host
 *    thread a pool of up to 4096 events for those of the QR; per device, the
 *    result of one occupancy query (how many QR block workgroups the device
 *    holds at once); and, while soap_timing_enable(1) is in force, timing
 *    events.
 *  - Work is enqueued on `stream` (0 = the null stream) and the call returns
 *    without synchronising.  Validation happens on the host before anything is
 *    enqueued: on failure nothing is enqueued, a negative soap_status is
 *    returned and soap_last_error() describes it.  A HIP launch error is
 *    reported as SOAP_ERR_HIP; a device fault surfaces at the caller's next
 *    synchronisation.  NaN/Inf in the inputs propagate and are not checked.
 *  - Calls on different streams are safe when their buffers and workspaces are
 *    disjoint (several steps running at once may make a QR give up and keep
 *    its old basis: see soap_workspace_status).  No C++ exception crosses
 *    this boundary.
 *  - Every dimension must be in [1, SOAP_MAX_DIM].
 */
#ifndef SOAP_MI355X_H
#define SOAP_MI355X_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SOAP_OK = 0,
  SOAP_ERR_NULL = -1,       /* a required pointer is NULL                       */
  SOAP_ERR_SHAPE = -2,      /* batch/m/n outside [1, SOAP_MAX_DIM] or overflow   */
  SOAP_ERR_HPARAM = -3,     /* beta outside [0,1), eps/lr/wd negative or not finite,
                               step < 1, unknown flag bits                       */
  SOAP_ERR_WORKSPACE = -4,  /* workspace smaller than the *_workspace_bytes value */
  SOAP_ERR_ALIGN = -5,      /* a pointer is not aligned as its entry point asks   */
  SOAP_ERR_ALIAS = -6,      /* grad overlaps a buffer the call writes, or two
                               written buffers overlap                           */
  SOAP_ERR_HIP = -7,        /* a HIP runtime call failed                         */
  SOAP_ERR_QR_GAVE_UP = -8  /* soap_workspace_status: a QR's bounded wait gave up  */
} soap_status;

/* Step flags (bitwise or):
 *  SOAP_FLAG_NO_BIAS_CORRECTION  c1 = c2 = 1 (Algorithm 2 as printed).
 *  SOAP_FLAG_SKIP_REFRESH        keep Q_L, Q_R: no power product, no QR this
 *                                step (Algorithm 2 refreshes when t mod F = 0;
 *                                the caller sets this flag on the other steps).
 *                                The factors and the Adam part are updated.
 *  SOAP_FLAG_STALE_REFRESH       refresh from the factors as they were before
 *                                this step's gradient was added: the lagging
 *                                preconditioner of Section 5.4.1, which the
 *                                real-time refresh of Section 5.4.2 replaces
 *                                (an ablation; no effect with SKIP_REFRESH). */
enum {
  SOAP_FLAG_NO_BIAS_CORRECTION = 1u << 0,
  SOAP_FLAG_SKIP_REFRESH = 1u << 1,
  SOAP_FLAG_STALE_REFRESH = 1u << 2
};

#define SOAP_MAX_DIM 16384

/* Bits of a step's status word (soap_workspace_status): the QR of the m x m
 * factor (or soap_qr_f32's matrix) / of the n x n factor gave up. */
enum { SOAP_STATUS_QR_L = 1u << 0, SOAP_STATUS_QR_R = 1u << 1 };

/* Bytes of device workspace soap_step / soap_step_batched need for `batch`
 * matrices of shape m x n (batch = 1 for soap_step).  Returns 0 for an invalid
 * shape.  The workspace holds the power products L Q_L and R Q_R, the QR
 * block reflectors and the rotation intermediates; its contents need not be
 * initialised and are garbage after the call. */
size_t soap_workspace_bytes(int64_t batch, int64_t m, int64_t n);

/* Initial optimizer state (the paper gives none; identity bases keep the
 * first power product nonsingular): L = R = Q_L = Q_R = I, M = V = 0, for
 * `batch` contiguous matrices.  Any of the six pointers may be NULL to skip
 * that tensor. */
int soap_init_state(int64_t batch, int64_t m, int64_t n, float *L, float *R, float *Q_L,
                    float *Q_R, float *M, float *V, hipStream_t stream);

/* One SOAP step on one m x n weight (Algorithm 2, F = 1).  `param`, L, R,
 * Q_L, Q_R, M, V are updated in place; `grad` is read only.  L and R are read
 * from their lower triangle and written fully symmetric.  `step` is the
 * 1-based t of this update.  beta1, beta2 in [0,1); eps, lr, weight_decay
 * finite and >= 0; flags is a combination of the SOAP_FLAG_* bits. */
int soap_step(float *param, const float *grad, float *L, float *R, float *Q_L, float *Q_R,
              float *M, float *V, int64_t m, int64_t n, float beta1, float beta2, float eps,
              float lr, float weight_decay, int64_t step, uint32_t flags, void *workspace,
              size_t workspace_bytes, hipStream_t stream);

/* soap_step on `batch` same-shape matrices in one call (e.g. the experts of an
 * MoE layer).  Every tensor is contiguous [batch][..][..] in the layout of
 * soap_step; the matrices are independent and share the hyperparameters. */
int soap_step_batched(int64_t batch, float *param, const float *grad, float *L, float *R,
                      float *Q_L, float *Q_R, float *M, float *V, int64_t m, int64_t n,
                      float beta1, float beta2, float eps, float lr, float weight_decay,
                      int64_t step, uint32_t flags, void *workspace, size_t workspace_bytes,
                      hipStream_t stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): soap_step
 * without a workspace argument.  The library's own scratch, a static device
 * array of SOAP_NOALLOC_MAX_WORKSPACE_BYTES per GPU (held until the process
 * ends), takes the workspace's place; the call allocates and frees nothing.
 * Shapes whose soap_workspace_bytes(1, m, n) exceed it are rejected with
 * SOAP_ERR_WORKSPACE (up to 2048 x 2048 fits).  Arguments, results and errors
 * otherwise as for soap_step.  Every call on one GPU shares that GPU's
 * scratch: calls that overlap on one GPU (different streams, or host threads
 * without ordering) race and must not be issued.  The step clears what it
 * needs cleared; the scratch keeps the last call's contents.  A QR give-up
 * keeps the basis as in soap_step, but its status word lives in the scratch
 * and is not readable through soap_workspace_status.  The first call on a
 * device and host thread creates the library's streams and events (host-side
 * objects, no device memory). */
#define SOAP_NOALLOC_MAX_WORKSPACE_BYTES ((size_t)256 << 20)
int soap_step_noalloc(float *param, const float *grad, float *L, float *R, float *Q_L,
                      float *Q_R, float *M, float *V, int64_t m, int64_t n, float beta1,
                      float beta2, float eps, float lr, float weight_decay, int64_t step,
                      uint32_t flags, hipStream_t stream);

/* ---- KL-SOAP (the variant the paper recommends: Sections 5.4.3 and 7) ----
 * One KL-SOAP step replaces step 1 of soap_step by the KL-Shampoo accumulation
 * of Algorithm 2.  With the bases and factors of the previous step:
 *
 *   lambda_L = diag(Q_L^T L Q_L),   lambda_R = diag(Q_R^T R Q_R)
 *   L <- bk L + (1-bk)/n  G Q_R diag(1/(lambda_R+eps)) Q_R^T G^T
 *   R <- bk R + (1-bk)/m  G^T Q_L diag(1/(lambda_L+eps)) Q_L^T G
 *
 * (bk = beta_kron; n = "out", m = "in").  Readings of Algorithm 2: bk
 * multiplies the old factor, as every EMA of the Section 2 primer does; the
 * exponent on (lambda + eps) is -1, the inverse that the KL-Shampoo rule of
 * Appendix A.3 uses; the estimates act in the basis that measured them, so
 * the weight is the other factor's inverse as that basis diagonalises it.
 * Steps 2-5 are those of soap_step; eps serves both the eigenvalue floor and
 * Adam (hyperparameter table of Section 5.4).  Arguments, layout, ownership
 * and errors as for soap_step, except that L and R must hold both triangles
 * on entry (the estimates read the whole stored factor; every step leaves
 * them symmetric); beta_kron must lie in [0, 1).  The workspace is larger
 * than soap_step's (one more m x n buffer and the estimates). */
size_t soap_kl_workspace_bytes(int64_t batch, int64_t m, int64_t n);
int soap_kl_step(float *param, const float *grad, float *L, float *R, float *Q_L, float *Q_R,
                 float *M, float *V, int64_t m, int64_t n, float beta1, float beta2,
                 float beta_kron, float eps, float lr, float weight_decay, int64_t step,
                 uint32_t flags, void *workspace, size_t workspace_bytes, hipStream_t stream);
int soap_kl_step_batched(int64_t batch, float *param, const float *grad, float *L, float *R,
                         float *Q_L, float *Q_R, float *M, float *V, int64_t m, int64_t n,
                         float beta1, float beta2, float beta_kron, float eps, float lr,
                         float weight_decay, int64_t step, uint32_t flags, void *workspace,
                         size_t workspace_bytes, hipStream_t stream);

/* ---- Muon (Algorithm 1, the paper's second optimizer) ----
 * One Muon step on an m x n weight ("in" x "out"):
 *
 *   M <- beta1 M + (1 - beta1) G
 *   X_0 = M / max(||M||_F, eps)
 *   for i = 1..n_iters:  A = X X^T,  B = b_i A + c_i A^2,  X <- a_i X + B X
 *   W <- (1 - lr wd) W - lr sqrt(max(m, n)) X_n
 *
 * The polynomial acts on singular values only, so the library forms the Gram
 * matrix on the smaller side (X^T X and X <- a X + X B when m > n); the
 * result is the same iterate.  coeffs is a HOST array of 3 n_iters floats
 * (a_1, b_1, c_1, a_2, ...): the paper uses the PolarExpress schedule with
 * n = 16 (hyperparameter table of Section 5.3) without printing it, so the
 * caller supplies the schedule.  param, grad, M are device pointers in the
 * layout of soap_step (grad read only, param and M updated); beta1 in [0, 1),
 * lr and weight_decay finite and >= 0, eps finite and > 0, n_iters in
 * [0, 1024].  flags 0: the products run in fp32 on the matrix cores.
 * flags SOAP_MUON_BF16: the Newton-Schulz iterations run in bfloat16, the
 * paper's precision for them (its discussion of orthogonalisation accuracy
 * in the conclusion): X_0, every A, B and X are bfloat16, each product
 * accumulated in fp32 on the bf16 matrix cores and rounded once to nearest
 * (ties to even); the momentum, the norm and the weight update stay fp32.
 * It needs m and n multiples of 8 (SOAP_ERR_SHAPE otherwise).
 * Ownership, streams and errors as for soap_step. */
enum { SOAP_MUON_BF16 = 1u << 0 };
size_t soap_muon_workspace_bytes(int64_t batch, int64_t m, int64_t n);
int soap_muon_step(float *param, const float *grad, float *M, int64_t m, int64_t n, float beta1,
                   float lr, float weight_decay, float eps, const float *coeffs, int64_t n_iters,
                   uint32_t flags, void *workspace, size_t workspace_bytes, hipStream_t stream);
int soap_muon_step_batched(int64_t batch, float *param, const float *grad, float *M, int64_t m,
                           int64_t n, float beta1, float lr, float weight_decay, float eps,
                           const float *coeffs, int64_t n_iters, uint32_t flags, void *workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* Description of the last failure on the calling thread ("" after success).
 * Valid until the next call on the same thread. */
const char *soap_last_error(void);

/* Device-side outcome of the last step (soap_step, soap_kl_step and their
 * batched forms) or soap_qr_f32 call enqueued with `workspace`.
 *
 * The QR factors each 128-column block with one launch whose workgroups must
 * all be resident at once (they exchange partial sums through memory); the
 * library sizes these launches from an occupancy query, but other work on the
 * GPU (another process, communication kernels that wait for peers, concurrent
 * steps on other streams) can hold the compute units they need.  Their waits
 * are therefore bounded: if one gives up, that factor's factorization is
 * marked failed, its eigenbasis (Q_L or Q_R; soap_qr_f32's Q) is LEFT AS IT
 * WAS ON ENTRY, and the rest of the step runs with it, exactly as a step with
 * SOAP_FLAG_SKIP_REFRESH would for that side.  The step sets the bit of that
 * side in the status word at offset 0 of its workspace; every step clears the
 * word when it starts.  Batches that take several launches per block (more
 * than 96 workgroups of 256 rows each on a side) never give up: their waits
 * are short, and a block whose wait ends without its partners is factored
 * again by one workgroup that waits for nobody.
 *
 * This call waits for `stream` (a host synchronisation), reads the word into
 * *status (if not NULL) and returns SOAP_OK when it is 0, SOAP_ERR_QR_GAVE_UP
 * when a SOAP_STATUS_QR_* bit is set (soap_last_error() names the side), or
 * SOAP_ERR_WORKSPACE when it holds other bits (not such a workspace). */
int soap_workspace_status(const void *workspace, uint32_t *status, hipStream_t stream);

/* Byte offset, inside the workspace of soap_step / soap_step_batched /
 * soap_kl_step(_batched), of the eigenbasis update N = (M'/c1) /
 * (sqrt(V/c2) + eps) that the last step wrote there (fp32, [batch][m][n]);
 * valid once that step's stream has been synchronised and until the next call
 * with the workspace.  For diagnostics; 0 for an invalid shape. */
size_t soap_workspace_update_offset(int64_t batch, int64_t m, int64_t n);

/* TEST HOOK, not for production use.  Every later QR (of a step or of
 * soap_qr_f32) whose SOAP_STATUS_QR_* bit is in `mask` starts with the abort
 * flags of its resident block factorizations raised, so that each of their
 * bounded waits gives up at once and every kernel still exits normally: the
 * give-up path above, on demand (in batches of several launches per block,
 * the repair of every block).  mask = 0 restores normal operation.  Only
 * QRs that take the resident block path are affected (matrices whose
 * factorization runs in more than one workgroup per block).  Returns
 * SOAP_ERR_HPARAM for other bits. */
int soap_test_force_qr_give_up(uint32_t mask);

/* TEST HOOK, not for production use.  on != 0: every later QR takes the panel
 * path, which devices (partitions) that cannot hold one matrix's block
 * workgroups at once take; its kernels wait for nobody.  on = 0 restores the
 * choice by the device. */
int soap_test_qr_panel_path(int on);

/* ---- stage entry points (used by the tests to check each kernel alone) ---- */

/* Eigenbasis refresh QR (Algorithm 2, "QR(.).Q"): A = Q Rf for one n x n
 * matrix, with diag(Rf) >= 0, by blocked Householder.  A is read only; Q (n x n)
 * receives the Q factor; Rf (n x n, may be NULL) the triangular factor with its
 * strict lower part zeroed.  If the factorization gives up (see
 * soap_workspace_status, bit SOAP_STATUS_QR_L) Q is left as it was on entry
 * and Rf is undefined. */
size_t soap_qr_workspace_bytes(int64_t n);
int soap_qr_f32(int64_t n, const float *A, float *Q, float *Rf, void *workspace,
                size_t workspace_bytes, hipStream_t stream);

/* The MFMA GEMM used for every product of the step:
 * C = alpha * op(A) op(B) + beta * C, op(X) = X or X^T (trans != 0),
 * op(A) M x K, op(B) K x N, row-major with leading dimensions lda, ldb, ldc.
 * When beta == 0, C is not read. */
int soap_gemm_f32(int trans_a, int trans_b, int64_t M, int64_t N, int64_t K, float alpha,
                  const float *A, int64_t lda, const float *B, int64_t ldb, float beta,
                  float *C, int64_t ldc, hipStream_t stream);

/* Factor EMA (Section 2 primer): F <- beta F + (1 - beta) X X^T for X = G
 * (trans = 0, F is m x m) or X = G^T (trans = 1, F is n x n), G m x n.  Only
 * the lower triangle of X X^T is computed; F is written fully symmetric. */
int soap_factor_ema_f32(int trans, int64_t m, int64_t n, const float *G, float *F, float beta,
                        hipStream_t stream);

/* KL-Shampoo accumulation alone (step 1 of soap_kl_step) for one m x n
 * gradient G: L (m x m) and R (n x n) are read whole (both triangles; the
 * new term is added to the lower triangle) and written fully symmetric; Q_L,
 * Q_R (the previous step's bases) are read only.  lam_L (m floats) and lam_R (n floats), if not NULL, receive the
 * eigenvalue estimates diag(Q_L^T L Q_L), diag(Q_R^T R Q_R) of the factors
 * as they were on entry.  All pointers are device pointers; the workspace
 * (soap_kl_factors_workspace_bytes) is the caller's. */
size_t soap_kl_factors_workspace_bytes(int64_t m, int64_t n);
int soap_kl_factors_f32(int64_t m, int64_t n, const float *G, float *L, float *R,
                        const float *Q_L, const float *Q_R, float beta_kron, float eps,
                        float *lam_L, float *lam_R, void *workspace, size_t workspace_bytes,
                        hipStream_t stream);
/* ---- operators of the layer around an expert bank ----
 * What a trainer runs next to soap_step_batched: the layer norm and the router
 * in front of a bank of experts, and the experts' products in microscaled 4-bit
 * floating point, up to the [batch][m][n] gradient that the batched steps read.
 * Streams, errors and ownership as above, with these differences:
 *  - Activations, logits and their gradients are fp32 or bfloat16 (soap_dtype),
 *    with a row stride ld* in elements (>= the number of columns), and need only
 *    the alignment of an element.  Layer norm, quantisation and values move 16 bytes
 *    at a time wherever a row starts; the router's rows and a product's C do where
 *    they are 16-byte aligned, and go an element at a time elsewhere.  Parameters,
 *    their gradients, statistics, gates and losses are fp32, indices int32.  Other
 *    buffers are 16-byte aligned where they are the library's own formats (packed
 *    matrices, workspaces; the scales of packed matrices 8-byte aligned) and
 *    element-aligned otherwise.
 *  - The token axis may be empty (rows = 0, tokens = 0: sums and counts are then
 *    zero) and goes up to SOAP_MAX_ROWS.
 *  - No output may overlap an input or another output; the range of a strided
 *    matrix is that from its first to its last element.
 *  - Results do not vary between runs: no floating-point sum depends on the order
 *    of atomics. */
typedef enum { SOAP_F32 = 0, SOAP_BF16 = 1 } soap_dtype;
#define SOAP_MAX_ROWS (1 << 24)

/* Layer norm of each row of x (rows x cols, 1 <= cols <= SOAP_MAX_DIM):
 *   mean = sum x / cols,  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps)
 *   y = weight (x - mean) rstd + bias
 * weight and bias hold cols floats (NULL: ones, zeros); mean and rstd receive
 * rows floats for the backward pass (NULL: not wanted); eps is finite and > 0.
 * The sums are fp32: a row whose sum (x - mean)^2 passes their range has rstd 0.
 * The backward pass gives, with h = (x - mean) rstd and g = weight dy,
 *   dx = rstd (g - mean(g) - h mean(g h)),  dweight = sum_rows dy h,  dbias = sum_rows dy
 * (each NULL where it is not wanted, dx too); the workspace holds the partial
 * sums of dweight and dbias (it may be NULL if neither is wanted).  Its size never
 * shrinks as rows or cols grow: one for the largest call serves the others. */
int soap_layer_norm_forward(int64_t rows, int64_t cols, int dtype, const void *x, int64_t ldx,
                            const float *weight, const float *bias, float eps, void *y, int64_t ldy,
                            float *mean, float *rstd, hipStream_t stream);
size_t soap_layer_norm_workspace_bytes(int64_t rows, int64_t cols);
int soap_layer_norm_backward(int64_t rows, int64_t cols, int dtype, const void *dy, int64_t lddy,
                             const void *x, int64_t ldx, const float *weight, const float *mean,
                             const float *rstd, void *dx, int64_t lddx, float *dweight, float *dbias,
                             void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Router of `tokens` rows of `experts` logits (1 .. SOAP_ROUTER_MAX_EXPERTS).
 * A token routes unless token_mask (tokens bytes, NULL: none) is 0 for it or it
 * has no logit above -inf.  It takes its top_k largest logits (1 ..
 * min(experts, SOAP_ROUTER_MAX_TOP_K)), equal ones by the lowest index, -inf and
 * NaN never:
 *   index[t][j]  the j-th largest's expert, or -1 where there is none
 *   gate[t][j]   p of that expert, p = softmax of the token's logits, divided by
 *                the sum of the token's chosen p under SOAP_ROUTER_RENORMALIZE
 *                (0 where index is -1)
 *   counts[e]    tokens that chose e; counts[experts] = N, the tokens that route
 *   loss         balance experts sum_e f_e P_e, f_e = counts[e] / (sum of counts),
 *                P_e = sum over those tokens of p_e / N  (0 if N = 0; may be NULL)
 * and the dispatch plan (offsets, position and row_token, all or none NULL): the
 * tokens of expert e have the rows offsets[e] + 0, 1, ... in ascending order, and
 * offsets[e + 1] is the next multiple of 32 (experts + 1 values); position[t][j]
 * is the row of index[t][j] (or -1), row_token[r] the token of row r, -1 where it
 * has none, over all soap_router_rows(tokens, experts, top_k) rows.  tokens top_k
 * is at most 2^30.  A NaN logit makes its token's gates and the loss NaN.
 *
 * The backward pass takes index and counts as the forward pass left them (the
 * experts of a token distinct) and writes dlogits from the gradient of the gates
 * (dgate, tokens x top_k, NULL: zero; not read where index is -1) and of the loss
 * (dloss, one device float, NULL: 1), f_e being constants:
 *   b_e = dloss balance experts f_e / N
 *   gates as p:    dlogits = p (d - sum p d), d = b + dgate at the chosen experts
 *   renormalised:  dlogits = p (b - sum p b) + gate (dgate - sum gate dgate)
 * and zeros for tokens that do not route. */
enum { SOAP_ROUTER_RENORMALIZE = 1u << 0 };
#define SOAP_ROUTER_MAX_EXPERTS 1024
#define SOAP_ROUTER_MAX_TOP_K 32
int64_t soap_router_rows(int64_t tokens, int64_t experts, int64_t top_k);
size_t soap_router_workspace_bytes(int64_t tokens, int64_t experts);
int soap_router_forward(int64_t tokens, int64_t experts, int64_t top_k, int dtype, const void *logits,
                        int64_t ld, const uint8_t *token_mask, uint32_t flags, float balance,
                        int32_t *index, float *gate, int32_t *counts, float *loss, int32_t *offsets,
                        int32_t *position, int32_t *row_token, void *workspace, size_t workspace_bytes,
                        hipStream_t stream);
int soap_router_backward(int64_t tokens, int64_t experts, int64_t top_k, int dtype, const void *logits,
                         int64_t ld, const uint8_t *token_mask, uint32_t flags, float balance,
                         const int32_t *index, const int32_t *counts, const float *dgate,
                         const float *dloss, void *dlogits, int64_t ldd, hipStream_t stream);

/* Microscaled 4-bit floating point (MXFP4).  A packed matrix of `rows` rows of k
 * values holds, per row, P / 2 bytes of data and P / 32 bytes of scales, P = k
 * padded to a multiple of 256 (zeros): value i is the lower (i even) or upper
 * half of byte i / 2, one bit of sign and three that stand for 0, 0.5, 1, 1.5, 2,
 * 3, 4, 6, times 2^(s - 127), s the scale byte of its block of 32.  Quantising takes
 * 2^(s - 127) = 2^(floor(log2 max|x|) - 2), at least 2^-127, and rounds x over it to
 * the nearest value, ties to the even code, 6 at most; a block that holds an
 * infinity or a NaN gets s = 255, which makes all its values NaN.
 *
 * soap_mx4_quantize packs `batch` matrices of rows x cols (matrix b at x + b rows
 * ldx) along the columns (data, scale: rows x cols), along the rows (data_t,
 * scale_t: the transposed cols x rows), or both in one pass over x; an unwanted
 * pair is NULL.  With row_index (batch = 1; `rows` int32), row r is row
 * row_index[r] of x, or zeros where that is outside [0, x_rows); without it x_rows
 * is ignored.  Packed matrices of a batch follow each other. */
size_t soap_mx4_data_bytes(int64_t rows, int64_t k);
size_t soap_mx4_scale_bytes(int64_t rows, int64_t k);
int soap_mx4_quantize(int64_t batch, int64_t rows, int64_t cols, int dtype, const void *x, int64_t ldx,
                      const int32_t *row_index, int64_t x_rows, uint8_t *data, uint8_t *scale,
                      uint8_t *data_t, uint8_t *scale_t, hipStream_t stream);
/* Rows of a packed matrix: row r of the output (rows x k) is row row_index[r] of the
 * input (x_rows x k), or zeros where that is outside [0, x_rows).  Quantising x_rows
 * rows and copying them so gives what soap_mx4_quantize gives with row_index, and is the
 * faster where rows are taken often, which is the caller's to choose, as the packed
 * x_rows x k are: about where rows k exceeds 28 2^20 + 1.6 x_rows k (bfloat16) or
 * 14 2^20 + 0.8 x_rows k (fp32) for k past 1280, more for shorter rows. */
int soap_mx4_gather(int64_t rows, int64_t k, const int32_t *row_index, int64_t x_rows,
                    const uint8_t *x_data, const uint8_t *x_scale, uint8_t *data, uint8_t *scale,
                    hipStream_t stream);
/* The values of a packed matrix, rounded once to a bfloat16 output. */
int soap_mx4_dequantize(int64_t rows, int64_t k, const uint8_t *data, const uint8_t *scale, int dtype,
                        void *out, int64_t ldo, hipStream_t stream);

/* Rows of a packed matrix along the columns and the k of one along the rows may be
 * as many as a dispatch plan has (2^31 - 1 rows, 2 SOAP_MAX_ROWS k); cols, N and K
 * otherwise go up to SOAP_MAX_ROWS. */

/* Products of packed matrices, C = A B^T summed over k in fp32 and rounded once to
 * a bfloat16 output.
 *   soap_mx4_gemm            A M x K, B N x K, C M x N with row stride ldc.
 *   soap_mx4_gemm_rows       B is `groups` packed N x K matrices; rows offsets[g] ..
 *                            offsets[g + 1] of C are those of A with B[g], the rows
 *                            from offsets[groups] on are zeros.
 *   soap_mx4_gemm_k          C[g] (M x N, groups of them contiguous) sums over the k
 *                            from offsets[g] to offsets[g + 1] only (zeros if none).
 * offsets: groups + 1 device int32 (groups <= SOAP_MAX_DIM), 0 first, ascending,
 * for soap_mx4_gemm_k multiples of 32, as the router's plan has them; values outside
 * the matrix are taken as its ends. */
int soap_mx4_gemm(int64_t M, int64_t N, int64_t K, const uint8_t *a_data, const uint8_t *a_scale,
                  const uint8_t *b_data, const uint8_t *b_scale, int dtype, void *C, int64_t ldc,
                  hipStream_t stream);
int soap_mx4_gemm_rows(int64_t groups, int64_t M, int64_t N, int64_t K, const int32_t *offsets,
                       const uint8_t *a_data, const uint8_t *a_scale, const uint8_t *b_data,
                       const uint8_t *b_scale, int dtype, void *C, int64_t ldc, hipStream_t stream);
int soap_mx4_gemm_k(int64_t groups, int64_t M, int64_t N, int64_t K, const int32_t *offsets,
                    const uint8_t *a_data, const uint8_t *a_scale, const uint8_t *b_data,
                    const uint8_t *b_scale, int dtype, void *C, hipStream_t stream);

/* ---- operators of a dense layer ----
 * The entry of attention, the feed-forward block and a loss on the logits, with their
 * gradients, under the rules of the operators around an expert bank above (types, empty
 * token axes, no overlapping outputs, results that do not vary between runs). */

/* RMS norm of every head of queries and keys and the rotation by its token's position, in
 * one pass: of a head x of dim values (even, 2 .. SOAP_HEAD_MAX_DIM)
 *   h = x / sqrt(sum x^2 / dim + eps),  y = w h
 * and the pairs (a, b) of the first `rotary` values of y (even, 0 .. dim) are turned to
 *   (a cos t - b sin t, b cos t + a sin t),  t = position frequencies[i] of pair i,
 * pair i being the values i and i + rotary / 2, or 2 i and 2 i + 1 with
 * SOAP_HEAD_INTERLEAVED.  q_heads queries and k_heads keys a token (0 .. SOAP_HEAD_MAX_HEADS;
 * a side without heads is not touched); strides of tokens and heads are in elements (below
 * 2^31), those of a head 1, so that q and k may lie in one fused row and heads in front of tokens.  Weights
 * hold dim floats (NULL: ones), positions one int32 a token (NULL: 0, 1, ..), frequencies
 * rotary / 2 doubles; the angle is formed in fp64.  Inputs may repeat (stride 0).  An output's
 * heads lie behind each other within a token and tokens behind each other, or tokens within a head;
 * they may lie between those of the other side: in rows of the same stride, the heads next to each
 * other or (of the same stride too) in turn with them.
 * A head whose sum of squares passes fp32's range becomes zeros (NaN if it holds an infinity
 * or a NaN).
 * The backward pass takes the gradients of the outputs and the inputs again and gives, with
 * g the gradient turned back,
 *   dx = r (w g - h sum(w g h) / dim), r = h / x,  dw = sum over tokens and heads of g h
 * (each NULL where it is not wanted); the workspace holds partial sums of the weights'
 * gradients (it may be NULL if neither is wanted). */
enum { SOAP_HEAD_INTERLEAVED = 1u << 0 };
#define SOAP_HEAD_MAX_DIM 512
#define SOAP_HEAD_MAX_HEADS 1024
int soap_head_norm_forward(int64_t tokens, int64_t q_heads, int64_t k_heads, int64_t dim, int64_t rotary,
                           int dtype, uint32_t flags, const void *q, int64_t q_token, int64_t q_head,
                           const void *k, int64_t k_token, int64_t k_head, const float *q_weight,
                           const float *k_weight, float eps, const int32_t *positions,
                           const double *frequencies, void *q_out, int64_t q_out_token, int64_t q_out_head,
                           void *k_out, int64_t k_out_token, int64_t k_out_head, hipStream_t stream);
size_t soap_head_norm_workspace_bytes(int64_t tokens, int64_t dim);
int soap_head_norm_backward(int64_t tokens, int64_t q_heads, int64_t k_heads, int64_t dim, int64_t rotary,
                            int dtype, uint32_t flags, const void *dq_out, int64_t dq_out_token,
                            int64_t dq_out_head, const void *dk_out, int64_t dk_out_token, int64_t dk_out_head,
                            const void *q, int64_t q_token, int64_t q_head, const void *k, int64_t k_token,
                            int64_t k_head, const float *q_weight, const float *k_weight, float eps,
                            const int32_t *positions, const double *frequencies, void *dq, int64_t dq_token,
                            int64_t dq_head, void *dk, int64_t dk_token, int64_t dk_head, float *dq_weight,
                            float *dk_weight, void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Gated feed-forward block in bfloat16 with fp32 sums:
 *   G = X Wg,  U = X Wu,  H = act(G) U (values one by one),  Y = H Wd
 * X tokens x m, Wg and Wu m x n, Wd n x p, Y tokens x p: the weights are stored "in" x "out"
 * as the steps update them, each rounded to bfloat16.  m, n and p are multiples of 8; rows of
 * X, Y and their gradients start at multiples of 16 bytes (ld a multiple of 8, up to
 * SOAP_GATED_MAX_LD), the other matrices are dense.  act is x / (1 + exp(-x)) (SILU) or
 * x (1 + erf(x / sqrt 2)) / 2 (GELU).  G, U (tokens x n, both or neither NULL) are kept for the
 * backward pass.  Sums are fp32; G, U, H and Y are rounded to bfloat16 once, H from unrounded
 * G and U.
 * The backward pass gives, from dY, X and the kept G and U (H is computed again),
 *   dH = dY Wd^T,  dG = dH U act'(G),  dU = dH act(G)
 *   dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU,  dWd = H^T dY
 * (each NULL where it is not wanted): dG, dU and H are rounded to bfloat16 as operands (so that a
 * bfloat16 result's error is sqrt 2 times that of its own rounding, Y's too), dX too, the weights'
 * gradients are fp32 (what the steps read) or bfloat16 (grad_dtype).  Up to 64 tokens' H, dG and dU
 * keep 16 binary digits, in two bfloat16 (where the matrix that they meet holds an infinity, their
 * product with it may be NaN).  Without tokens the gradients are zeros.  The workspace's size never
 * shrinks as tokens, m, n or p grow. */
typedef enum { SOAP_ACT_SILU = 0, SOAP_ACT_GELU = 1 } soap_activation;
#define SOAP_GATED_MAX_HIDDEN 65536
#define SOAP_GATED_MAX_LD (1 << 21)
size_t soap_gated_workspace_bytes(int64_t tokens, int64_t m, int64_t n, int64_t p, int backward);
int soap_gated_forward(int64_t tokens, int64_t m, int64_t n, int64_t p, int activation, const void *x,
                       int64_t ldx, const void *w_gate, const void *w_up, const void *w_down, void *gate,
                       void *up, void *y, int64_t ldy, void *workspace, size_t workspace_bytes,
                       hipStream_t stream);
int soap_gated_backward(int64_t tokens, int64_t m, int64_t n, int64_t p, int activation, const void *dy,
                        int64_t lddy, const void *x, int64_t ldx, const void *w_gate, const void *w_up,
                        const void *w_down, const void *gate, const void *up, void *dx, int64_t lddx,
                        int grad_dtype, void *dw_gate, void *dw_up, void *dw_down, void *workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* Distillation from a teacher's top logits: rows of logits z over `classes` (1 ..
 * SOAP_DISTILL_MAX_CLASSES) against a list of `slots` (1 .. SOAP_DISTILL_MAX_SLOTS) classes
 * index and values t of the teacher.  With tau the temperature, q = softmax(z / tau) and
 *   p_j = softmax of t / tau over the list,  r = 0, or with SOAP_DISTILL_TAIL
 *   p_j = exp(t_j) (t: the teacher's log probabilities),  r = max(0, 1 - sum p),
 * r against q_rest, the sum of q over the classes not listed:
 *   loss = tau^2 (sum_j p_j (log p_j - log q(index_j)) + r (log r - log q_rest))
 * A slot whose index is outside [0, classes) is empty, whatever its t.  A list of empty
 * slots, or (without a tail) whose t are all -inf, has loss 0 and gradient 0; a term with p_j = 0 (or r = 0) is 0.  Where no class
 * outside the list has a logit above -inf, r is taken as 0.  A class may be listed
 * more than once: its p add up in the gradient.  Cross entropy to labels is slots = 1.
 * stats (rows x 2 floats, may be NULL forward): log sum exp(z / tau), over all classes and
 * (SOAP_DISTILL_TAIL, otherwise 0) over those not listed, for soap_distill_backward; with
 * SOAP_DISTILL_SUMS rows x 6: these two, then the largest logit m and sum exp((z - m) / tau) of
 * either (0, 0 without a tail).  From the logs alone q has an error of up to 2^-24 of their size,
 * and none is left of logs past fp32's range; from the sums it is the single pass':
 *   dlogits = dloss tau ((sum p + r) q - p)             at the listed classes, elsewhere
 *   dlogits = dloss tau ((sum p + r) q - r q / q_rest)
 * with dloss one float a row (NULL: ones); a row whose dloss is 0 gets zeros, whatever its
 * logits.  soap_distill_forward_backward gives both in one pass over the logits.  Sums are
 * fp32; a NaN or +inf among the logits makes its row NaN.  Logits that are all -inf have no q: their
 * loss and gradient are NaN (with a tail the gradient at the listed classes, elsewhere 0), but for
 * the zeros of empty lists and of a dloss of 0. */
enum { SOAP_DISTILL_TAIL = 1u << 0, SOAP_DISTILL_SUMS = 1u << 2 };
#define SOAP_DISTILL_MAX_CLASSES (1 << 18)
#define SOAP_DISTILL_MAX_SLOTS 512
#define SOAP_DISTILL_MIN_TEMPERATURE 0.01
#define SOAP_DISTILL_MAX_TEMPERATURE 100.0
int soap_distill_forward(int64_t rows, int64_t classes, int64_t slots, int dtype, const void *logits,
                         int64_t ld, const int32_t *index, int64_t ldi, int teacher_dtype,
                         const void *teacher, int64_t ldt, uint32_t flags, float temperature, float *loss,
                         float *stats, hipStream_t stream);
int soap_distill_backward(int64_t rows, int64_t classes, int64_t slots, int dtype, const void *logits,
                          int64_t ld, const int32_t *index, int64_t ldi, int teacher_dtype,
                          const void *teacher, int64_t ldt, uint32_t flags, float temperature,
                          const float *stats, const float *dloss, void *dlogits, int64_t ldd,
                          hipStream_t stream);
int soap_distill_forward_backward(int64_t rows, int64_t classes, int64_t slots, int dtype,
                                  const void *logits, int64_t ld, const int32_t *index, int64_t ldi,
                                  int teacher_dtype, const void *teacher, int64_t ldt, uint32_t flags,
                                  float temperature, const float *dloss, float *loss, float *stats,
                                  void *dlogits, int64_t ldd, hipStream_t stream);

/* ---- measurement ---- */

/* When enabled, every stage of soap_step / soap_step_batched records a pair
 * of HIP events on the call's stream.  soap_timing_collect synchronises on
 * them and adds their durations to per-stage totals; soap_timing_reset clears
 * the totals.  Stage ids are 0 .. soap_timing_num_stages()-1. */
int soap_timing_enable(int enable);
int soap_timing_num_stages(void);
const char *soap_timing_stage_name(int stage);
int soap_timing_collect(void);
int soap_timing_reset(void);
/* Totals since the last reset: milliseconds, launches, and the algorithmic
 * flops of those launches (one triangle for the factor EMA, 2 m n k for a
 * product, (4/3) n^3 + (4/3) n^3 for a QR with its explicit Q). */
int soap_timing_get(int stage, double *total_ms, int64_t *launches, double *flops);

#ifdef __cplusplus
}
#endif

#endif /* SOAP_MI355X_H */
