/*
 * shampoo.h -- C ABI of the MI355X (gfx950) per-block Shampoo optimizer step.
 *
 * The library computes, entirely in hand-written HIP kernels, the optimizer
 * step of Shi et al., "A Distributed Data-Parallel PyTorch Implementation of
 * the Distributed Shampoo Optimizer for Training Neural Networks At-Scale"
 * (arXiv 2309.06497), restricted to one GPU: blocked Kronecker-factor
 * accumulation (matrices, and tensors of order one, three and four after merging
 * of small dimensions), periodic inverse-root refresh by batched symmetric
 * eigendecomposition (or the coupled inverse Newton iteration), preconditioning
 * by the roots, AdaGrad / SGD / RMSprop / Adam grafting, gradient filtering,
 * bias correction, weight decay, (Nesterov) momentum and the parameter update.
 * The multi-GPU distribution of the paper (Sec. 4.1) is not part of this library.
 *
 * Conventions for every entry point
 *   - "device pointer": memory of the GPU the optimizer was created on,
 *     owned by the caller and never freed by the library.
 *   - "host pointer": ordinary process memory.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Work is enqueued on it; calls return without waiting unless stated.
 *   - Return value: 0 on success, negative error code otherwise (see
 *     shampoo_strerror).  Argument errors (every code except SHAMPOO_ERR_HIP)
 *     are detected before any work is enqueued: nothing has been modified.
 *   - No entry point throws; none is safe to call concurrently on the same
 *     shampoo_opt from several threads.
 */
#ifndef SHAMPOO_H
#define SHAMPOO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct shampoo_opt shampoo_opt; /* opaque, owned by the library */

enum {
  SHAMPOO_OK = 0,
  SHAMPOO_ERR_NULL = -1,      /* a required pointer is NULL                      */
  SHAMPOO_ERR_SHAPE = -2,     /* bad n_params / ndim / shape / block_size / index */
  SHAMPOO_ERR_HYPER = -3,     /* hyper-parameter out of range                     */
  SHAMPOO_ERR_WORKSPACE = -4, /* workspace NULL, misaligned or too small          */
  SHAMPOO_ERR_STEP = -5,      /* step not strictly increasing                     */
  SHAMPOO_ERR_HIP = -6,       /* a HIP runtime call failed, or host memory ran out */
  SHAMPOO_ERR_UNSUPPORTED = -7 /* size outside what the kernels support           */
};

enum { SHAMPOO_GRAD_F32 = 0, SHAMPOO_GRAD_BF16 = 1 };
enum { SHAMPOO_GRAFT_ADAGRAD = 0, SHAMPOO_GRAFT_SGD = 1, SHAMPOO_GRAFT_RMSPROP = 2, SHAMPOO_GRAFT_ADAM = 3 };
enum { SHAMPOO_ROOT_EIGH = 0, SHAMPOO_ROOT_NEWTON = 1 };
enum { SHAMPOO_MATRIX_CORES_AUTO = 0, SHAMPOO_MATRIX_CORES_FP32 = 1 };
enum { SHAMPOO_LARGE_DIM_BLOCKING = 0, SHAMPOO_LARGE_DIM_ADAGRAD = 1, SHAMPOO_LARGE_DIM_DIAGONAL = 2 };
#define SHAMPOO_MAX_NDIM 4

/*
 * Optimizer configuration (copied at create; the arrays need not outlive the call).
 * Hyper-parameters are those of the paper's complete pseudocode (Sec. 3,
 * "Complete Distributed Shampoo Pseudocode").
 */
typedef struct {
  int32_t n_params;       /* number of parameters (tensors), >= 1                          */
  const int32_t *ndim;    /* host [n_params]: 1 (diagonal AdaGrad path, Sec. 4.2.2), 2, 3 or 4.
                             A parameter of 3 or 4 dimensions first has its small dimensions
                             merged (Sec. 4.2.1: from the left, a dimension joins the current
                             group while the product stays <= block_size, a dimension of size 1
                             always; only a view, no data moves).  Two dimensions left: the matrix case on the merged shape.
                             Three or four left, or one (all merged): Shampoo for a tensor of that
                             order w (Sec. 2.3), one factor per dimension, root exponent
                             2 * root_exponent / w, blocks of at most block_size per dimension
                             (a block of more than 2^30 elements: SHAMPOO_ERR_UNSUPPORTED)   */
  const int64_t *shape;   /* host [SHAMPOO_MAX_NDIM * n_params]: the ndim[i] dimensions of
                             parameter i, slowest first, at shape[SHAMPOO_MAX_NDIM * i ...];
                             the remaining entries are ignored                               */
  int32_t block_size;     /* b: max_preconditioner_dim of Sec. 4.2.1, >= 1                  */
  float beta2;            /* in (0,1]; 1 = plain sum of G G^T, < 1 = EMA (Sec. 3.1.1)       */
  float epsilon;          /* > 0: added to the eigenvalues in the root inverse (Sec. 3.2.1) */
  float root_exponent;    /* r > 0: factors are raised to the power -r (0.25 for matrices)  */
  int32_t precondition_frequency;     /* f >= 1: roots refreshed when step % f == 0 (Sec. 4.3) */
  int32_t start_preconditioning_step; /* >= 0: before it the grafted direction is used alone   */
  float graft_epsilon;    /* >= 0: P_graft = G / (sqrt(A) + graft_epsilon) (Sec. 2.4)        */
  float momentum;         /* mu in [0,1): 0 disables the momentum state (Sec. 3.1.3)         */
  float beta1;            /* in [0,1): > 0 filters the gradient, Gf <- beta1 Gf + (1-beta1) G;
                             grafting state and factors use G, directions use Gf (Sec. 3.1.1) */
  float weight_decay;     /* >= 0 (Sec. 3.1.2)                                               */
  int32_t use_decoupled_weight_decay; /* != 0: P <- P - wd W after grafting; 0: G <- G + wd W  */
  int32_t use_nesterov;   /* != 0: W += lr (mu M + P) instead of lr M (Sec. 3.1.3)            */
  int32_t grafting_type;  /* SHAMPOO_GRAFT_ADAGRAD (A <- A + G.^2), SHAMPOO_GRAFT_SGD (P_graft = G, no
                             state), SHAMPOO_GRAFT_RMSPROP / _ADAM (A <- beta_g A + (1-beta_g) G.^2;
                             Adam divides A by 1 - beta_g^(step+1) when bias correction is on).
                             1-D parameters run that diagonal method itself (AdaGrad under SGD) */
  float grafting_beta2;   /* beta_g in (0,1] of RMSprop / Adam grafting; ignored otherwise   */
  int32_t use_bias_correction; /* != 0: directions use Gf / (1 - beta1^(step+1)) and roots are
                             taken of L / (1 - beta2^(step+1)) (beta2 < 1), epsilon added after
                             the division; stored state stays uncorrected (Sec. 3.1.1)        */
  int32_t large_dim_method; /* what happens to a 2-D parameter with a dimension above block_size (Sec. 4.2):
                             SHAMPOO_LARGE_DIM_BLOCKING (default): cut into blocks (Sec. 4.2.1);
                             SHAMPOO_LARGE_DIM_ADAGRAD: the diagonal method on its entries, as for a
                             1-D parameter (Sec. 4.2.2);
                             SHAMPOO_LARGE_DIM_DIAGONAL: kept whole, the factor of each such
                             dimension replaced by its diagonal (Sec. 4.2.3).
                             Tensors of order 1, 3 or 4 (after merging) are always blocked;
                             more than 65535 whole parameters or tensor blocks of one shape:
                             SHAMPOO_ERR_UNSUPPORTED                                          */
  int32_t root_method;    /* SHAMPOO_ROOT_EIGH: eigendecomposition (framed box of Sec. 3.2.1, default);
                             SHAMPOO_ROOT_NEWTON: coupled inverse Newton iteration of the same
                             section on L + epsilon I, in float32; needs 1/root_exponent in
                             {1, 2, 4, 8} (else SHAMPOO_ERR_UNSUPPORTED; for a tensor parameter
                             the exponent in question is 2 * root_exponent / w).  A factor whose
                             iterates do not stay finite (condition number beyond float32) is
                             handed to the eigendecomposition instead (the guard of Sec. 3.2.3);
                             to learn whether any did, a refresh step under this method waits
                             for `stream` once per batch of factors                          */
  float newton_tolerance; /* stop when ||M_k - I||_inf < this; 0 selects 1e-6 (Sec. 3.2.1)     */
  int32_t newton_max_iterations; /* iteration cap, <= 1000; 0 selects 100                     */
  int32_t precond_matrix_cores; /* SHAMPOO_MATRIX_CORES_AUTO (default): for blocks whose shape and
                             alignment allow it, Lbar G Rbar runs on the 16-bit matrix cores from split
                             operands.  bf16 gradients: float32 operands as two fp16 planes each, scaled
                             per block by a power of two (exact products accumulated in
                             float32: float32 accuracy at 3/16 of the float32-MFMA time; elements
                             below 2^-16 of a block's largest keep absolute, not relative,
                             accuracy).  Float32 or filtered gradients, more than 128 rows and columns:
                             three bf16 planes each, all 24 bits of every element, six products;
                             the factor updates of float32 gradients take the same planes.  All other
                             blocks: the same three terms, split on the way into the kernels.
                             SHAMPOO_MATRIX_CORES_FP32: always the float32 MFMA for Lbar G Rbar; the factor
                             updates are as under AUTO where no planes are kept: bf16 gradients as they
                             are, float32 ones as three bf16 terms, sums of 32 products in float64 */
  int32_t warm_start_roots; /* != 0: the eigendecomposition of a refresh starts from the eigenvectors of
                             the previous one (Sec. 3.2.1, 4.3: between refreshes a factor changes
                             little) instead of from the identity: W = Q^T L Q is formed (float64
                             sums) and the Jacobi sweeps begin there.  Factors of dimension <= 128 (solved
                             inside one workgroup) and the coupled Newton iteration ignore it.  Costs
                             one more float32 matrix per factor in the workspace.  Every 16th refresh
                             starts cold, which bounds the drift of the accumulated float32
                             eigenvectors away from orthogonality.  0 (default): every refresh cold */
  int32_t grad_dtype;     /* SHAMPOO_GRAD_F32 or SHAMPOO_GRAD_BF16; parameters are float32   */
  int32_t device;         /* HIP device ordinal                                              */
} shampoo_config;

/*
 * Block planner (host only, touches no GPU).  Sec. 4.2.1: a rows x cols
 * parameter is cut into ceil(rows/b) x ceil(cols/b) blocks, all b x b except
 * in the last block row / column.  Blocks of equal (m, n) form a bucket and
 * are numbered (slot) in parameter order, row-major inside a parameter.
 * Writes up to `cap` rows of 12 int64
 * {param, row0, col0, m, n, bucket, slot, flags, s3, d3, s4, d4}
 * into `table` (host, may be NULL when cap == 0) and the total number of
 * blocks / buckets into *n_blocks / *n_buckets (host, may be NULL).
 * A block of a tensor parameter (flags bit 2, and the order 1, 3 or 4 of the merged tensor
 * in flags bits 4..6) starts at (row0, col0, s3, s4) of the merged
 * shape and measures m x n x d3 x d4 (sizes 1 for the dimensions it does not have); matrix
 * blocks have s3 = s4 = 0, d3 = d4 = 1.  Tensor blocks are numbered in row-major order of
 * their block indices.
 * Under SHAMPOO_LARGE_DIM_DIAGONAL a parameter with a dimension above b is one row
 * (m, n = its shape) with flags bit 0 / bit 1 set where the left / right factor is
 * diagonal; under SHAMPOO_LARGE_DIM_ADAGRAD such a parameter has no row (it is handled
 * like a 1-D parameter).
 */
int shampoo_plan(const shampoo_config *cfg, int64_t *table, int64_t cap,
                 int64_t *n_blocks, int64_t *n_buckets);

/* Bytes of device workspace shampoo_create needs for cfg; 0 if cfg is invalid.  Beside the state (factors, roots,
 * A, M, the last direction) it holds scratch of the size of the largest bucket or of several up to 2 GiB, scratch of the root refresh (at most
 * about 8 GiB; half of what it would otherwise be with warm_start_roots and for exponents above 0.66; the same memory, where no
 * planes of float32 gradients wait for the end of a refresh), and for blocks
 * whose products run on the 16-bit matrix cores a second copy of the roots: 4 bytes per element, 6 for float32
 * directions, whose planes take up to 2 GiB more. */
size_t shampoo_workspace_bytes(const shampoo_config *cfg);

/*
 * Create an optimizer.  `workspace` is a device pointer, 256-byte aligned, of
 * at least shampoo_workspace_bytes(cfg) bytes; it holds all optimizer state
 * (factors L, R, roots, grafting state A, momentum M) and scratch, and must
 * stay allocated until shampoo_destroy.  State is initialised (L = R = 0,
 * roots = I, A = M = 0) on `stream`, which is synchronised before returning.
 * *out (host) receives the handle.
 */
int shampoo_create(const shampoo_config *cfg, void *workspace, size_t workspace_bytes,
                   void *stream, shampoo_opt **out);

/*
 * One optimizer iteration t = `step` (0-based, strictly increasing between
 * calls) of the complete pseudocode for every block of every parameter:
 *   G <- G + wd W   (l2 weight decay only)               (Sec. 3.1.2)
 *   L <- beta2 L + (1-beta2) G G^T, R likewise          (Sec. 3.1.1)
 *   A <- A + G.^2   (AdaGrad grafting; EMA for RMSprop / Adam)   (Sec. 2.4, 2.2)
 *   if step >= start and step % f == 0: roots refreshed  (Sec. 3.2.1 box, 4.3)
 *   Gf <- beta1 Gf + (1-beta1) G  (Gf = G when beta1 = 0) (Sec. 3.1.1)
 *       (with bias correction the lines below read Gf / (1 - beta1^(step+1)))
 *   P_graft = Gf/(sqrt(A)+eps_g)  or  Gf (SGD grafting)
 *   P = -||P_graft||_F * Lbar Gf Rbar / ||Lbar Gf Rbar||_F           (Sec. 2.4)
 *       (P = -P_graft while step < start; 1-D parameters: -Gf/(sqrt(A)+eps_g))
 *   P <- P - wd W   (decoupled weight decay only)        (Sec. 3.1.2)
 *   M <- mu M + P ; W <- W + lr M  (Nesterov: lr (mu M + P))          (Sec. 3.1.3)
 * A block of a tensor parameter has one factor per dimension k,
 *   L_k <- beta2 L_k + (1-beta2) G_(k) G_(k)^T  (G_(k): mode-k unfolding),
 * and P_shampoo = G x_1 Lbar_1 x_2 Lbar_2 ... x_w Lbar_w (mode products, Sec. 2.3); the
 * other lines apply unchanged.
 * params: host array [n_params] of device pointers, float32, contiguous
 *         row-major with the shapes given at create; updated in place.
 * grads:  host array [n_params] of device pointers, float32 or bfloat16 per
 *         grad_dtype, same shapes; read only.
 * Asynchronous on `stream` (except refresh steps under SHAMPOO_ROOT_NEWTON, see
 * root_method).  Recorded into a graph (stream capture), a step keeps the pointers, lr and step number that it was
 * given: replays work on those tensors, whatever eager steps come between them.
 * With bf16 gradients the factor update of the first steps, while a factor has summed fewer than
 * four times as many gradient columns as it has rows, adds up in float64 (the later ones in the
 * float32 accumulators of the matrix cores): a root taken from such a young factor weights its
 * smallest eigenvalues most.  If a launch fails (SHAMPOO_ERR_HIP) the state is partly updated
 * and `step` does not count as taken.  A factor whose eigendecomposition is not finite keeps its
 * previous root (Sec. 3.2.3); such events are counted, see shampoo_status.
 */
int shampoo_step(shampoo_opt *opt, void *const *params, const void *const *grads,
                 float lr, int64_t step, void *stream);

/* State selectors for shampoo_get. */
enum {
  SHAMPOO_GET_L = 0,      /* m x m float32 (m floats, the diagonal, where that factor is diagonal) */
  SHAMPOO_GET_R = 1,      /* n x n (n)       */
  SHAMPOO_GET_LINV = 2,   /* m x m (m)       */
  SHAMPOO_GET_RINV = 3,   /* n x n (n)       */
  SHAMPOO_GET_A = 4,      /* m x n (block) or len (1-D parameter, block = 0) */
  SHAMPOO_GET_M = 5,      /* same shape as A; error if momentum == 0         */
  SHAMPOO_GET_PSH = 6,    /* m x n: last Lbar G Rbar                         */
  SHAMPOO_GET_NORMS = 7,  /* 2 floats: ||P_graft||_F^2, ||P_shampoo||_F^2 of the last step */
  SHAMPOO_GET_GF = 8,     /* same shape as A: filtered gradient; error if beta1 == 0       */
  SHAMPOO_GET_L2 = 9,     /* tensor blocks of order 3 or 4: the factor of the second dimension, n x n */
  SHAMPOO_GET_L2INV = 10, /* and its root                                                    */
  SHAMPOO_GET_L3 = 11,    /* tensor blocks of order 4: the factor of the third dimension, d3 x d3 */
  SHAMPOO_GET_L3INV = 12  /* and its root                                                    */
};
/* For a block m x n x d3 (x d4) of a tensor parameter: L / LINV belong to the first dimension
 * (m x m), R / RINV to the last one, L2 / L2INV and L3 / L3INV to those between; A, M, PSH,
 * GF are the dense block. */

/*
 * Copy one piece of state of block `block` (row-major index inside parameter
 * `param`) into dst (device pointer, dense row-major float32, `bytes` must
 * equal the size listed above).  Asynchronous on `stream`.
 */
int shampoo_get(shampoo_opt *opt, int32_t param, int32_t block, int32_t which,
                void *dst, size_t bytes, void *stream);

/*
 * Synchronises `stream` and reports (host pointers, each may be NULL):
 * the number of root refreshes performed, and the total number of factors
 * whose refresh was skipped because the factor or its spectrum was not finite.
 */
int shampoo_status(shampoo_opt *opt, void *stream, int64_t *n_refreshes,
                   int64_t *n_failed_roots);

/* Per-stage device timing (HIP events on the step's stream). */
enum {
  SHAMPOO_STAGE_FACTOR = 0,   /* both symmetric rank-k factor updates       */
  SHAMPOO_STAGE_GRAFT = 1,    /* grafting state + graft norm                */
  SHAMPOO_STAGE_ROOT = 2,     /* root-inverse refresh                       */
  SHAMPOO_STAGE_PRECOND = 3,  /* T = Lbar G (diagonal Shampoo: the whole Lbar G Rbar) */
  SHAMPOO_STAGE_UPDATE = 4,   /* rescale + momentum + parameter update      */
  SHAMPOO_STAGE_DIAG = 5,     /* 1-D parameters                             */
  SHAMPOO_STAGE_FUSED = 6,    /* blocks <= 128 x 128 on steps without refresh: factor update,
                                 grafting, preconditioning and update in one kernel */
  SHAMPOO_STAGE_PRECOND2 = 7, /* P = T Rbar, with the sums of squares of P  */
  SHAMPOO_STAGE_COUNT = 8
};
/* enable != 0: later steps record events around each stage (small overhead). */
int shampoo_set_timing(shampoo_opt *opt, int32_t enable);
/*
 * Synchronises the recorded events and returns, for `stage`, the summed
 * milliseconds and the number of timed intervals since the last call for that
 * stage (host pointers).  Resets that stage's record.
 */
int shampoo_get_timing(shampoo_opt *opt, int32_t stage, double *ms_total, int64_t *intervals);

/* Frees the host-side handle only (the workspace belongs to the caller). */
int shampoo_destroy(shampoo_opt *opt);

/*
 * Stand-alone batched root inverse (the framed box of Sec. 3.2.1):
 *   lambda, Q = eigh(A_i);  lambda' = lambda - min(lambda_min, 0) + epsilon;
 *   X_i = Q diag(lambda'^(-r)) Q^T               for i = 0 .. batch-1.
 * a:      device, batch dense row-major symmetric n x n float32 matrices (read only)
 * x:      device, batch n x n float32 outputs (may not alias a)
 * lambda: device, batch x n float32 eigenvalues in the solver's order
 *         (unsorted), or NULL
 * workspace: device, 256-byte aligned, at least
 *         shampoo_root_inverse_workspace_bytes(n, batch) bytes: what the faster path without
 *         eigenvectors takes (128 < n <= 2048; 33 MB a matrix at n = 1024, chunks of at most
 *         4 GiB).  Where lambda is given, shampoo_root_inverse_warm_workspace_bytes(n, batch)
 *         are enough for n > 128 (half of it)
 * failed: device int32[batch] set to 1 where A_i or its spectrum is not
 *         finite (X_i is then left untouched), else 0; or NULL
 * Asynchronous on `stream`.
 */
size_t shampoo_root_inverse_workspace_bytes(int32_t n, int32_t batch);
int shampoo_root_inverse(const float *a, int32_t n, int32_t batch, float epsilon, float r,
                         float *x, float *lambda, int32_t *failed,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * shampoo_root_inverse with a warm start (n > 128 only, else SHAMPOO_ERR_UNSUPPORTED): the
 * eigenvectors are kept in the caller's array qt between calls.
 * qt:     device, batch x np x np float32, np = n rounded up to a multiple of 64, aligned to 16
 *         bytes (else SHAMPOO_ERR_WORKSPACE); rows are eigenvectors.  start == 0: a cold solve (qt is overwritten).  start != 0: qt holds the
 *         result of an earlier call on matrices close to a (the same factors some steps
 *         earlier): the solve starts from W = qt a qt^T (float64 sums), and qt is updated.
 *         A matrix that fails (see `failed`) leaves its part of qt as it was.
 * sweeps: device int32[batch] or NULL: the number of Jacobi sweeps in which anything rotated
 *         (the last one of a solve never does: it finds every pair below the threshold).
 * Everything else as shampoo_root_inverse; the workspace has no room for the path without eigenvectors.
 */
size_t shampoo_root_inverse_warm_workspace_bytes(int32_t n, int32_t batch);
int shampoo_root_inverse_warm(const float *a, int32_t n, int32_t batch, float epsilon, float r,
                              float *x, float *lambda, int32_t *failed, float *qt, int32_t start,
                              int32_t *sweeps, void *workspace, size_t workspace_bytes, void *stream);

/*
 * shampoo_root_inverse for callers that cannot allocate device memory or must not see an
 * allocation happen: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments and results as shampoo_root_inverse without the
 * workspace: the solver's working arrays live in a fixed array of
 * SHAMPOO_STATIC_SCRATCH_BYTES inside the library's device image (one copy per GPU, held
 * until the process ends), and matrices are processed as many at a time as fit there
 * (n = 2048: one, n = 1024: four; n <= 128 needs no scratch at all).  The call allocates
 * nothing, creates no streams and enqueues kernels only (no memset nodes), all on `stream`.
 * n > SHAMPOO_STATIC_MAX_N: SHAMPOO_ERR_UNSUPPORTED, nothing enqueued.
 * Every call on a GPU uses that GPU's one array: calls whose work overlaps on one GPU (two
 * streams, two threads) race; the caller orders them.
 */
#define SHAMPOO_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
#define SHAMPOO_STATIC_MAX_N 2048
int shampoo_root_inverse_static(const float *a, int32_t n, int32_t batch, float epsilon, float r,
                                float *x, float *lambda, int32_t *failed, void *stream);

/*
 * Stand-alone batched coupled inverse Newton iteration (Sec. 3.2.1, item 2):
 *   A_i = a_i + epsilon I,  c = (2 ||A_i||_F / (p + 1))^(1/p),  X_0 = I / c,  M_0 = A_i / c^p,
 *   X_{k+1} = X_k T_k,  M_{k+1} = T_k^p M_k,  T_k = ((p + 1) I - M_k) / p,
 * ended per matrix at the first k with ||M_k - I||_inf < tolerance, at k = max_iterations,
 * or when the norm has reached the floor of float32 arithmetic (below 0.1 and no longer
 * halving).  M_k itself is not formed where ||M_{k-1} - I||_inf^2 < tolerance, which bounds its norm
 * (in exact arithmetic): the matrix ends at that k.
 * x_i = X_k approximates A_i^(-1/p).
 * a:          device, batch dense row-major symmetric n x n float32 matrices (read only)
 * p:          1, 2, 4 or 8 (else SHAMPOO_ERR_UNSUPPORTED)
 * x:          device, batch n x n float32 outputs (may not alias a)
 * iterations: device int32[batch], the k at which each matrix ended, or NULL
 * failed:     device int32[batch] set to 1 where A_i or an iterate is not finite (x_i is
 *             then left untouched), else 0; or NULL
 * workspace:  device, 256-byte aligned, at least
 *             shampoo_root_inverse_newton_workspace_bytes(n, batch) bytes
 * Asynchronous on `stream`; no host synchronisation inside.
 */
size_t shampoo_root_inverse_newton_workspace_bytes(int32_t n, int32_t batch);
int shampoo_root_inverse_newton(const float *a, int32_t n, int32_t batch, float epsilon, int32_t p,
                                float tolerance, int32_t max_iterations, float *x,
                                int32_t *iterations, int32_t *failed,
                                void *workspace, size_t workspace_bytes, void *stream);

/* The order in which the Jacobi eigensolver of the refresh (Sec. 3.2.1: the root inverse by
 * symmetric eigendecomposition) visits index pairs: pair `k` (0 <= k < s / 2) of round `round`
 * (0 <= round < s - 1) of a sweep over s indices, written to *p < *q.  Every round is a
 * perfect matching and the s - 1 rounds cover every pair once.  halves = 0: the plain
 * tournament (any even s >= 2, the solver for n <= 128).  halves = 1: the order of the
 * 64 x 64 pivots of the blocked solver (s / 2 a power of two, s >= 4): rounds 0 .. s / 2 - 1
 * pair the first half of the indices with the second, the remaining rounds pair within the
 * halves.  halves = 2: the order of the block columns of the blocked solver when their number
 * s is a multiple of 4: indices 2 S and 2 S + 1 form a super-column, round 0 pairs the members
 * of every super-column, and rounds 1 + 2 R, 2 + 2 R are the two rounds of the meetings (S, T)
 * of round R of the super-columns' own tournament: (2 S, 2 T), (2 S + 1, 2 T + 1), then
 * (2 S, 2 T + 1), (2 S + 1, 2 T); pairs 2 K and 2 K + 1 of both rounds belong to meeting K.
 * Host only, no device work; SHAMPOO_ERR_NULL / SHAMPOO_ERR_SHAPE on bad arguments. */
int shampoo_jacobi_pair(int32_t s, int32_t halves, int32_t round, int32_t k, int32_t *p, int32_t *q);

/* ------------------------------------------------------------------------------------------
 * Operators of a training pass that make the gradients of a step.  Each is asynchronous on `stream` and works on the
 * current device; pointers are device pointers unless a line says otherwise; argument errors are returned before any work
 * is enqueued.  Matrices are row-major, a leading dimension (ld..., in elements) is the distance of their rows.  dtype codes
 * are SHAMPOO_GRAD_F32 and SHAMPOO_GRAD_BF16.  Sums, norms and softmax statistics are float32.  The same call on the
 * same inputs gives the same bits.
 * ------------------------------------------------------------------------------------------ */

/* How a weight lies in memory: rows of inputs for every output, or the other way round. */
enum { SHAMPOO_OUT_IN = 0, SHAMPOO_IN_OUT = 1 };

/*
 * Softmax cross entropy of a linear layer over many classes, and its gradients:
 *   z = x w^T + bias,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_{i,t_i},
 *   g_iv = scale weight_i (exp(z_iv - lse_i) - [v = t_i]),  dx = g w,  dw = g^T x,  dbias_v = sum_i g_iv
 * (the gradients of scale sum_i weight_i loss_i).  For gradients the logits of a piece of the rows at a time lie in the workspace,
 * with what is made of them 2 to 10 bytes each: as many rows as fit in 4 GiB, at least 256, so all logits of a call that fits.
 * The loss alone keeps none of them.
 * A row whose target is outside 0 ... classes - 1 is ignored: loss 0 and g_i = 0 whatever its logits are (its row of x
 * still is a factor of dw: 0 times a value that is not finite is not 0).  bias may mask classes by -infinity: their
 * probability is 0 and so is their gradient; a masked target has loss +infinity and, as p = 0, the gradient -scale weight_i; a row with every class
 * masked has g_i = 0.  The loss and p are those of z - max z: a common offset of the logits takes nothing but the bits that it takes of z.
 */
typedef struct {
  int64_t rows;           /* >= 0                                                              */
  int32_t features;       /* 1 ... 65536                                                       */
  int32_t classes;        /* 1 ... 4194304; at most 2^23 blocks of 128 features by 128 classes  */
  int32_t dtype;          /* of x, w and dx.  bf16: z from exact products; g is rounded to bf16 for the products of dx
                             and bf16 dw, and has float32 accuracy (three bf16 terms) for float32 dw.  float32: all
                             products to float32 accuracy (three terms per value, six products) */
  int32_t grad_dtype;     /* of dw; float32 x: float32                                         */
  int32_t w_layout;       /* of w and dw: SHAMPOO_OUT_IN [classes][features], SHAMPOO_IN_OUT [features][classes] */
  int32_t has_bias;       /* != 0: bias is given                                              */
  int32_t gradients;      /* != 0: dx, dw (and dbias) are wanted; 0: the loss alone             */
  int64_t ldx, ldw, lddx, lddw;
} shampoo_cross_entropy;
/* bytes of workspace; 0 if c is invalid */
size_t shampoo_linear_cross_entropy_workspace_bytes(const shampoo_cross_entropy *c);
/*
 * x [rows][features], w per w_layout: 16-byte aligned (else SHAMPOO_ERR_UNSUPPORTED); bias [classes] float32 or NULL;
 * targets [rows] int64; weight [rows] float32 or NULL (all 1); loss [rows] float32, not weighted;
 * dx [rows][features], dw like w, dbias [classes] float32: overwritten; each may be NULL where it is not wanted.
 * workspace: 256-byte aligned.
 */
int shampoo_linear_cross_entropy(const shampoo_cross_entropy *c, const void *x, const void *w, const float *bias,
                                 const int64_t *targets, const float *weight, float scale, float *loss,
                                 void *dx, void *dw, float *dbias, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Activation checkpoints in 8 bits.  A matrix is kept as codes q (int8) and one exponent s per row and group of 32
 * neighbouring columns: x ~ q 2^s with q = rint(x 2^-s) and the smallest s for which the group's largest |x| rounds to at
 * most 127.  Groups below 2^-100 are kept as zeros; a group with an infinity, a NaN or a value from 255 2^120 on
 * reads NaN as a whole.  33 bytes per 32 values (columns are padded to a multiple of 32).
 * `packed` is opaque: 256-byte aligned memory of shampoo_checkpoint_bytes(rows, cols) bytes (0 if they are invalid:
 * rows < 0, cols < 1 or above 1048576).
 */
enum { SHAMPOO_ACT_NONE = 0, SHAMPOO_ACT_RELU = 1, SHAMPOO_ACT_GELU = 2 /* with erf */, SHAMPOO_ACT_SILU = 3 };
size_t shampoo_checkpoint_bytes(int64_t rows, int32_t cols);
int shampoo_checkpoint_pack(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t ldx,
                            void *packed, size_t packed_bytes, void *stream);
/* y = a(x) of what the checkpoint holds */
int shampoo_checkpoint_unpack(const void *packed, size_t packed_bytes, int64_t rows, int32_t cols, int32_t activation,
                              void *y, int32_t dtype, int64_t ldy, void *stream);
/* dx = dy a'(x) (ReLU: 0 at 0); dx may be dy */
int shampoo_checkpoint_activation_grad(const void *packed, size_t packed_bytes, int64_t rows, int32_t cols, int32_t activation,
                                       const void *dy, int32_t dtype, int64_t lddy, void *dx, int64_t lddx, void *stream);
/*
 * Gradient of a linear layer y = a(x) W + b from the checkpoint of x [rows][in] and dy [rows][out]:
 *   dW = a(x)^T dy (SHAMPOO_IN_OUT; SHAMPOO_OUT_IN: transposed),  db = column sums of dy (float32; NULL: not wanted).
 * dtype: of dy (16-byte aligned, else SHAMPOO_ERR_UNSUPPORTED).  Float32 dy: products to float32 accuracy, dw float32.
 * bf16 dy: x and dy enter as they are; a(x), where an activation is given, rounded to bf16 for bf16 dw, with float32 accuracy for
 * float32 dw.  An infinity in float32 dy reaches its results as in the sum; in bf16 dy it makes them infinite or NaN.
 * in <= 65536, out <= 4194304, at most 2^23 blocks of 128 by 128.
 */
size_t shampoo_checkpoint_weight_grad_workspace_bytes(int64_t rows, int32_t in, int32_t out, int32_t activation, int32_t dtype,
                                                      int64_t lddy, int32_t grad_dtype, int32_t want_bias);
int shampoo_checkpoint_weight_grad(const void *packed, size_t packed_bytes, int64_t rows, int32_t in, int32_t activation,
                                   const void *dy, int32_t dtype, int32_t out, int64_t lddy, void *dw, int32_t grad_dtype,
                                   int32_t w_layout, int64_t lddw, float *db, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Residual sum with the norms after and before a block, its gate and its scale:
 *   u = norm_post(f),  r_out = r + scale gate u,  h = norm_pre(r_out),
 *   norm(x) = (x - mean) / sqrt(mean of its squares + epsilon) w + b   (SHAMPOO_NORM_RMS: without mean and b).
 * Sums and norms in float32 on values that are not rounded between the steps.
 */
enum { SHAMPOO_NORM_NONE = 0, SHAMPOO_NORM_RMS = 1, SHAMPOO_NORM_LAYER = 2 };
typedef struct {
  int64_t rows;            /* >= 0                                                             */
  int32_t cols;            /* 1 ... 16384                                                       */
  int32_t dtype;           /* of r, f, r_out, h and their gradients                              */
  int32_t post, pre;       /* SHAMPOO_NORM_*; NONE: u = f, no h                                  */
  int64_t gates;           /* 0: no gate; otherwise gate is [gates][cols] and every rows / gates rows share one (gates divides rows) */
  float epsilon, scale;    /* epsilon >= 0                                                       */
  const float *w_post, *b_post, *gate, *w_pre, *b_pre; /* [cols] float32; w of every norm that is there, b of a layer norm or NULL */
} shampoo_residual_norm;
/* r, f, r_out, h: [rows][cols], dense (ld = cols unless ld is given); r_out may be r.  packed_r, packed_f: where checkpoints of r and f are written
 * (both or neither), as by shampoo_checkpoint_pack. */
int shampoo_residual_norm_forward(const shampoo_residual_norm *c, const void *r, int64_t ldr, const void *f, int64_t ldf,
                                  void *r_out, int64_t ld_r_out, void *h, int64_t ldh,
                                  void *packed_r, void *packed_f, size_t packed_bytes, void *stream);
/*
 * Gradients from those of r_out (dr_out, NULL: 0) and of h (dh; NULL where there is no h).  r and f as the forward call had them: packed != 0:
 * their checkpoints, shampoo_checkpoint_bytes(rows, cols) bytes each (ldr, ldf ignored), otherwise the matrices.  dr may be dr_out, df may be dh.  dgate [gates][cols], dw_post, db_post,
 * dw_pre, db_pre [cols]: float32, each NULL where it is not wanted.
 */
size_t shampoo_residual_norm_backward_workspace_bytes(const shampoo_residual_norm *c);
int shampoo_residual_norm_backward(const shampoo_residual_norm *c, int32_t packed, const void *r, int64_t ldr, const void *f, int64_t ldf,
                                   const void *dr_out, int64_t ld_dr_out, const void *dh, int64_t ld_dh,
                                   void *dr, int64_t ld_dr, void *df, int64_t ld_df, float *dgate, float *dw_post, float *db_post,
                                   float *dw_pre, float *db_pre, void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------------
 * Operators on given logits: what a program learns from, scores with or answers with where a product has made them.  Conventions as above.
 * ------------------------------------------------------------------------------------------ */

/*
 * Of every row of logits z, with x = (z - max z) / T and log p = x - log sum exp x:
 *   log_probs_j = log p of given token j,  entropy = -sum_v p_v log p_v,  and the `top` most probable tokens with their log p.
 * The order of tokens is that of the logits as they are given; of equal ones the lower token comes first.
 * A given token outside 0 ... classes - 1 is ignored: log_probs 0, no gradient.  -infinity masks a token: its log p is -infinity, it adds nothing to the
 * entropy and is none of the most probable; where fewer than `top` are left, the rest of top_tokens is -1 and of top_log_probs -infinity.  A row with nothing
 * left has entropy 0.  A NaN or +infinity makes all log p of its row and its entropy NaN; top_tokens are in the order of what is not NaN.
 */
typedef struct {
  int64_t rows;               /* 0 ... 2^31 - 1                                                   */
  int32_t classes;            /* 1 ... 4194304                                                    */
  int32_t tokens;             /* given tokens of a row, 0 ... 64; the same one may be given twice */
  int32_t top;                /* 0 ... 64                                                         */
  int32_t dtype;              /* of the logits and of their gradient                              */
  float inverse_temperature;  /* 1 / T, > 0, at most 2e38                                        */
  int64_t ld;                 /* of the logits, >= classes                                        */
} shampoo_logits;
size_t shampoo_log_probs_workspace_bytes(const shampoo_logits *c);  /* 0 also if c is invalid */
/* tokens [rows][c->tokens] int64 (log_probs alike, float32; both may be NULL where there are none), entropy [rows] float32, top_tokens [rows][top] int64,
 * top_log_probs [rows][top] float32 (NULL where top is 0), statistics [rows][4] float32, 16-byte aligned: what the gradient needs of a row.
 * workspace: 256-byte aligned, may be NULL where none is needed. */
int shampoo_log_probs(const shampoo_logits *c, const void *logits, const int64_t *tokens, float *log_probs, float *entropy, int64_t *top_tokens,
                      float *top_log_probs, float *statistics, void *workspace, size_t workspace_bytes, void *stream);
/*
 * Gradient of the logits from those of log_probs (a, [rows][c->tokens] float32, or NULL: none) and of the entropy (b, [rows] float32, or NULL):
 *   dz_v = (sum_j a_j [v = t_j] - p_v (sum_j a_j + b (log p_v + entropy))) / T
 * c, logits, tokens and statistics as the forward call had and left them.  d_logits [rows][classes] may be the logits themselves (the same
 * leading dimension then).  A given token that is masked has p = 0 and the gradient a / T; a row with nothing left, or whose coefficients are all zero,
 * has the gradient 0.
 */
int shampoo_log_probs_grad(const shampoo_logits *c, const void *logits, const int64_t *tokens, const float *statistics, const float *d_log_probs,
                           const float *d_entropy, void *d_logits, int64_t ld_d_logits, void *stream);

/* ------------------------------------------------------------------------------------------
 * All tensors of a model at once: the norm of the gradients, and an AdamW step (for parameters that have no factors worth keeping: vectors, embeddings).
 * ------------------------------------------------------------------------------------------ */

/*
 * norm = sqrt of the sum of the squares of all elements of n gradients, norms[i] (or NULL) that of gradient i; sums in 64 bits.
 * grads: host array [n] of device pointers, contiguous; numel: host array [n], >= 0 each, at most 2^39 together (NULL is a pointer for none).  norm, norms: float32 device
 * pointers.  NaN and infinities reach the results, and so does a norm that float32 does not hold.
 */
size_t shampoo_gradient_norm_workspace_bytes(int32_t n, const int64_t *numel);
int shampoo_gradient_norm(int32_t n, const void *const *grads, const int64_t *numel, int32_t dtype, float *norm, float *norms, void *workspace,
                          size_t workspace_bytes, void *stream);

/*
 * AdamW (decoupled weight decay, bias correction):
 *   g <- g min(1, max_norm / norm)  (where a norm is given)
 *   m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2,  t = step + 1
 *   w <- (1 - lr weight_decay) w - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + epsilon)
 * in float32.  bf16 parameters are rounded up with the probability of what is left over (an update is mostly less than half a step of theirs); the
 * random numbers are a mix of the element's index and the step's number, so that the same call gives the same bits.
 * state_bits = 8: 128 neighbouring elements of a tensor share a power of two; m has a sign, 4 bits of exponent and 3 of mantissa, v 5 and 3, rounded the same way (v > 0
 * never to 0).  Groups whose largest is below 2^-100 are kept as zeros; one with an infinity, a NaN or a value from 2^127 on reads NaN as a whole.
 */
typedef struct shampoo_adamw shampoo_adamw; /* opaque, owned by the library; no two calls on the same one at once */
typedef struct {
  int32_t n_params;        /* 1 ... 2^20                                            */
  const int64_t *numel;    /* host [n_params]: elements, >= 0 each, at most 2^39 together */
  const int32_t *decay;    /* host [n_params]: != 0 where weight_decay applies; NULL: everywhere */
  int32_t state_bits;      /* 32 or 8                                               */
  int32_t param_dtype;     /* SHAMPOO_GRAD_F32 or SHAMPOO_GRAD_BF16                 */
  int32_t grad_dtype;
  int32_t device;          /* HIP device ordinal: the current one in every call     */
  double beta1, beta2;     /* in [0, 1)                                             */
  double epsilon;          /* 1e-12 ... 1e12                                        */
  double weight_decay;     /* >= 0                                                  */
} shampoo_adamw_config;
/* 0 if cfg is invalid.  With 32 bits the workspace begins with m, [all elements] float32, one parameter behind the other; v follows at the next multiple of 256 bytes. */
size_t shampoo_adamw_workspace_bytes(const shampoo_adamw_config *cfg);
/* workspace: 256-byte aligned; holds all state and stays allocated until shampoo_adamw_destroy.  m = v = 0; `stream` is synchronised before returning. */
int shampoo_adamw_create(const shampoo_adamw_config *cfg, void *workspace, size_t workspace_bytes, void *stream, shampoo_adamw **out);
/*
 * params, grads: host arrays [n_params] of device pointers, contiguous, aligned to their elements; params are updated in place.  copies: NULL, or bf16 tensors [n_params]
 * that get the updated float32 parameters, rounded to the nearest.  step: 0-based, strictly increasing.  norm: NULL, or a device pointer to the norm of these gradients
 * (max_norm > 0, may be infinite); where it is not finite the call changes nothing on the device, and the step counts as taken.
 * Recorded into a graph, a step keeps the pointers, lr and step number that it was given.
 * A step of many tensors is several launches.  If one fails (SHAMPOO_ERR_HIP) the step does not count as taken, but tensors of earlier launches have had it: their parameters, states and
 * copies are to be restored before it is tried again, which would otherwise apply it to them twice.
 */
int shampoo_adamw_step(shampoo_adamw *opt, void *const *params, const void *const *grads, void *const *copies, double lr, int64_t step,
                       const float *norm, float max_norm, void *stream);
/* m and v of all parameters, one behind the other without gaps ([all elements] each, of `dtype`; bf16 holds what 8 bits hold), and the other way round from float32 (8 bits: rounded to
 * the nearest). */
int shampoo_adamw_get(shampoo_adamw *opt, void *m, void *v, int32_t dtype, void *stream);
int shampoo_adamw_set(shampoo_adamw *opt, const float *m, const float *v, void *stream);
/* Frees the host-side handle only. */
int shampoo_adamw_destroy(shampoo_adamw *opt);

/* Static, NUL-terminated description of a return code. */
const char *shampoo_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SHAMPOO_H */
