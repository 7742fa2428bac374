/*
 * mi355svm.h -- C ABI of a kernel-SVM dual solver for one AMD Instinct
 * MI355X (gfx950).
 *
 * The library trains C-SVC and eps-SVR models with the linear, polynomial,
 * RBF or sigmoid kernel by the working-set decomposition of Wang et al.,
 * "Rgtsvm: Support Vector Machines on a GPU in R" (arXiv 1706.05544), and
 * evaluates their decision function.
 * Everything that computes runs in hand-written HIP kernels; this header
 * only moves pointers and sizes.
 *
 * Problem (Section 3, Eq. 2):
 *     min_a  1/2 a^T Q a + p^T a   s.t.  y^T a = 0,  0 <= a_t <= C,
 *     Q_ts = y_t y_s K(x_smp(t), x_smp(s)),  K one of the kernels below.
 *   C-SVC:   one variable per sample, y_t = label in {+1,-1}, p_t = -1.
 *   eps-SVR: two variables per sample (Section 3, "positive and negative
 *            copy"; Eq. 1): copy (i,+) with y = +1, p = eps - z_i and copy
 *            (i,-) with y = -1, p = eps + z_i.
 * Decision function: D(x) = sum_i c_i K(x_i, x) + b with c_i = y_i a_i
 * (C-SVC) or c_i = a_(i,+) - a_(i,-) (eps-SVR).
 *
 * Conventions shared by every call:
 *   - status: 0 OK, > 0 warning (result valid), < 0 error (nothing written,
 *     *out set to NULL where there is one).  svm_last_error() returns a
 *     thread-local message for the last non-OK status.
 *   - All argument validation happens before any device call, so invalid
 *     arguments are reported even on a machine without a GPU.
 *   - Host inputs are read during the call and copied once to the device;
 *     they are never retained.  Device inputs (on_device = 1) are borrowed
 *     for the duration of the call and used on params->stream (dense ones
 *     with ld = d, d a multiple of 4 and 16-byte aligned values are read
 *     in place, not copied; they are never written).
 *   - Calls are synchronous: they return after the device work they queued
 *     has finished.  Models and solvers are not shared between threads
 *     without external locking.
 */
#ifndef MI355SVM_H
#define MI355SVM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SVM_OK = 0,
    SVM_W_MAX_ITER = 1,        /* max_iter reached; model valid, gap > tol */
    SVM_W_NOT_CONVERGED = 2,   /* the gap met tol on the incrementally
                                  updated responses but not, after 3
                                  re-runs, on responses recomputed from
                                  alpha; model valid, gap (recomputed) > tol */
    SVM_E_INVALID = -1,        /* bad argument (message says which) */
    SVM_E_UNSUPPORTED = -2,    /* valid but not implemented (e.g. kernel) */
    SVM_E_NOMEM = -3,          /* device or host allocation failed */
    SVM_E_DEVICE = -4,         /* no usable GPU, or a HIP runtime error */
    SVM_E_INTERNAL = -5
} svm_status;

typedef enum { SVM_C_SVC = 0, SVM_EPS_SVR = 1 } svm_type;

/* The four kernels of Section 3's list, in the e1071 (LIBSVM)
 * parameterisation (the paper names them without formulas):
 *   linear      K(u,v) = u.v
 *   polynomial  K(u,v) = (gamma u.v + coef0)^degree
 *   RBF         K(u,v) = exp(-gamma |u - v|^2)
 *   sigmoid     K(u,v) = tanh(gamma u.v + coef0)
 * Kernel values are computed in fp32 from an fp32 dot product; the
 * sigmoid kernel is not positive semidefinite in general (a pair of
 * non-positive curvature gets the floor 1e-12, as in LIBSVM). */
typedef enum {
    SVM_KERNEL_LINEAR = 0,
    SVM_KERNEL_POLY = 1,
    SVM_KERNEL_RBF = 2,
    SVM_KERNEL_SIGMOID = 3
} svm_kernel;

typedef enum { SVM_DENSE = 0, SVM_CSR = 1 } svm_layout;

/* A feature matrix of n rows and d columns.
 *   dense: values[i*ld + k], fp32, ld >= d.
 *   CSR:   row_ptr[0..n] (row_ptr[0] = 0, nondecreasing, row_ptr[n] = nnz),
 *          col_idx[nnz] sorted and unique within each row, in [0, d),
 *          values[nnz].
 * on_device = 1: every pointer is device memory of params->device. */
typedef struct {
    int32_t layout;
    int32_t on_device;
    int64_t n, d;
    const float *values;
    int64_t ld;
    const int64_t *row_ptr;
    const int32_t *col_idx;
    int64_t nnz;
} svm_matrix;

typedef struct {
    int32_t type;          /* svm_type */
    int32_t kernel;        /* svm_kernel */
    double C;              /* > 0 */
    double epsilon;        /* >= 0, eps-SVR tube half-width */
    double gamma;          /* >= 0; 0 means 1/d (the e1071 default) */
    double tol;            /* > 0; stop when max_{I_up} v - min_{I_low} v <= tol */
    int64_t max_iter;      /* outer iterations; <= 0: max(1e7, 100 N) */
    int32_t working_set;   /* q, even, in [2, 64]; 16 as in Section 3 */
    int32_t device;        /* HIP device ordinal */
    int64_t cache_bytes;   /* kernel-row cache budget; < 0 off; 0 default:
                              the whole K if it fits a quarter of the free
                              device memory, else a quarter of it, at most
                              8 GiB (the memory is kept for the next
                              training: svm_cache_release).  When the budget
                              holds the whole K of a dense problem, n^2 d is
                              at most 6e10 and 4 n^2 bytes at most 7.2e9 for
                              each training that shares K (one: n <= 42426;
                              n <= 61440 in any case), K is computed at once
                              and the outer iterations run many to a launch
                              (working sets of at most 16; not with profile
                              or fused, nor a max_iter too small to gain
                              from it); the trainings of a one-vs-rest model
                              or a cross-validation then run side by side
                              (each train_ms spans all of them, up to the end
                              of its own problem's finish).
                              A single training to which K would cost much
                              does its first iterations without, as does a
                              warm start.  Results are the same bits */
    void *stream;          /* hipStream_t; NULL: a stream of the library */
    int32_t check_every;   /* outer iterations between host polls (0: 64;
                              fewer near convergence, down to an eighth,
                              from the rate at which the gap falls) */
    double inner_ratio;    /* subproblem stops at local gap <= max(ratio *
                              global gap, tol/2); 0: 0.3 */
    int32_t max_inner;     /* subproblem step cap; 0: 8 q */
    int32_t profile;       /* 1: time the row/update kernel with events
                              (a sample: the launches of one chunk of
                              check_every iterations in four); 2: also the
                              select/solve kernel of those iterations (a
                              timed launch of it costs the loop ~5 us) */
    double coef0;          /* polynomial and sigmoid offset (finite; 0) */
    int32_t degree;        /* polynomial degree, in [1, 64] (3) */
    int32_t scale;         /* 1: standardise each feature (and eps-SVR
                              targets) to mean 0 and sample sd 1 before
                              training, as e1071 does; dense X only; the
                              model applies the same statistics to the rows
                              it predicts (0: inputs used as given) */
    const double *alpha0;  /* warm start for svm_train: N host values (n for
                              C-SVC, 2n for eps-SVR: copy (i,+) then (i,-))
                              with 0 <= a <= C and y^T a = 0 (checked to
                              1e-9 C N when y is in host memory); the solve
                              starts there instead of at 0.  NULL: 0.  Not
                              for one-vs-rest or cross-validation */
    int32_t lockstep;      /* one-vs-rest, cross-validation and svm_tune:
                              up to this many binary problems (classes,
                              folds; in svm_tune also of different grid
                              points) train in lockstep, their outer
                              iterations together, one selection launch (a
                              block per problem) and one pass over X per
                              iteration; each problem's result is the one
                              it has when trained alone without the row
                              cache, which lockstep does not use.  In [0, 4];
                              0 or 1: one problem after another.  Fewer
                              when the working-set rows of more would not
                              fit the row kernel's LDS (2 at d = 784).  > 1
                              needs dense X and working_set = 16, else
                              SVM_E_UNSUPPORTED.  No effect on svm_train.
                              train_ms of a problem then spans its group's
                              run (the groups' problems overlap in time).
                              Not used where the whole K is computed at
                              once into the cache (see cache_bytes, whose
                              memory is then taken and kept; < 0: lockstep
                              all the same) */
    int32_t fused;         /* 1: every outer iteration as one launch, in
                              which each block merges the selection
                              candidates and solves the subproblem itself
                              while its rows stream (Section 3's loop);
                              dense X and working_set <= 16 only, no row
                              cache.  0 (default): selection and row update
                              as two launches.  The result is the same bit
                              for bit; one launch has been the slower so far
                              (its blocks' selection chains run longer than
                              the stream they hide) */
} svm_params;

/* Result of a k-fold cross-validation. */
typedef struct {
    int32_t folds;
    int32_t status;        /* SVM_OK or SVM_W_MAX_ITER (some fold) */
    int64_t n;             /* rows, each predicted by the model of the folds
                              it is not in */
    int64_t iters;         /* outer iterations over all trainings */
    double accuracy;       /* C-SVC / one-vs-rest: share of correct labels */
    double mse;            /* eps-SVR: mean squared error */
    double scc;            /* eps-SVR: squared correlation of D and targets */
    double error;          /* 1 - accuracy (C-SVC), or mse (eps-SVR) */
    int64_t kernel_rows;   /* kernel rows used over all trainings */
    /* params->profile = 1: the row/update launches that computed rows from
     * X, over all trainings (as in svm_model_info) */
    double row_kernel_ms;
    int64_t row_kernel_launches;
    double row_kernel_bytes;
} svm_cv_stats;

/* Per-output statistics of a trained model. */
typedef struct {
    int32_t type;          /* svm_type */
    int32_t n_outputs;     /* 1, or the number of classes (one-vs-rest) */
    int64_t n_train;       /* training samples */
    int64_t n_features;
    int64_t n_sv;          /* support rows stored (union over outputs) */
    double gamma;          /* resolved gamma */
    int32_t kernel;        /* svm_kernel of the model */
    int32_t degree;        /* its polynomial degree */
    double coef0;          /* its polynomial / sigmoid offset */
    /* the rest refers to the output asked for */
    int32_t status;        /* SVM_OK or SVM_W_MAX_ITER */
    int64_t n_sv_output;   /* samples with non-zero coefficient */
    int64_t n_bounded;     /* variables at C */
    int64_t iters;         /* outer iterations (working sets optimised) */
    double gap;            /* final m - M */
    double b;              /* bias */
    double dual_obj;       /* f(a) of Eq. 2 */
    int64_t kernel_rows;   /* kernel rows K(x_s, X) used (computed + cached) */
    int64_t cache_hits;    /* kernel rows served by the row cache */
    int64_t cache_fills;   /* kernel rows written to the row cache (K
                              computed at once: rows of samples used for the
                              first time in this training; rows served: of
                              working sets whose samples were all used
                              before) */
    double train_ms;       /* device time from solver start to model ready;
                              problems that train side by side (lockstep,
                              cache_bytes) overlap in it, so the sum over
                              the classes of a model may be several times
                              the time that it took */
    /* profile = 1: row/update kernel launches that computed the rows from X */
    double row_kernel_ms;        /* summed kernel time */
    int64_t row_kernel_launches; /* launches included in row_kernel_ms */
    int64_t row_kernel_rows;     /* rows of X processed by those launches */
    double row_kernel_bytes;     /* their algorithmic HBM bytes */
    /* profile = 1: launches served entirely from the row cache */
    double cached_kernel_ms;
    int64_t cached_kernel_launches;
    double cached_kernel_bytes;
    /* profile = 2: the select/solve kernel of the same iterations (one
       block: merge, K_BB, subproblem; latency-bound) */
    double select_kernel_ms;
    int64_t select_kernel_launches;
} svm_model_info;

typedef struct svm_model svm_model;  /* opaque, owned by the library */

/* Defaults: C-SVC, RBF, C = 1, eps = 0.1, gamma = 0 (1/d), coef0 = 0,
 * degree = 3, tol = 1e-3, working_set = 16, device 0, NULL stream. */
void svm_params_default(svm_params *p);

/* Train a binary C-SVC (y = labels, each +1 or -1, both present) or an
 * eps-SVR (y = targets z).  y has n entries in the memory space of X.
 * On success *out receives a model the caller frees with svm_model_free. */
svm_status svm_train(const svm_matrix *X, const float *y,
                     const svm_params *p, svm_model **out);

/* One-vs-rest multi-class C-SVC (Section 3, multi-class classification):
 * labels in [0, n_classes), n_classes >= 2; one binary problem per class
 * (class c against the rest), all sharing X on the device. */
svm_status svm_train_ovr(const svm_matrix *X, const int32_t *labels,
                         int32_t n_classes, const svm_params *p,
                         svm_model **out);

/* Decision values D (m x n_outputs, row-major, fp64) for the m rows of X,
 * written to `decision` in the memory space of X (caller-owned). */
svm_status svm_predict(const svm_model *m, const svm_matrix *X,
                       double *decision);

/* For callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  The
 * decision values of svm_predict (bitwise the same kernels and values) for
 * the m dense rows of X, which must be in device memory (layout SVM_DENSE,
 * on_device = 1, any ld >= d), into `decision` (device, m x n_outputs,
 * row-major fp64, caller-owned), queued on `stream` (hipStream_t; NULL:
 * the null stream) and NOT waited for: the values are there when the
 * stream's work up to this call has finished.  The call allocates nothing,
 * frees nothing and does not synchronise with the host: the rows are
 * staged, chunk by chunk, in a static array of 32 MiB per device (held by
 * each GPU the library runs on until the process ends), which every call
 * on that GPU shares, so calls that overlap in time on one GPU race.  X is
 * not checked for finite values (a non-finite row gives non-finite
 * decision values).  Errors: SVM_E_UNSUPPORTED for CSR or host rows, or a
 * row too long for the staging array (over about 8.3 million features);
 * SVM_E_INVALID for a NULL model or output or a different number of
 * features. */
svm_status svm_predict_noalloc(const svm_model *m, const svm_matrix *X,
                               double *decision, void *stream);

/* Labels: +1 / -1 (D >= 0 gives +1) for C-SVC, argmax over classes (ties to
 * the lowest class) for one-vs-rest.  eps-SVR models: SVM_E_INVALID. */
svm_status svm_predict_labels(const svm_model *m, const svm_matrix *X,
                              int32_t *labels);

svm_status svm_model_get_info(const svm_model *m, int32_t output,
                              svm_model_info *info);

/* Host copies of one output: sv_idx[n_sv_output] (training-row indices,
 * increasing) and coef[n_sv_output]; alpha[N] (N = n or 2n) may be NULL. */
svm_status svm_model_get(const svm_model *m, int32_t output, int32_t *sv_idx,
                         double *coef, double *alpha);

void svm_model_free(svm_model *m);

/* Memory management of the library, not an operation of the method.  The
 * device memory of the kernel-row cache (svm_params.cache_bytes) is kept
 * per device between trainings, one block as large as the largest cache
 * used so far on that device, and lent to one training at a time (a
 * training that finds it in use allocates its own): allocating and freeing
 * tens of GB per training would make later allocations wait while the
 * driver clears the freed memory.  This frees the kept block of `device`
 * (device < 0: of every device) unless a training holds it, and writes
 * the bytes freed to *freed (nullable).  Errors: SVM_E_INVALID for a
 * device ordinal out of range, SVM_E_DEVICE without a HIP device. */
svm_status svm_cache_release(int32_t device, int64_t *freed);

/* k-fold cross-validation (Section 3's feature list: "K-fold cross
 * validation", "accuracy or correlation, mean square error").  Give either
 * y (n labels +-1 for C-SVC, or n targets for eps-SVR) with labels = NULL,
 * or labels (n class indices in [0, n_classes)) with y = NULL for
 * one-vs-rest.  fold: n host entries in [0, k), every fold non-empty, or
 * NULL for fold i mod k.  For each fold the model is trained on the other
 * rows (their dual restricted to those rows: the held-out variables stay
 * at 0) and predicts the held-out rows: decision (host, n x n_outputs,
 * nullable) receives every row's decision value from the model that did
 * not see it; stats the metrics over all rows.  With params->scale the
 * data are standardised once over all rows.  y, labels and fold in host
 * memory (X may be on the device).  Returns SVM_W_MAX_ITER when some
 * training stopped at max_iter (results still written). */
svm_status svm_cross_validate(const svm_matrix *X, const float *y,
                              const int32_t *labels, int32_t n_classes,
                              const svm_params *params, int32_t k,
                              const int32_t *fold, double *decision,
                              svm_cv_stats *stats);

/* Grid tuning by cross-validation (Section 3: "tuning parameters ... (C,
 * eps)", e1071's tune): for grid point g the parameters are params with C
 * = C[g], gamma = gamma[g] and epsilon = epsilon[g] (each array nullable:
 * then params' value), and cv_error[g] the k-fold error (1 - accuracy, or
 * the MSE for eps-SVR) on the given folds; *best = the first g of least
 * error.  Same inputs as svm_cross_validate. */
svm_status svm_tune(const svm_matrix *X, const float *y,
                    const int32_t *labels, int32_t n_classes,
                    const svm_params *params, int32_t k, const int32_t *fold,
                    int32_t n_grid, const double *C, const double *gamma,
                    const double *epsilon, double *cv_error, int32_t *best);

/* ------------------------------------------------------------------------
 * Feature maps: the layers whose outputs a model is trained on (random
 * cosine features for a linear SVM, or a residual network trained under the
 * SVM's squared hinge loss), with their gradients.
 *
 * Conventions of these calls, where they differ from the ones above:
 *   - Every array is device memory of `device` (on_device = 1; else
 *     SVM_E_UNSUPPORTED) and is borrowed for the work that the call queues.
 *   - The work is queued on `stream` (hipStream_t; NULL: the null stream)
 *     and NOT waited for.  Nothing is allocated or freed and nothing is
 *     copied to the host, so the calls can be captured into a HIP graph.
 *     The thread's current device is left as it was.
 *   - All arrays of a call have one type (svm_dtype), except where stated.
 *     Products, sums, statistics and states are held in 32 bits and rounded
 *     to that type once, when they are written; the one value rounded in
 *     between is dZ of svm_linear_backward (SVM_F32 products are made
 *     of three 8-bit parts of each factor: as exact as 32-bit products for
 *     factors from 2^-109 (1.5e-33) up to the largest; a smaller one is
 *     held to within 2^-134).
 *   - Outputs must not overlap inputs or each other, except where stated.
 *   - work: device memory of the caller, 16-byte aligned, of at least the
 *     bytes that the call's _workspace function writes to *bytes for the
 *     same arrays; its contents matter only during the call's work.
 *   - Results do not depend on earlier calls, and repeat bit for bit. */
typedef enum { SVM_F32 = 0, SVM_BF16 = 1, SVM_F16 = 2 } svm_dtype;

/* rows x cols values of one type, row i at data + i*ld values, ld >= cols.
 * Vectors (bias, weight) have rows = 1. */
typedef struct {
    void *data;
    int64_t rows, cols, ld;
    int32_t dtype;      /* svm_dtype */
    int32_t on_device;  /* 1 */
} svm_array;

typedef enum {
    SVM_ACT_NONE = 0,
    SVM_ACT_RELU = 1,   /* max(z, 0), NaN for NaN; its slope is 1 where
                           z > 0, else 0 (at 0 and for NaN too) */
    SVM_ACT_GELU = 2,   /* z (1 + erf(z / sqrt 2)) / 2 */
    SVM_ACT_SILU = 3,   /* z / (1 + exp(-z)) */
    SVM_ACT_TANH = 4,
    SVM_ACT_COS = 5     /* random Fourier features: with rows of W from
                           N(0, 2 gamma I), bias from U[0, 2 pi) and n
                           features, (2/n) phi(u).phi(v) tends to the RBF
                           kernel (train with SVM_KERNEL_POLY, degree 1,
                           gamma = 2/n).  Angles up to 1e8 in magnitude */
} svm_act;

/* One layer: Z = X W^T + bias, Y = act(Z) + residual.
 * X m x k (m >= 0), W n x k, bias 1 x n, residual, Y and Z m x n; bias,
 * residual and Z are nullable.  Z receives what the gradient needs (for
 * every act but SVM_ACT_NONE).  residual may be Y itself (same data and
 * ld).  m < 2^31, n and k in [1, 2^21]. */
svm_status svm_linear(const svm_array *X, const svm_array *W,
                      const svm_array *bias, const svm_array *residual,
                      int32_t act, const svm_array *Y, const svm_array *Z,
                      void *work, int64_t work_bytes, int32_t device,
                      void *stream);
svm_status svm_linear_workspace(const svm_array *X, const svm_array *W,
                                int64_t *bytes);

/* Its gradients for dY = dL/dY (m x n): with dZ = dY act'(Z),
 *   dX = dZ W,  dW = dZ^T X,  dbias = sum of the rows of dZ.
 * The residual's gradient is dY itself.  Z is what svm_linear wrote (may be
 * NULL for SVM_ACT_NONE).  dX, dW and dbias are nullable: those not asked
 * for cost nothing.  X may be NULL when dW is, W when dX is.  With m = 0,
 * dW and dbias are set to 0.
 * With 16-bit types and an activation, dX and dW are made from dZ rounded to
 * that type, as the matrix instructions need their factors (dbias from the
 * unrounded one): each term is off by up to 2^-8 (SVM_BF16) or 2^-11
 * (SVM_F16) of itself.  In SVM_F16 a dZ past 65504 is infinite and one below
 * 6e-5 is held in steps of 6e-8: scale the loss so that dZ lies between. */
svm_status svm_linear_backward(const svm_array *dY, const svm_array *X,
                               const svm_array *W, const svm_array *Z,
                               int32_t act, const svm_array *dX,
                               const svm_array *dW, const svm_array *dbias,
                               void *work, int64_t work_bytes,
                               int32_t device, void *stream);
svm_status svm_linear_backward_workspace(const svm_array *dY,
                                         const svm_array *X,
                                         const svm_array *W, int32_t act,
                                         const svm_array *dX,
                                         const svm_array *dW,
                                         const svm_array *dbias,
                                         int64_t *bytes);

/* Layer norm of each row: y = (x - mean) rstd weight + bias with the row's
 * mean and rstd = 1 / sqrt(mean of (x - mean)^2 + eps).  weight and bias
 * (1 x cols) are nullable (1 and 0).  mean and rstd (rows floats each,
 * nullable) receive the statistics that the gradient needs.  Y may be X
 * itself (same data and ld).  cols in [1, 2^21]. */
svm_status svm_layer_norm(const svm_array *X, const svm_array *weight,
                          const svm_array *bias, double eps,
                          const svm_array *Y, float *mean, float *rstd,
                          int32_t device, void *stream);

/* Its gradients: with xh = (x - mean) rstd and a = dY weight,
 *   dX = rstd (a - mean(a) - xh mean(a xh)) + residual,
 *   dweight = sum over rows of dY xh,  dbias = sum over rows of dY.
 * residual (rows x cols, nullable): the gradient that reaches X past the
 * norm, as in a residual network.  dX, dweight and dbias are nullable; dX
 * may be dY or the residual itself.  With no rows dweight and dbias are set
 * to 0. */
svm_status svm_layer_norm_backward(const svm_array *dY, const svm_array *X,
                                   const float *mean, const float *rstd,
                                   const svm_array *weight,
                                   const svm_array *residual,
                                   const svm_array *dX,
                                   const svm_array *dweight,
                                   const svm_array *dbias, void *work,
                                   int64_t work_bytes, int32_t device,
                                   void *stream);
svm_status svm_layer_norm_backward_workspace(int64_t rows, int64_t cols,
                                             int64_t *bytes);

/* Squared hinge loss, one class against the rest, and its gradient:
 *   *loss = scale * sum_ic max(0, 1 - y_ic S_ic)^2,
 *   dS_ic = -2 scale y_ic max(0, 1 - y_ic S_ic),
 * y_ic = +1 where c is labels[i], else -1; with one column, label 1 is +1
 * and label 0 is -1.  A label outside [0, C) (outside {0, 1} with one
 * column) leaves its row out: it adds nothing and its gradient is 0.  2 scale
 * has to be finite in 32 bits.  S and dS rows x C, C in [1, 2^21]; dS is
 * nullable and may be S itself.  labels: int32, rows of them; loss: one
 * float; both on the device. */
svm_status svm_hinge_loss(const svm_array *S, const int32_t *labels,
                          double scale, const svm_array *dS, float *loss,
                          void *work, int64_t work_bytes, int32_t device,
                          void *stream);
svm_status svm_hinge_loss_workspace(int64_t rows, int64_t cols,
                                    int64_t *bytes);

/* One tensor of svm_adamw_step: n contiguous values and their states.  The
 * states come in whole blocks of 256 values, B = ceil(n / 256) of them; what
 * lies past n in the last is updated as with a gradient of 0 (zeros stay
 * zeros).  In 32 bits m and v are 256 B floats each and the scales NULL.  In
 * 8 bits m is 256 B int8, v 256 B uint8, each block has a scale in m_scale
 * and v_scale (B floats each), and they stand for
 *   m = m_scale (c/127)^2 sign(c),  sqrt(v) = v_scale (c/254)^2,
 * the square roots giving small values more of the codes; -128 and 255
 * stand for NaN (a value that is not finite leaves its block's others
 * alone), a block whose largest magnitude is at most 1e-30 is held as
 * zeros, and a positive sqrt(v) in any other takes code 1 at least, so that
 * no value that moves is divided by eps alone.  All zeros are the states to
 * start from, in either form.  m, v and master are aligned to 16 bytes.
 * n = 0 is allowed. */
typedef struct {
    void *param;         /* dtype; updated in place */
    const void *grad;    /* grad_dtype */
    float *master;       /* nullable: the weights in 32 bits (256 B floats),
                            which the step works on; param receives them
                            rounded.  Not with SVM_F32 parameters */
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    int32_t dtype;       /* svm_dtype of param */
    int32_t grad_dtype;  /* dtype or SVM_F32 */
} svm_adamw_tensor;

typedef struct {
    double lr;            /* finite */
    double beta1, beta2;  /* in [0, 1) */
    double eps;           /* >= 0 */
    double weight_decay;  /* finite */
    double grad_scale;    /* factor of the gradients (1) */
    int64_t step;         /* t >= 1, the number of this step */
    int32_t bits;         /* states: 32 or 8 */
} svm_adamw_params;

/* One AdamW step (weight decay apart from the gradient) over all tensors of
 * a host array, read during the call, in as few launches as they fit:
 *   g = grad_scale grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;
 *   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
 * in 32 bits.  No two tensors may overlap. */
svm_status svm_adamw_step(const svm_adamw_tensor *tensors, int32_t n_tensors,
                          const svm_adamw_params *params, int32_t device,
                          void *stream);

/* The values that n 8-bit states stand for, their scales one to 256 (m_out,
 * v_out: n floats each, nullable), as a checkpoint wants them. */
svm_status svm_adamw_state(const int8_t *m, const uint8_t *v,
                           const float *m_scale, const float *v_scale,
                           int64_t n, float *m_out, float *v_out,
                           int32_t device, void *stream);

/* Group norm with an activation, channels last.  X has `positions` rows to a
 * sample and cols channels in `groups` groups of consecutive ones; for each
 * sample and group, over its positions and channels,
 *   y = act((x - mean) rstd weight + bias),
 *   rstd = 1 / sqrt(mean of (x - mean)^2 + eps).
 * rows a multiple of positions (>= 1), cols of groups.  weight and bias
 * (1 x cols) are nullable (1 and 0).  mean and rstd (samples x groups floats
 * each, nullable) receive the statistics that the gradient needs, and overlap
 * nothing.  Y may be X itself (same data and ld).  The sum of a group's values
 * and that of their squared deviations have to stay in 32 bits' range (an
 * infinite mean makes Y NaN, an infinite sum of squares rstd 0). */
svm_status svm_group_norm(const svm_array *X, int64_t positions,
                          int64_t groups, const svm_array *weight,
                          const svm_array *bias, double eps, int32_t act,
                          const svm_array *Y, float *mean, float *rstd,
                          void *work, int64_t work_bytes, int32_t device,
                          void *stream);
svm_status svm_group_norm_workspace(int64_t rows, int64_t positions,
                                    int64_t cols, int64_t groups,
                                    int32_t dtype, int64_t *bytes);

/* Its gradients: with xh = (x - mean) rstd, dZ = dY act'(xh weight + bias)
 * and a = dZ weight, means over a sample's group,
 *   dX = rstd (a - mean(a) - xh mean(a xh)) + residual,
 *   dweight = sum over rows of dZ xh,  dbias = sum over rows of dZ.
 * residual (rows x cols, nullable): the gradient that reaches X past the
 * norm.  dX, dweight and dbias are nullable and overlap neither each other
 * nor any input, mean and rstd among them, but dX may be dY or the residual
 * itself.  With no rows dweight and dbias are set to 0. */
svm_status svm_group_norm_backward(
    const svm_array *dY, const svm_array *X, int64_t positions,
    int64_t groups, const float *mean, const float *rstd,
    const svm_array *weight, const svm_array *bias, int32_t act,
    const svm_array *residual, const svm_array *dX, const svm_array *dweight,
    const svm_array *dbias, void *work, int64_t work_bytes, int32_t device,
    void *stream);
svm_status svm_group_norm_backward_workspace(int64_t rows, int64_t positions,
                                             int64_t cols, int64_t groups,
                                             int32_t dtype, int64_t *bytes);

/* One tensor of svm_grad_norm: n contiguous values.  n = 0 is allowed. */
typedef struct {
    const void *data;
    int64_t n;
    int32_t dtype;  /* svm_dtype, each tensor its own */
} svm_grad;

/* The norm of the gradients of a host array (read during the call), taken as
 * one vector, and the factor that brings it down to max_norm:
 *   *norm = |grad_scale| sqrt(sum of all g^2),
 *   *factor = max_norm / *norm where that is above max_norm, else 1,
 * one float each on the device; factor is nullable.  Squares and sums are
 * held in 64 bits.  Where a gradient is NaN or infinite, *norm is not finite
 * and *factor NaN.  max_norm >= 0, or infinite (a factor of 1 or NaN).  Both
 * are written after all gradients have been read. */
svm_status svm_grad_norm(const svm_grad *grads, int32_t n_grads,
                         double grad_scale, double max_norm, float *norm,
                         float *factor, void *work, int64_t work_bytes,
                         int32_t device, void *stream);
svm_status svm_grad_norm_workspace(const svm_grad *grads, int32_t n_grads,
                                   int64_t *bytes);

/* svm_adamw_step on clipped gradients: g = (grad_scale *factor) grad, with
 * the factor (one float, from svm_grad_norm) read on the device as the step
 * runs.  Where it is not finite nothing is written: the step is left out.
 * params->step counts it all the same (svm_adamw_step_counted does not).
 * factor NULL: svm_adamw_step.  It lies in nothing that the step writes. */
svm_status svm_adamw_step_clipped(const svm_adamw_tensor *tensors,
                                  int32_t n_tensors,
                                  const svm_adamw_params *params,
                                  const float *factor, int32_t device,
                                  void *stream);

/* svm_adamw_step_clipped that counts the steps left out, in *left_out on the
 * device (0 to begin with): the bias corrections are those of step
 * params->step - *left_out, so that the steps after one that was left out are
 * as if it had never been asked for.  Where this step is left out, *left_out
 * goes up by one (given a value to step).  factor and left_out overlap neither
 * each other nor what the step writes; left_out NULL: svm_adamw_step_clipped. */
svm_status svm_adamw_step_counted(const svm_adamw_tensor *tensors,
                                  int32_t n_tensors,
                                  const svm_adamw_params *params,
                                  const float *factor, int64_t *left_out,
                                  int32_t device, void *stream);

/* The weights of a linear layer in 4 bits, rows x cols, with a scale to each
 * `group` (32, 64 or 128) consecutive inputs of an output.  A weight stands
 * for scale times 0, 0.5, 1, 1.5, 2, 3, 4 or 6 with a sign.  data: device
 * memory, 16-byte aligned, of the bytes that svm_pack_weights_bytes states, in
 * an order of the library's own; it may be copied and kept, and read by any
 * call with the same rows, cols, group and dtype. */
typedef struct {
    void *data;
    int64_t bytes;       /* of data */
    int64_t rows, cols;  /* outputs, inputs: each in [1, 2^21] */
    int32_t group;       /* 32, 64 or 128 */
    int32_t dtype;       /* svm_dtype of the weights and of the scales */
} svm_packed;

/* Rounds the weights W to 4 bits.  A group's scale is a sixth of its largest
 * magnitude (times 1/6 in 32 bits), cut to six significant bits (SVM_F16: and
 * to whole steps of 2^-23), so that what a weight stands for is a value of its type; each weight
 * takes the nearest of the magnitudes, in the middle between two the one with
 * the even place (0, 1, 2, 4).  A weight that is not finite makes all of its
 * group NaN.  to: rows, cols and dtype of W. */
svm_status svm_pack_weights(const svm_array *W, const svm_packed *to,
                            int32_t device, void *stream);
svm_status svm_pack_weights_bytes(int64_t rows, int64_t cols, int32_t group,
                                  int32_t dtype, int64_t *bytes);

/* What packed weights stand for, exactly: W rows x cols, of their type. */
svm_status svm_unpack_weights(const svm_packed *packed, const svm_array *W,
                              int32_t device, void *stream);

/* One layer on packed weights: Y = act(X W^T + bias) + residual, arrays as in
 * svm_linear.  No weight is rounded further: sums of X times codes over a
 * group's inputs are held in 32 bits and multiplied by the group's scale there
 * (and formed again, smaller by a power of two, where they would leave 32 bits
 * before the scale).  Made for few rows, whose time is
 * that of reading the weights; many go through svm_linear's products on the
 * unpacked weights, in the workspace.  residual may be Y itself. */
svm_status svm_linear_packed(const svm_array *X, const svm_packed *W,
                             const svm_array *bias, const svm_array *residual,
                             int32_t act, const svm_array *Y, void *work,
                             int64_t work_bytes, int32_t device,
                             void *stream);
svm_status svm_linear_packed_workspace(const svm_array *X,
                                       const svm_packed *W, int64_t *bytes);

const char *svm_last_error(void);

/* ------------------------------------------------------------------------
 * Test hooks: a solver whose state can be set and stepped one phase at a
 * time, so the tests can compare single steps with the CPU oracle from an
 * identical state.  Not needed for training.  Host pointers only.
 * ---------------------------------------------------------------------- */
typedef struct svm_solver svm_solver;

svm_status svm_test_solver_create(const svm_matrix *X, const float *y,
                                  const svm_params *p, svm_solver **out);
void svm_test_solver_free(svm_solver *s);

/* Replace the state: alpha[N] and responses F[n] (fp64). */
svm_status svm_test_set_state(svm_solver *s, const double *alpha,
                              const double *F);
svm_status svm_test_get_state(svm_solver *s, double *alpha, double *F);

/* Working-set selection on the current state: the q/2 largest keys of I_up
 * interleaved with the q/2 smallest of I_low, ties to the lowest index:
 * B[<= q] variable indices, *nB, and m = max_{I_up} v, M = min_{I_low} v. */
svm_status svm_test_select(svm_solver *s, int32_t *B, int32_t *nB, double *m,
                           double *M);

/* Kernel rows K(x_samples[j], X) for k <= 64 samples: out[j*n + i], fp32. */
svm_status svm_test_rows(svm_solver *s, const int32_t *samples, int32_t k,
                         float *out);

/* Solve the subproblem on B from the current state; returns the new
 * alpha_B and the number of inner steps (state unchanged). */
svm_status svm_test_subproblem(svm_solver *s, const int32_t *B, int32_t nB,
                               double inner_tol, int32_t max_inner,
                               double *alpha_B_new, int32_t *steps);

/* Set alpha_B to the given values and update F with the row/update kernel. */
svm_status svm_test_apply(svm_solver *s, const int32_t *B, int32_t nB,
                          const double *alpha_B_new);

/* Run up to k full outer iterations; *iters gets the count, *gap the gap. */
svm_status svm_test_iterate(svm_solver *s, int64_t k, int64_t *iters,
                            double *gap);

/* End a training on the current state as svm_train ends it: recompute F
 * from alpha, re-test the gap and, while it exceeds tol, run the loop again
 * and re-test, at most max_passes (>= 0) times (svm_train uses 3).  *gap,
 * *b (bias: the mean key over free variables, else (m + M) / 2) and
 * *obj (f(a)) come from the recomputed responses; *status is SVM_OK,
 * SVM_W_MAX_ITER or SVM_W_NOT_CONVERGED (the gap still above tol). */
svm_status svm_test_finish(svm_solver *s, int32_t max_passes, double *gap,
                           double *b, double *obj, int32_t *status);

#ifdef __cplusplus
}
#endif
#endif /* MI355SVM_H */
