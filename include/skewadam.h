/*
 * libskewadam -- the SkewAdam optimizer step (tiered optimizer state for MoE
 * training) on one NVIDIA GB300 (sm_103a).
 *
 * The step follows "Where Should Optimizer State Live? Tiered State Allocation
 * for Memory-Efficient MoE Training":
 *   - tiers (Sec. 3 "The tiers", Fig. 1): backbone tensors keep fp32 momentum
 *     and a factored second moment; expert tensors keep only the factored
 *     second moment; the router keeps the exact (unfactored) second moment and
 *     no weight decay; any vector (1-D tensor) keeps the exact second moment
 *     (Algorithm 1);
 *   - factored second moment (Eq. 1): per matrix W (n x m) an fp32 row vector
 *     R (n) and column vector C (m) of exponential moving averages of the row
 *     and column means of G*G; Vhat = R C^T / mean(R);
 *   - update (Algorithm 1): D = sqrt(max(Vhat, eps)); backbone
 *     U = sqrt(1-beta2^t)/(1-beta1^t) * M / D with M = beta1 M + (1-beta1) G;
 *     other tiers U = sqrt(1-beta2^t) * G / D;
 *   - update clipping (Sec. 3 "Update clipping and low-precision updates"):
 *     U <- U / max(1, RMS(U)/d), RMS over the whole tensor;
 *   - decoupled weight decay fused into the fp32 update ahead of the cast
 *     (Sec. 3 footnote, Sec. 5): x = w (1 - lr*lambda) - lr * U;
 *   - dithered bf16 write-back (Sec. 3, Algorithm 1 last line): the fp32 value
 *     x is rounded to bf16 by adding a uniform 16-bit integer r to its bit
 *     pattern and truncating (unbiased stochastic rounding with the exact bf16
 *     ulp of x); r is a Philox-4x32-10 draw keyed by (seed) and counted by
 *     (element index / 8, tensor id, step), so a step is bit-reproducible;
 *   - state size (Sec. 3 "Memory model", Eq. 2, App. B Table 5): 4 bytes per
 *     momentum element, per exact-second-moment element and per R / C entry.
 *
 * Conventions for every entry point:
 *   - Return SKEW_OK (0) or a negative SKEW_E* code; nothing aborts or throws.
 *     skew_last_error() gives a one-line reason for the last failure on a
 *     handle (skew_create failures: pass NULL).
 *   - Device memory (weights, gradients, state, workspace) is owned by the
 *     caller; the library owns only host-side metadata in the handle.
 *   - Pointers passed as `void *stream` are cudaStream_t values (0 = legacy
 *     default stream). Work is enqueued asynchronously on that stream; one
 *     stream per handle at a time.
 *   - Element counts are 64-bit; a tensor may exceed 2^31 elements.
 */
#ifndef SKEWADAM_H_
#define SKEWADAM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes -------------------------------------------------------- */
#define SKEW_OK 0
#define SKEW_EINVAL (-1)   /* invalid argument (null, shape, tier, hyper-parameter, step, size) */
#define SKEW_ENOMEM (-2)   /* host allocation failed                                        */
#define SKEW_ECUDA (-3)    /* a CUDA runtime call failed                                   */
#define SKEW_ETIMEOUT (-4) /* a bounded device-side wait gave up (see skew_sync_status)    */
#define SKEW_ESTATE (-5)   /* call out of order (e.g. skew_step before skew_bind)          */
#define SKEW_ETOOBIG (-6)  /* tensor needs more scratch than skew_step_tensor_noalloc has */

/* ---- tiers (Sec. 3 "The tiers") -------------------------------------------- */
#define SKEW_TIER_BACKBONE 0 /* embeddings, positions, attention, dense FFN, norms */
#define SKEW_TIER_EXPERT 1   /* expert matrices                                     */
#define SKEW_TIER_ROUTER 2   /* the gate                                            */

/* ---- allocation policies: the paper's policy and the Table 3 variants ------ */
#define SKEW_POLICY_TIERED 0          /* SkewAdam as published                         */
#define SKEW_POLICY_EXPERT_MOMENTUM 1 /* "+ momentum on experts"                        */
#define SKEW_POLICY_FACTORED_ROUTER 2 /* "factored router"                              */
#define SKEW_POLICY_UNIFORM 3         /* "uniform (momentum + factored)" on every tier  */
/* The Adafactor comparator (Sec. 5, Table 4 and its footnote, App. A; Shazeer &
 * Stern 2018): every matrix factored (the router too), vectors exact, no momentum, the
 * second-moment decay annealed as beta2_t = 1 - t^-0.8 (beta1 and beta2 are then
 * unused) and no bias correction; the same clipping, decay and write-back. */
#define SKEW_POLICY_ADAFACTOR 4

/* ---- per-tensor flags ------------------------------------------------------ */
#define SKEW_F_NO_DECAY 1u /* exempt this tensor from weight decay (the router always is) */
/* Weights and gradient are fp32 (4-byte aligned), as the paper keeps the norms and
 * the router (App. A): the new weight is the fp32 update itself, with no dithered
 * cast. Such a tensor takes the scalar tile path (it is small). */
#define SKEW_F_FP32 2u

/* ---- second-moment kinds reported by skew_tensor_info ----------------------- */
#define SKEW_KIND_FULL 0     /* exact second moment v (router, vectors)  */
#define SKEW_KIND_FACTORED 1 /* row / column factors R, C (Eq. 1)        */

typedef struct skew_handle skew_handle_t; /* opaque */

/*
 * One parameter tensor. The tensor id used by the dither is its index in the
 * array passed to skew_create.
 *   weight : device pointer to the bf16 weights (fp32 with SKEW_F_FP32),
 *            contiguous row-major, updated in place by skew_step; 2-byte
 *            aligned, 4-byte for fp32 (16-byte alignment enables the
 *            vectorised bf16 path). Borrowed: must stay valid while the handle
 *            is bound.
 *   grad   : device pointer to the gradient, the weights' type, shape and
 *            layout; read only. Borrowed like `weight`.
 *   shape  : shape[0] = rows n (>= 1); shape[1] = columns m (>= 1) when
 *            ndim >= 2, ignored when ndim == 1.
 *   ndim   : 1 (vector), 2 (matrix) or 3 (a stack of `stack` matrices of
 *            n x m, contiguous: matrix e starts at element e*n*m).
 *   tier   : SKEW_TIER_*.
 *   flags  : SKEW_F_* bits.
 *   stack  : the number of matrices when ndim == 3 (>= 1); 0 otherwise.
 *
 * A stacked tensor (experts kept as one (E, n, m) array) is stepped as E
 * matrices, each with its own second-moment factors, RMS and clip factor
 * (Algorithm 1 is stated per matrix; the paper counts 128 x 3 expert
 * matrices); its dither uses the descriptor's index as tensor id and the flat
 * index e*n*m + i*m + j over the whole stack.
 */
typedef struct {
    void *weight;
    const void *grad;
    int64_t shape[2];
    int32_t ndim;
    int32_t tier;
    uint32_t flags;
    uint32_t stack;
} skew_param_desc_t;

/*
 * Hyper-parameters (Algorithm 1, App. A Table 9). The paper's defaults are
 * beta1 = 0.9, beta2 = 0.999, eps = 1e-8, clip_d = 1, weight_decay = 0.05.
 *   0 <= beta1 < 1, 0 <= beta2 < 1, eps > 0 (finite), clip_d > 0 (finite),
 *   weight_decay >= 0 (finite), policy = SKEW_POLICY_*.
 */
typedef struct {
    float beta1;
    float beta2;
    float eps;
    float clip_d;
    float weight_decay;
    int32_t policy;
} skew_hparams_t;

/*
 * Where one tensor's state lives inside the caller's state buffer (offsets in
 * fp32 elements from its start; -1 when the tensor has no such array).
 *   m_offset: momentum M (numel floats, row-major)
 *   v_offset: exact second moment v (numel floats)
 *   r_offset: R (rows floats), c_offset: C (cols floats)
 */
typedef struct {
    int32_t kind;       /* SKEW_KIND_*                                         */
    int32_t momentum;   /* 1 if the tensor keeps fp32 momentum                 */
    int32_t decay;      /* 1 if weight decay applies                           */
    int32_t vectorized; /* 1 if the 16-byte vector path serves it (after bind) */
    int64_t rows, cols, numel;
    int64_t m_offset, v_offset, r_offset, c_offset;
    int32_t rowpath;    /* 1 at the widths 512, 1024, 2048 and 4096 (bf16, 16-byte */
                        /* aligned); what a step runs on: skew_tensor_route        */
    int32_t stack;      /* matrices of a stacked tensor (ndim 3), else 0; then   */
                        /* rows / cols are one matrix's, numel the whole stack's, */
                        /* and each state array holds the E matrices' in order   */
} skew_tensor_info_t;

/*
 * Plans the step for `n_params` tensors (n_params >= 0; 0 gives a handle whose
 * step does nothing). Validates every descriptor and the hyper-parameters,
 * resolves each tensor's tier policy (kind / momentum / decay), lays out the
 * optimizer state and the workspace. Host only: no CUDA call, no device
 * memory touched. On success *out receives a new handle (free with
 * skew_destroy). Errors: SKEW_EINVAL (reason in skew_last_error(NULL)),
 * SKEW_ENOMEM.
 */
int skew_create(const skew_param_desc_t *params, int32_t n_params, const skew_hparams_t *hp,
                skew_handle_t **out);

/* Frees the handle's host metadata (not the caller's device memory). NULL is a no-op. */
int skew_destroy(skew_handle_t *h);

/*
 * Exact optimizer-state size in bytes: 4 * (sum over momentum tensors of numel
 * + sum over factored tensors of (rows + cols) + sum over exact-second-moment
 * tensors of numel) -- Eq. 2 with the vectors' full v of Table 5. The caller
 * allocates exactly this many bytes of device memory for the state. 0 for NULL.
 */
size_t skew_state_bytes(const skew_handle_t *h);

/*
 * Scratch the step needs besides the state (per-tensor partial sums, scalars,
 * descriptor and tile tables). Not optimizer state. 0 for NULL.
 */
size_t skew_workspace_bytes(const skew_handle_t *h);

/*
 * Binds caller-owned device buffers to the handle: `state` (exactly
 * skew_state_bytes bytes) and `workspace` (exactly skew_workspace_bytes bytes),
 * both 256-byte aligned device pointers (NULL allowed when the size is 0).
 * Uploads the descriptor and tile tables into the workspace and zero-fills the
 * state (the paper's initial M = v = R = C = 0), enqueued on `stream`.
 * May be called again to re-bind (the state is zeroed again).
 * Errors: SKEW_EINVAL (size / alignment), SKEW_ECUDA.
 */
int skew_bind(skew_handle_t *h, void *state, size_t state_bytes, void *workspace, size_t workspace_bytes,
              void *stream);

/*
 * Enqueues one SkewAdam step over every tensor on `stream`: reads each
 * gradient, updates the state and writes the bf16 weights in place.
 *   step : global 1-based step t (bias corrections beta^t; the dither counter
 *          uses its low 32 bits). All tensors advance together.
 *   lr   : the scheduled learning rate eta_t (finite, >= 0); the caller owns
 *          the schedule.
 *   seed : 64-bit dither seed.
 * Asynchronous: device-side problems are reported by skew_sync_status.
 * Errors: SKEW_ESTATE (not bound), SKEW_EINVAL (step < 1, lr not finite or
 * negative), SKEW_ECUDA (launch failure).
 */
int skew_step(skew_handle_t *h, int64_t step, float lr, uint64_t seed, void *stream);

/*
 * skew_step with the trainer's global gradient-norm clip applied inside the step.
 * The paper's training setup (Sec. 4) and App. A Table 9 clip the global gradient
 * norm at 1.0 before the optimizer step: G <- gamma * G with gamma = min(1, c /
 * ||G||). Here the step sees gamma * G without a separate pass over the gradients:
 * gamma enters only the moving-average increments ((1 - beta1) gamma on g,
 * (1 - beta2) gamma^2 on g^2) and the update coefficient of momentum-free tensors,
 * so the step reads and writes exactly the bytes of skew_step. (Scaling the learning
 * rate instead is not the same step: the second moments are moving averages of the
 * scaled gradient.)
 *   grad_scale : device pointer to one fp32 gamma (finite), computed by the caller
 *                on `stream` before this call (e.g. from its norm reduction); read
 *                by the kernels, never by the host; 4-byte aligned. NULL means
 *                gamma = 1, and then the call is skew_step, bit for bit; so is a
 *                pointer to 1.0f.
 * Other arguments, asynchrony and errors as skew_step (SKEW_EINVAL also for a
 * misaligned grad_scale).
 */
int skew_step_scaled(skew_handle_t *h, int64_t step, float lr, uint64_t seed, const float *grad_scale, void *stream);

/*
 * Synchronises `stream` and reports the device-side status word of the last
 * steps: SKEW_OK, or SKEW_ETIMEOUT if a bounded device wait gave up (the word
 * is cleared by this call). Errors: SKEW_ESTATE, SKEW_ECUDA.
 */
int skew_sync_status(skew_handle_t *h, void *stream);

/*
 * Self-test of the failure path of the bounded device waits: enqueues on
 * `stream` one thread that waits, exactly as the whole-row kernels wait for a
 * copied chunk, on an mbarrier phase that nothing completes. The wait gives up
 * after its poll limit (about two seconds at most) and records the timeout in
 * the handle's status word, so the next skew_sync_status returns SKEW_ETIMEOUT
 * and clears it; the context stays usable and later steps are unaffected.
 * Asynchronous. Errors: SKEW_EINVAL (null), SKEW_ESTATE (not bound),
 * SKEW_ECUDA (launch failure).
 */
int skew_selftest_wait_timeout(skew_handle_t *h, void *stream);

/*
 * Per-tensor scalars of the last completed step, for inspection and tests:
 * out[0] = mean(R) (factored tensors, else 0), out[1] = sum of U^2 over the
 * tensor, out[2] = RMS(U), out[3] = clip factor 1/max(1, RMS/d). Synchronises
 * `stream`. Errors: SKEW_EINVAL (tid), SKEW_ESTATE, SKEW_ECUDA.
 */
int skew_tensor_scalars(skew_handle_t *h, int32_t tid, double out[4], void *stream);

/* As skew_tensor_scalars, for matrix `e` of stacked tensor `tid` (e = 0 for any
 * other tensor). Errors: SKEW_EINVAL (tid, e), SKEW_ESTATE, SKEW_ECUDA. */
int skew_matrix_scalars(skew_handle_t *h, int32_t tid, int32_t e, double out[4], void *stream);

/* Resolved policy and state offsets of tensor `tid`. Errors: SKEW_EINVAL. */
int skew_tensor_info(const skew_handle_t *h, int32_t tid, skew_tensor_info_t *out);

/*
 * Which launches step tensor `tid` (every matrix of a stack alike), as skew_create
 * planned them: a SKEW_ROUTE_* value, or SKEW_EINVAL. Inspection, tests and byte
 * accounting; results do not depend on it beyond the summation order.
 */
#define SKEW_ROUTE_OWN 0    /* strip or flat tiles: k_sumsq, k_finalize, k_rms, k_apply              */
#define SKEW_ROUTE_RIDING 1 /* the same tiles in the row tiles' launches                            */
#define SKEW_ROUTE_ROWS 2   /* whole-row tiles: k_rowsq, k_finalize, k_fallback, k_apply_rows        */
#define SKEW_ROUTE_SMALL 3  /* the whole step is one launch, k_small                                 */
int skew_tensor_route(const skew_handle_t *h, int32_t tid);

/*
 * Benchmark support: launch timing. After skew_profile_begin(h, n), each of the
 * next n calls of skew_step records a CUDA event before and after each timed
 * launch it makes on the step's stream (seven places, named by
 * skew_kernel_name; a phase with no work times ~0; no extra
 * synchronisation). skew_profile_end(h, ms, cap, &steps, &launches)
 * synchronises, writes the durations in milliseconds row-major into
 * ms[steps][launches] (up to cap values), releases the events and stops
 * recording. skew_kernel_name(k) names timed launch k of a step.
 * Errors: SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_profile_begin(skew_handle_t *h, int32_t max_steps);
int skew_profile_end(skew_handle_t *h, double *ms, int64_t cap, int32_t *n_steps, int32_t *n_kernels);
const char *skew_kernel_name(int32_t k);

/*
 * A step over ONE tensor that allocates nothing -- no cudaMalloc / cudaFree, no
 * allocating library routine, no host heap. The paper has no counterpart; this
 * is a deployment convenience.
 *
 * Who needs it: callers that cannot allocate device memory when they step the
 * optimizer, e.g. code running while a framework's caching allocator holds all
 * free memory, plugins that are only handed pre-sized buffers, or runtimes that
 * forbid allocation after start-up. skew_bind needs a caller-allocated
 * workspace; this entry point instead uses a fixed scratch array compiled into
 * the library: SKEW_NOALLOC_SCRATCH_BYTES of device memory on every GPU that
 * loads the library, held until the process exits. That is enough for one
 * 4,096-wide matrix of up to about 65,000 rows with momentum (the paper's
 * 50,304 x 4,096 embedding fits; the whole-row partials take 256 bytes per row)
 * and about twice that without (128 bytes per row on its 256-row tiles); larger
 * tensors are rejected with SKEW_ETOOBIG before any work is enqueued.
 *
 * Arguments: weight / grad as in skew_param_desc_t (device, bf16 or with
 * SKEW_F_FP32 fp32, row-major);
 * ndim, rows, cols, tier, flags as in skew_param_desc_t; hp as for
 * skew_create; state: this tensor's fp32 state, exactly state_bytes =
 * 4 * ((momentum ? numel : 0) + (full second moment ? numel : rows + cols))
 * bytes, laid out [M][v] or [M][R][C] (absent arrays take no room), 4-byte
 * aligned, zero-filled by the caller before the first step; tensor_id: the id
 * fed to the dither (use the tensor's index in a skew_create list to get the
 * same bits as skew_step); step, lr, seed as for skew_step; stream: a
 * cudaStream_t. Updates weight and state in place, asynchronously on stream,
 * with the same kernels and results as skew_step on a one-tensor handle (up to
 * summation order at the few sizes whose row tiles must be larger to fit the scratch).
 *
 * Every call looks up the array's device address on the current device with
 * cudaGetSymbolAddress. The first such lookup on a device may load the
 * library's device code there: make the first call on each device before any
 * stream capture. All calls on a device share the one array: calls whose
 * work overlaps on the GPU (different streams, or other host threads) race
 * and corrupt each other's results -- serialise them. The array keeps the
 * last call's contents; everything a step needs zeroed is cleared by the step.
 *
 * Device-side failures: the whole-row kernels' bounded waits (as for
 * skew_step) record a copy that did not land in a status word at the start of
 * the array. No call clears it; skew_noalloc_sync_status reads it. A step
 * whose wait gave up has left some tiles of that tensor unwritten.
 * Errors: SKEW_EINVAL (argument or state size), SKEW_ETOOBIG, SKEW_ECUDA.
 */
#define SKEW_NOALLOC_SCRATCH_BYTES (16u * 1024u * 1024u)
int skew_step_tensor_noalloc(void *weight, const void *grad, int32_t ndim, int64_t rows, int64_t cols, int32_t tier,
                             uint32_t flags, const skew_hparams_t *hp, void *state, size_t state_bytes,
                             uint32_t tensor_id, int64_t step, float lr, uint64_t seed, void *stream);

/*
 * Synchronises `stream` and reports the no-alloc status word of the current
 * device: SKEW_OK, or SKEW_ETIMEOUT if a bounded device wait of a
 * skew_step_tensor_noalloc call gave up since the word was last read (the word
 * is then cleared, with a memset enqueued on `stream` and waited for). Uses no
 * allocation (a 4-byte device-to-host copy). Errors: SKEW_ECUDA.
 */
int skew_noalloc_sync_status(void *stream);

/*
 * Self-test of that failure path: enqueues on `stream` one thread that waits,
 * exactly as the whole-row kernels wait for a copied chunk, on an mbarrier
 * phase that nothing completes; after its poll limit (about two seconds) the
 * wait gives up and sets the no-alloc status word, so the next
 * skew_noalloc_sync_status returns SKEW_ETIMEOUT. Nothing else is touched and
 * the context stays usable. Asynchronous. Errors: SKEW_ECUDA.
 */
int skew_noalloc_selftest_wait_timeout(void *stream);

/*
 * Kernel launches one skew_step performs: the one that clears the per-step
 * scalars and the grouped launches over item tables, or the single launch of a
 * step of small tensors; 0 for NULL or an empty handle.
 */
int64_t skew_launches_per_step(const skew_handle_t *h);

/* Number of tensors the handle plans for (0 for NULL). */
int32_t skew_num_tensors(const skew_handle_t *h);

/* One-line reason for the last failure on `h` (or of skew_create when h is NULL). */
const char *skew_last_error(const skew_handle_t *h);

/* ==========================================================================
 * Around the step: what a trainer computes with the tiers' tensors before it.
 *
 * Conventions as above; the tensors and the stream are the current device's. The
 * entry points below report the reason of a failed
 * call through skew_ops_last_error (per host thread). They neither synchronise
 * nor allocate device memory (skew_clip_bind and skew_ops_sync_status alone synchronise), and can be
 * captured into a CUDA graph after one call outside of it.
 * ======================================================================== */

/* One-line reason for the last failure of an entry point below on this host thread. */
const char *skew_ops_last_error(void);

/* ---- global gradient norm and clipping -------------------------------------
 *   norm  = sqrt(sum over all tensors and elements of g^2)
 *   gamma = min(1, max_norm / (norm + 1e-6))
 *   out   = gamma * g
 * gamma is what skew_step_scaled takes as grad_scale, so that a trainer whose
 * gradients go to the step only needs skew_clip_norm (one read of them). Squares
 * are summed in fp32 (two-term sums) and joined in fp64, in an order that depends on the
 * tensors' sizes, types and alignment alone; elements whose squares leave fp32's range are summed scaled,
 * so the norm is right for any finite gradient (and Inf only where it exceeds fp32
 * itself). A NaN in a gradient makes norm and gamma NaN; an Inf makes norm Inf and
 * gamma 0 (0 * Inf is then NaN in the clipped tensor).
 */
#define SKEW_CLIP_GRAD_FP32 1u /* g is fp32 (else bf16)                          */
#define SKEW_CLIP_OUT_FP32 2u  /* out is fp32 (else bf16); needs an fp32 g       */

typedef struct skew_clip skew_clip_t; /* opaque */

/*
 * One gradient tensor.
 *   grad  : device pointer to `numel` contiguous elements, aligned to their type
 *           (16-byte alignment enables vector accesses). Borrowed while bound.
 *   out   : where skew_clip_apply writes; `grad` itself to clip in place (same
 *           type), else memory that overlaps no gradient and no other `out`. NULL
 *           in every descriptor of a handle that only computes norms.
 *   numel : 0 to 2^40.
 */
typedef struct {
    const void *grad;
    void *out;
    int64_t numel;
    uint32_t flags; /* SKEW_CLIP_* */
    uint32_t zero;  /* 0 */
} skew_clip_desc_t;

/* Plans for `n` tensors (0 allowed: the norm is then 0). Host only. Errors: SKEW_EINVAL, SKEW_ENOMEM. */
int skew_clip_create(const skew_clip_desc_t *tensors, int32_t n, skew_clip_t **out);
int skew_clip_destroy(skew_clip_t *h); /* NULL is a no-op */
/* Bytes of device workspace (tile table and partial sums); 0 for NULL. */
size_t skew_clip_workspace_bytes(const skew_clip_t *h);
/* Binds a 256-byte aligned workspace and uploads the table on `stream` (synchronises it). */
int skew_clip_bind(skew_clip_t *h, void *workspace, size_t workspace_bytes, void *stream);
/*
 * result[0] = norm, result[1] = gamma (device, fp32, 4-byte aligned). max_norm: finite, >= 0.
 * Calls on one handle must not overlap on the GPU. Errors: SKEW_ESTATE, SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_clip_norm(skew_clip_t *h, float max_norm, float *result, void *stream);
/* skew_clip_norm, then out = gamma * g for every tensor (nothing is read or written for one that is clipped in
 * place by gamma = 1). Errors: also SKEW_ESTATE for a handle planned without `out`. */
int skew_clip_apply(skew_clip_t *h, float max_norm, float *result, void *stream);

/* ---- routing of tokens to experts --------------------------------------------
 * Per token, with logits x over the experts:
 *   score   s = softmax(x) or sigmoid(x)
 *   choice  c = s + bias (bias != NULL), else x, which orders as s does
 *   groups  (groups > 1) experts are `groups` consecutive runs; a run counts by its largest
 *           c (group_top 1) or the sum of its two largest s + bias (group_top 2); the
 *           top_groups best keep their experts
 *   chosen  the top_k largest c of what is left, largest first, the lowest index first among equals
 *   weight  w = scale * s, divided by the sum of the chosen s with SKEW_GATE_RENORM
 * A bias steers which experts are chosen and never enters a weight (it balances
 * loads without a loss term). Experts with a logit of -Inf or NaN, or a choice that is
 * -Inf or NaN, are never chosen: a slot that finds no expert is -1 with weight 0. A sum of
 * zero gives weights of zero. A NaN logit makes the weights of its token NaN (and, by a softmax, its
 * scores, so that nothing is chosen where a bias makes experts go by them). Scores are fp32.
 */
#define SKEW_GATE_SOFTMAX 0
#define SKEW_GATE_SIGMOID 1
#define SKEW_GATE_RENORM 1u /* weights divided by their sum                     */
#define SKEW_GATE_FP32 2u   /* logits and their gradient are fp32 (else bf16)   */

/*
 * experts 1 to 512; groups 1 to 32, a divisor of experts; top_groups 1 to groups; group_top
 * 1 or 2; top_k 1 to 32 and at most the experts of top_groups groups; score
 * SKEW_GATE_SOFTMAX or _SIGMOID; scale finite.
 */
typedef struct {
    int32_t experts, top_k, groups, top_groups, group_top, score;
    float scale;
    uint32_t flags; /* SKEW_GATE_* */
} skew_gate_config_t;

/* Bytes of device workspace that `counts` need (0 for an invalid config). */
size_t skew_gate_workspace_bytes(const skew_gate_config_t *c);
/*
 * logits: `tokens` rows of `experts` elements, `ld` >= experts elements apart, aligned to their type
 * (16-byte aligned rows enable vector loads). bias: fp32 per expert, or NULL. chosen, weights:
 * (tokens, top_k), contiguous. counts: how many tokens chose each expert (int32 per expert), or
 * NULL. workspace: zero-filled once by the caller; every call leaves it zeroed; calls that
 * share one must not overlap on the GPU. tokens: 0 to 2^31 - 1.
 * Errors: SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_gate_forward(const skew_gate_config_t *c, const void *logits, int64_t ld, const float *bias, int64_t tokens,
                      int32_t *chosen, float *weights, int32_t *counts, void *workspace, size_t workspace_bytes, void *stream);
/*
 * The logits' gradient from the weights' (tokens, top_k), for the experts in `chosen` (distinct within a
 * token; entries outside [0, experts) have none). Every element of the `tokens` rows of dlogits, `ld_out`
 * elements apart, is written (zeros included). dlogits has the logits' type and may not overlap any input.
 */
int skew_gate_grad(const skew_gate_config_t *c, const void *logits, int64_t ld, const int32_t *chosen, const float *dweights,
                   int64_t tokens, void *dlogits, int64_t ld_out, void *stream);

/* ---- embedding lookup and its gradient -----------------------------------------
 *   lookup    y[t] = scale * W[id_t]
 *   gradient  dW[v] = base[v] + scale * (sum over the t with id_t = v of dy[t])
 * W is (rows, width), contiguous. An id outside [0, rows) is padding: its y is zero and it has no
 * gradient. Terms are added in fp32 in the tokens' order (a row with many terms: in runs of at most
 * 32, then sixteen of those sums at a time, then the rest, each in order), so results do not depend on
 * timing; each element is rounded once.
 */
#define SKEW_EMBED_TABLE_FP32 1u /* W, base and dW are fp32 (else bf16) */
#define SKEW_EMBED_ACT_FP32 2u   /* y and dy are fp32 (else bf16)       */
#define SKEW_EMBED_IDS_64 4u     /* ids are int64 (else int32)          */

/* rows 1 to 2^31 - 1, width 1 to 2^20, scale finite. */
typedef struct {
    int64_t rows, width;
    float scale;
    uint32_t flags; /* SKEW_EMBED_* */
} skew_embed_config_t;

/*
 * tokens: 0 to 2^30 ids, contiguous. out: `tokens` rows of `width` elements, `ld_out` >= width
 * elements apart. Pointers aligned to their types (rows that start on 16-byte boundaries, of a
 * width that 8 divides, enable vector accesses). Errors: SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_embed_lookup(const skew_embed_config_t *c, const void *table, const void *ids, int64_t tokens, void *out,
                      int64_t ld_out, void *stream);
/* Bytes of device workspace that the gradient of `tokens` tokens needs (0 for an invalid config). */
size_t skew_embed_workspace_bytes(const skew_embed_config_t *c, int64_t tokens);
/*
 * dout: the gradient of `out`, rows `ld_dout` apart. Every element of dtable is written, rows without
 * tokens as base or zero. base: NULL, a tensor like dtable that overlaps nothing else, or dtable itself, to which the
 * gradient is then added; rows without tokens are not touched (the gradient of a table
 * that the output head shares). workspace: 256-byte aligned, of any content; calls that share one
 * must not overlap on the GPU.
 */
int skew_embed_grad(const skew_embed_config_t *c, const void *ids, int64_t tokens, const void *dout, int64_t ld_dout,
                    const void *base, void *dtable, void *workspace, size_t workspace_bytes, void *stream);

/* ---- rows by expert and back ---------------------------------------------------
 * What lies between the routing and the experts' products. Of the (tokens, top_k) experts that a router chose,
 *   order         place of (t, j): how many entries go before it, by (expert, t, j); -1 for an entry outside
 *                 [0, experts). offsets[e]: the first place of expert e; offsets[experts]: how many there are.
 *   spread        rows[place(t, j)] = x[t]
 *   combine       out[t] = sum over j of weights[t, j] * rows[place(t, j)]
 *   combine_grad  drows[place(t, j)] = weights[t, j] * dout[t], dweights[t, j] = <dout[t], rows[place(t, j)]>
 * The gradient of spread is combine without weights. A row that an entry without a place would read is zero (so is its
 * dweights); rows from offsets[experts] up to tokens * top_k are written as zeros by spread and combine_grad. Sums are fp32: combine's in the
 * order of j, so that results do not depend on timing; each element is rounded once.
 */
#define SKEW_DISPATCH_TOKENS_FP32 1u /* x, out and dout are fp32 (else bf16)  */
#define SKEW_DISPATCH_ROWS_FP32 2u   /* rows and drows are fp32 (else bf16)   */

/* experts 1 to 1024, top_k 1 to 64. */
typedef struct {
    int32_t experts, top_k;
    uint32_t flags; /* SKEW_DISPATCH_* */
    uint32_t zero;  /* 0 */
} skew_dispatch_config_t;

/* Bytes of device workspace that the order of `tokens` tokens needs (0 for an invalid config). tokens * top_k: at most 2^30. */
size_t skew_dispatch_workspace_bytes(const skew_dispatch_config_t *c, int64_t tokens);
/*
 * chosen, places: (tokens, top_k), contiguous; offsets: experts + 1. workspace: 256-byte aligned, of any content; calls that share one must
 * not overlap on the GPU. Errors, here and below: SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_dispatch_order(const skew_dispatch_config_t *c, const int32_t *chosen, int64_t tokens, int32_t *offsets, int32_t *places, void *workspace,
                        size_t workspace_bytes, void *stream);
/*
 * x: `tokens` rows of `width` elements (1 to 2^20), `ld_x` >= width apart. rows: tokens * top_k rows, contiguous. offsets, places: as skew_dispatch_order
 * made them (a place outside [0, tokens * top_k) is none). No output may overlap an input. Rows that start on 16-byte boundaries, of a width that 8
 * divides, enable vector accesses.
 */
int skew_dispatch_spread(const skew_dispatch_config_t *c, const void *x, int64_t ld_x, const int32_t *offsets, const int32_t *places, int64_t tokens,
                         int64_t width, void *rows, void *stream);
/* weights: (tokens, top_k) fp32, contiguous, or NULL: ones. */
int skew_dispatch_combine(const skew_dispatch_config_t *c, const void *rows, const float *weights, const int32_t *places, int64_t tokens, int64_t width,
                          void *out, int64_t ld_out, void *stream);
int skew_dispatch_combine_grad(const skew_dispatch_config_t *c, const void *dout, int64_t ld_dout, const void *rows, const float *weights,
                               const int32_t *offsets, const int32_t *places, int64_t tokens, int64_t width, void *drows, float *dweights, void *stream);

/* ---- products grouped by expert -------------------------------------------------
 * Rows ordered by expert, as skew_dispatch_spread makes them: those of expert e are [offsets[e], offsets[e + 1]), any number
 * of them. With E = experts matrices W_e of n x m in one array (E, n, m), as a stack of skew_create's:
 *   product    y[r]  = x[r] W_e                       x (rows, n), y (rows, m)
 *   grad_rows  dx[r] = dy[r] W_e^T
 *   grad       dW_e  = base_e + sum over its rows r of x[r]^T dy[r]
 * x, dy and W are bf16; sums are fp32 on the tensor cores, whose additions round towards zero (fp32 results are off by some 5e-7 of a sum of products of one sign, bf16
 * ones by up to 8e-6 before they are rounded, once). Rows of no expert (before offsets[0] and from
 * offsets[E] on) give zeros, and enter no dW, whatever they hold. Offsets are read on the device and taken as they come: one
 * below the one before counts as that one, one beyond `rows` as `rows`. Results do not depend on timing.
 */
#define SKEW_EXPERTS_ROWS_FP32 1u /* y and dx are fp32 (else bf16)    */
#define SKEW_EXPERTS_GRAD_FP32 2u /* base and dW are fp32 (else bf16) */

/* experts 1 to 1024; n, m 1 to 2^20. */
typedef struct {
    int32_t experts, n, m;
    uint32_t flags; /* SKEW_EXPERTS_* */
} skew_experts_config_t;

/*
 * rows: 0 to 2^30; x and dy have rows `ld` elements apart (at least their width), y, dx, W and dW are contiguous. offsets: experts + 1. No output may overlap
 * an input. Pointers aligned to their types; rows that start on 16-byte boundaries (W: n and m that 8 divides) are much quicker. The kernel's waits on
 * the device are bounded: see skew_ops_sync_status. Errors: SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_experts_product(const skew_experts_config_t *c, const void *x, int64_t ld_x, const void *w, const int32_t *offsets, int64_t rows, void *y, void *stream);
int skew_experts_grad_rows(const skew_experts_config_t *c, const void *dy, int64_t ld_dy, const void *w, const int32_t *offsets, int64_t rows, void *dx,
                           void *stream);
/* Bytes of device workspace that skew_experts_grad needs, for any number of rows (0 for an invalid config); how many SMs the current device has enters. */
size_t skew_experts_workspace_bytes(const skew_experts_config_t *c);
/*
 * base: NULL, a tensor like dW that overlaps nothing else, or dW itself, to which the gradient is then added; matrices of experts without rows are
 * then not touched. workspace: 256-byte aligned, of any content; calls that share one must not overlap on the GPU.
 */
int skew_experts_grad(const skew_experts_config_t *c, const void *x, int64_t ld_x, const void *dy, int64_t ld_dy, const int32_t *offsets, int64_t rows,
                      const void *base, void *dw, void *workspace, size_t workspace_bytes, void *stream);

/* ---- the output head's softmax cross entropy, without its logits ------------------
 * With h (tokens, width), the table W (rows, width) that the embedding may share, and l[t, v] = scale * <h[t], W[v]>:
 *   lse[t]  = log sum over v of exp(l[t, v])
 *   loss[t] = lse[t] - l[t, target_t]
 *   dh[t]   = scale * sum over v of p[t, v] W[v],  dW[v] = base[v] + scale * sum over t of p[t, v] h[t]
 *   p[t, v] = dloss[t] * (exp(l[t, v] - lse[t]) - [v = target_t])
 * A target outside [0, rows) is padding: its loss is zero, its dloss is not read, and neither it nor its h, NaN included, enters a gradient. h, W, dh, base and dW
 * are bf16. l is summed in fp32 and never stored; the gradients take the vocabulary in pieces and make a piece's p from l anew, rounded to bf16 (for the
 * tensor cores: an error of up to 2^-8 of each term, about that of rounding the result), with sums in fp32. Both sum l alike, so that at a target that is nearly
 * certain exp(l - lse) - 1 is off by fp32's rounding of lse alone besides (some 2^-21 of its size). Results do not depend on timing.
 */
#define SKEW_HEAD_IDS_64 1u /* targets are int64 (else int32) */

/* rows 1 to 2^24, width 1 to 2^20, scale finite. */
typedef struct {
    int64_t rows, width;
    float scale;
    uint32_t flags; /* SKEW_HEAD_* */
} skew_head_config_t;

/*
 * Bytes of device workspace that the loss, or its gradients, of `tokens` tokens (0 to 2^24) need (0 for an invalid config). Room for a copy of h is among them: the loss
 * makes it of rows off 16-byte boundaries alone. How many SMs the current device has enters the gradients'.
 */
size_t skew_head_loss_workspace_bytes(const skew_head_config_t *c, int64_t tokens);
size_t skew_head_grad_workspace_bytes(const skew_head_config_t *c, int64_t tokens);
/*
 * h: rows `ld_h` >= width elements apart; table: contiguous; loss, lse: fp32, one for each token. Rows on 16-byte boundaries, of a
 * width that 8 divides, are much quicker. workspace: 256-byte aligned, of any content; calls that share one must not overlap on the GPU. Waits on the device are
 * bounded: see skew_ops_sync_status. Errors: SKEW_EINVAL, SKEW_ECUDA.
 */
int skew_head_loss(const skew_head_config_t *c, const void *h, int64_t ld_h, const void *table, const void *targets, int64_t tokens, float *loss, float *lse,
                   void *workspace, size_t workspace_bytes, void *stream);
/*
 * lse: as skew_head_loss made it; dloss: fp32, one for each token; dh (tokens, width) and dtable: contiguous. base: NULL, a tensor like dtable that
 * overlaps nothing else, or dtable itself, to which the gradient is then added (rounded once).
 */
int skew_head_grad(const skew_head_config_t *c, const void *h, int64_t ld_h, const void *table, const void *targets, int64_t tokens, const float *lse,
                   const float *dloss, void *dh, const void *base, void *dtable, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Synchronises `stream` and reports whether a bounded wait on the device, of any skew_experts_* or skew_head_* kernel on the current device, has
 * given up since the last such call (SKEW_ETIMEOUT; what that call wrote is then not to be used). Errors: also SKEW_ECUDA.
 */
int skew_ops_sync_status(void *stream);
/* Self-test of that: enqueues one such wait, for what nothing completes; it gives up after some four seconds. Errors: SKEW_ECUDA. */
int skew_ops_selftest_wait_timeout(void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SKEWADAM_H_ */
