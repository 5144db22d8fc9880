/*
 * hieravg.h -- C ABI of the Hier-AVG data-parallel hot path on one MI355X.
 *
 * Hier-AVG (Zhou & Cong, "A Distributed Hierarchical Averaging SGD
 * Algorithm: Trading Local Reductions for Global Reductions", arXiv
 * 1903.05133), Algorithm 1 in Sec. 3.1: P learners each run K1 local SGD
 * steps on their own minibatch of size B, then every local cluster of S
 * learners replaces its parameters by their mean; after K2 such blocks all P
 * learners replace their parameters by the global mean.  Sec. 2 fixes
 * S | P and S >= 1.
 *
 * Units.  K2 here counts local-averaging blocks per round (the paper's beta,
 * Sec. 3.1), so one round is K1*K2 SGD steps per learner and the paper's
 * global averaging interval is K1*K2 steps.
 *
 * All P learners are rows of one replica array on one GPU; a round is a
 * sequence of kernels enqueued on the handle's HIP stream.  The handle owns
 * every device buffer it allocates; callers own the buffers they pass in.
 * A handle is not thread-safe; distinct handles are independent.
 *
 * Errors.  Functions returning int return HIERAVG_OK (0) or a negative code;
 * hieravg_last_error() then describes the failure (thread-local string,
 * valid until the next failing call on the same thread).  Constructors return
 * NULL on failure.  Asynchronous GPU faults surface as HIERAVG_EHIP at the
 * next call that synchronises.
 */
#ifndef HIERAVG_H
#define HIERAVG_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hieravg* hieravg_t;

/* Return codes. */
#define HIERAVG_OK 0
#define HIERAVG_EINVAL (-1) /* bad argument or handle                      */
#define HIERAVG_EHIP (-2)   /* HIP runtime or kernel error                 */
#define HIERAVG_ENONFINITE (-3) /* hieravg_check_finite: a replica holds inf or NaN */
#define HIERAVG_ESIZE (-4)  /* destination/source size too small / too big */

/* Model kinds (what one learner's SGD step computes). */
#define HIERAVG_KIND_SOFTMAX 0   /* softmax regression, IN -> C             */
#define HIERAVG_KIND_MLP 1       /* IN -> H (ReLU) -> C, softmax CE         */
#define HIERAVG_KIND_AVERAGING 2 /* momentum SGD on given gradients, no model */

/* Named workloads accepted by hieravg_create (the `model` argument). */
#define HIERAVG_MODEL_SOFTMAX_3072_10 0      /* N=2048, class means z, noise std 1 */
#define HIERAVG_MODEL_MLP_3072_512_10 1      /* N=50000, noise std 0.5             */
#define HIERAVG_MODEL_MLP_150528_1024_1000 2 /* N=100000, noise std 1              */
#define HIERAVG_MODEL_AVERAGING_11_7M 3      /* D=11.7e6, momentum 0.9, stds 0.01  */

/*
 * How the first weight block (W1 of the MLP) takes its SGD steps inside a
 * round.  Both give the result of Algorithm 1 up to float32 rounding.
 *  EAGER:   every step reads and writes each learner's W1 (the fused
 *           update-and-next-forward kernel).
 *  DELAYED: within a block of K1 steps each learner's W1 is its cluster's
 *           block-start copy minus lr times the sum of its steps' rank-B
 *           updates G^T X.  The forward uses the block-start copy plus the
 *           correction -lr * sum_{k'<k} (X_k X_k'^T) G_k' and the cluster
 *           mean at the block end is one update of the copy by the summed
 *           G^T X of the cluster's learners and steps.  Needs the MLP with
 *           B <= 32, K1 <= 8, K1*S*B <= 16384, whole blocks (k_global a
 *           multiple of K1), a dataset under 2^38 floats, momentum buffers
 *           that the means leave alone (avg_momentum = 0), and a round that
 *           starts with equal W1 in every replica (true after create, after
 *           every round, and after hieravg_set_params with equal W1 rows;
 *           otherwise that next round runs EAGER).  With momentum or weight
 *           decay the K1 heavy-ball steps of a block are linear in (W1, V1):
 *           W1 and its buffer at step n are fixed multiples of the block-start
 *           pair plus weighted sums of the step gradients, and the block end
 *           applies those weights in the same cluster GEMM.
 *  AUTO:    DELAYED where it applies and its extra Gram products cost at most
 *           an eighth of the step's flops ((K1 - 1) * B <= H / 2); also, with
 *           plain SGD, for 32 < B <= 128 where (K1 - 1) * B <= H and W1 holds
 *           2^19 floats or more (B, H, W1 padded to 16, 64, 64 x 64) and its
 *           buffers fit in memory; else EAGER.
 */
#define HIERAVG_UPDATE_AUTO 0
#define HIERAVG_UPDATE_EAGER 1
#define HIERAVG_UPDATE_DELAYED 2

/*
 * Full description of a workload.  Synthetic data, minibatch draws, initial
 * parameters and (averaging kind) the given gradients are all generated on
 * the GPU from `seed` with the SplitMix64 counter generator (Steele, Lea &
 * Flood, OOPSLA 2014), H(key, c) = mix64(key + (c + 1) * 0x9E3779B97F4A7C15):
 *   sample s of learner j at global step t: H(k_index, t<<32 | j<<16 | s) mod N
 *   label of row i:                         H(k_label, i) mod C
 *   X[i][d] = fp32(mu[y_i][d] + noise_std * z(k_noise, i*IN + d)),
 *   mu[c][d] = z(k_mean, c*IN + d),  z = exact Irwin-Hall(12) normal surrogate,
 *   weights (2u - 1) * fp32(1/sqrt(fan_in)), u = (H(k_init, layer<<48 | e) >> 40) / 2^24,
 *   biases 0; averaging kind: w0[d] = fp32(init_std * z(k_init, d)) and
 *   gradient of learner j at step-in-round k: fp32(grad_std * z(k_grad, (k*2^16 + j)*D + d)).
 * Stream keys are k_x = H(seed, tag_x) for fixed 64-bit tags.
 */
typedef struct hieravg_config {
  int32_t P;        /* learners, 1 <= P < 65536                            */
  int32_t S;        /* learners per local cluster, S | P                    */
  int32_t K1;       /* local SGD steps per block, >= 1                      */
  int32_t K2;       /* blocks per round (the paper's beta), >= 1            */
  int32_t B;        /* minibatch size, 1 <= B < 65536 (ignored: averaging)  */
  int32_t kind;     /* HIERAVG_KIND_*                                        */
  int64_t in_dim;   /* softmax/MLP: input features; averaging: D            */
  int64_t hidden;   /* MLP hidden width; 0 otherwise                        */
  int64_t classes;  /* softmax/MLP classes; 0 for averaging                 */
  int64_t n_samples;/* dataset rows N (softmax/MLP), N < 2^32               */
  float noise_std;  /* data noise std                                       */
  float lr;         /* step size gamma, finite and >= 0                     */
  float momentum;   /* heavy-ball coefficient mu in [0, 1) (every kind):    */
                    /*   d = g + weight_decay*w, v <- mu*v + d, w <- w - lr*v */
  float init_std;   /* averaging kind: std of the initial replica           */
  float grad_std;   /* averaging kind: std of the given gradients           */
  uint64_t seed;
  int32_t update_mode; /* HIERAVG_UPDATE_* (how the first weight block is updated) */
  int32_t k_global;    /* SGD steps per round (the paper's global interval K2 in steps,
                          Sec. 3.1); 0: K1*K2.  When set, K2 is not used: a local mean
                          follows every K1 steps of the round except its last step, which
                          takes the global mean, so a round of k_global steps that K1
                          does not divide ends with a shorter block (a non-integer beta);
                          the count of local steps restarts at every global mean */
  float weight_decay;  /* L2 coefficient lambda >= 0 of the step above; with
                          momentum = weight_decay = 0 the step is Algorithm 1's
                          plain SGD step.  The paper states no optimizer beyond
                          SGD; these follow the usual heavy-ball convention.
                          The MLP's schedules with either set: see
                          HIERAVG_UPDATE_*; softmax runs EAGER updates. */
  int32_t avg_momentum; /* 1: every local and global mean also averages the
                           momentum buffers v; 0: v stays per learner (Algorithm 1
                           averages parameters only) */
} hieravg_config;

/*
 * Create a handle for one of the named workloads (HIERAVG_MODEL_*), as
 * Algorithm 1's first line: builds the dataset, draws the initial global
 * parameter w~_1 and copies it into all P replica rows.  Blocks until the
 * set-up kernels have finished.  Returns NULL (and sets the last error) on
 * invalid arguments (P<1, S<1, S not dividing P, K1<1, K2<1, B<1, P or B >=
 * 65536, lr not finite or negative, unknown model) or allocation failure.
 */
hieravg_t hieravg_create(int32_t P, int32_t S, int32_t K1, int32_t K2, int32_t model, float lr,
                         int32_t B, uint64_t seed);

/* Same, for an explicit workload description (any dimensions).  Also NULL for
 * an update_mode outside HIERAVG_UPDATE_* or DELAYED where it does not apply. */
hieravg_t hieravg_create_config(const hieravg_config* cfg);

/*
 * Enqueue one round (one outer iteration n of Algorithm 1): K2 blocks of K1
 * local SGD steps, a local mean over each cluster after every block but the
 * last, and the global mean at the end (the local mean right before the
 * global mean does not change the exact result and is skipped).
 * Asynchronous with respect to the host.  The first call captures the
 * round's kernels into a HIP graph; later calls launch that graph on the
 * handle's current stream (while profiling, the kernels are launched one by
 * one instead).  Returns HIERAVG_OK or an error.
 */
int hieravg_round(hieravg_t h);

/*
 * Synchronise the handle's stream and copy all replicas to `dst` as a dense
 * row-major [P][D] float32 array (D = hieravg_dim(h)), each row packed as
 * softmax [W (C x IN row-major) | b (C)], MLP [W1 (H x IN) | b1 (H) |
 * W2 (C x H) | b2 (C)], averaging [w (D)].  `dst` may be host or device
 * memory; `n_floats` is its capacity and must be >= P*D (else HIERAVG_ESIZE).
 */
int hieravg_params(hieravg_t h, float* dst, size_t n_floats);

/* Overwrite all replicas from a dense [P][D] array laid out as above (host
 * or device memory, n_floats >= P*D).  Momentum buffers are left as they are.
 * Synchronous.  When every replica's first weight block is then the same
 * (a checkpoint taken at a round boundary), the next round may take delayed
 * updates; otherwise it runs EAGER. */
int hieravg_set_params(hieravg_t h, const float* src, size_t n_floats);

/* The momentum buffers v of all learners, copied out / in as a dense [P][D]
 * array in the layout of hieravg_params (host or device memory, n_floats >=
 * P*D, else HIERAVG_ESIZE).  Synchronous.  HIERAVG_EINVAL when the handle has
 * no buffers (momentum = 0: the step keeps no state). */
int hieravg_momentum(hieravg_t h, float* dst, size_t n_floats);
int hieravg_set_momentum(hieravg_t h, const float* src, size_t n_floats);

/*
 * Minibatch size of the rounds enqueued from now on (a per-round schedule
 * B_n, Thm 3.3), 1 <= B <= the B given at create (the buffers' capacity).
 * The draws of sample s keep their counters, so the first B samples of a
 * step are the same for any B.  Synchronises; the next round rebuilds its
 * launch plan.  HIERAVG_EINVAL for the averaging kind or B out of range.
 */
int hieravg_set_batch(hieravg_t h, int32_t B);

/*
 * Step size of the rounds enqueued from now on (a per-round schedule, e.g.
 * the step decay 0.1 -> 0.01 of Sec. 4 or the gamma_n of Thm 3.3).  The value
 * lives in device memory and every kernel reads it, so a change needs no new
 * launch plan.  Synchronises the handle's stream.  HIERAVG_EINVAL for a
 * non-finite or negative lr.
 */
int hieravg_set_lr(hieravg_t h, float lr);

/*
 * Quality of one replica's model (softmax or MLP kinds): the mean softmax
 * cross-entropy F(w; xi) over `n_rows` rows (the empirical risk of Sec. 2)
 * and the number of rows whose first largest logit is the label's.  split 0
 * takes the training rows 0 .. n_rows-1 (n_rows <= N); split 1 takes held-out
 * rows 0 .. n_rows-1 of a second synthetic set with the same class means and
 * its own label and noise streams (labels H(k_tlabel, i) mod C, noise
 * z(k_tnoise, i*IN + d)), generated on the GPU at the first call that needs
 * them.  Runs on the handle's stream and synchronises; allocates its
 * buffers at the first call.  HIERAVG_EINVAL for the averaging kind, a bad
 * replica or split, or n_rows out of range.
 */
int hieravg_evaluate(hieravg_t h, int32_t replica, int32_t split, int64_t n_rows, double* mean_loss,
                     int64_t* correct);

/*
 * hieravg_evaluate for callers that cannot allocate device memory (code that
 * must not call hipMalloc or hipFree: tight serving or evaluation loops,
 * harnesses that forbid allocation).  Same arguments, results and errors as
 * hieravg_evaluate; it allocates nothing.  Its chunk buffers (row list,
 * split-K partials, activations, per-row losses and hits) live in one
 * file-scope device array of HIERAVG_EVAL_SCRATCH_BYTES bytes that exists
 * once on every GPU the library runs on and is held until the process ends;
 * the chunk is the largest of 4096, 2048, ..., 16 rows whose buffers fit.
 * Every call on a GPU shares that GPU's array (nothing in it needs to start
 * at zero), so calls that overlap on one GPU, from any handles or threads,
 * race and must be serialised by the caller.  Split 1 evaluates held-out
 * rows that an earlier hieravg_evaluate call of the handle generated
 * (n_rows above that count: HIERAVG_ESIZE).  A model whose 16-row chunk does
 * not fit the array (2*hidden + classes above about 262000 for the MLP,
 * classes above that for softmax regression) gets HIERAVG_ESIZE with the
 * size it would need.  Runs on the handle's stream,
 * on the handle's device, and synchronises.
 */
#define HIERAVG_EVAL_SCRATCH_BYTES ((size_t)16 << 20)
int hieravg_evaluate_noalloc(hieravg_t h, int32_t replica, int32_t split, int64_t n_rows, double* mean_loss,
                             int64_t* correct);

/*
 * The scores of single rows behind those two numbers: for rows 0 .. n_rows-1 of
 * a split (as hieravg_evaluate takes them; same errors) on replica `replica`'s
 * model the log probability of the row's label, the entropy of its distribution
 * over the classes, and the `top` <= min(classes, HIERAVG_TOP_MAX) most probable
 * classes with their log probabilities (hieravg_log_probs below, whose rules
 * hold).  logp, entropy: [n_rows]; top_ids, top_logp: [n_rows][top], or NULL for
 * top = 0; host or device memory.  Allocates; runs on the handle's stream and
 * synchronises.
 */
int hieravg_scores(hieravg_t h, int32_t replica, int32_t split, int64_t n_rows, int32_t top, float* logp,
                   float* entropy, int32_t* top_ids, float* top_logp);

/* Release every resource of the handle.  NULL-safe. */
void hieravg_destroy(hieravg_t h);

/* Thread-local description of the last failure ("" if none). */
const char* hieravg_last_error(void);

/* Parameters per replica D, or a negative code for a NULL handle. */
int64_t hieravg_dim(hieravg_t h);

/* Global SGD steps taken since creation (K1*K2 per round). */
int64_t hieravg_step_count(hieravg_t h);

/* Divergence check: synchronise and scan every replica; HIERAVG_OK when all
 * parameters are finite, HIERAVG_ENONFINITE when any is inf or NaN (for
 * example after a step size too large for the data). */
int hieravg_check_finite(hieravg_t h);

/* Set the global step counter t (t >= 0): the next round draws its
 * minibatches for steps t, t+1, ...  With hieravg_set_params (and
 * hieravg_set_momentum) this resumes a run exactly from a checkpoint taken
 * at a round boundary.  Synchronous; HIERAVG_EINVAL for t < 0. */
int hieravg_set_step_count(hieravg_t h, int64_t t);

/*
 * Copy the minibatch indices the last round drew, as int32 [T][P][B] with T
 * the steps per round (K2*K1 or k_global) and B the current minibatch size
 * (hieravg_set_batch), to `dst` (host or device,
 * n >= T*P*B).  Synchronises.  HIERAVG_EINVAL for the averaging kind (it
 * draws no samples).
 */
int hieravg_last_indices(hieravg_t h, int32_t* dst, size_t n);

/*
 * Make the handle enqueue on `hip_stream` (a hipStream_t, e.g. a torch
 * stream's handle; NULL selects the handle's own stream).  The caller keeps
 * ownership of the stream and must keep it alive while the handle uses it.
 * Synchronises the previous stream first.
 */
int hieravg_set_stream(hieravg_t h, void* hip_stream);

/* Block until all work enqueued by the handle has finished. */
int hieravg_sync(hieravg_t h);

/*
 * Per-kernel timing with HIP events: while enabled, every launch carries two
 * events that its dispatch packet stamps at kernel start and end, so the
 * recorded durations are the kernels' execution times.  enable != 0 starts
 * recording (clearing earlier records); enable == 0 stops.  hieravg_profile_read synchronises and writes, for every
 * kernel class c < min(n, hieravg_kernel_classes()), the number of launches
 * and their summed duration in milliseconds.
 */
int hieravg_profile(hieravg_t h, int enable);
int hieravg_profile_read(hieravg_t h, int64_t* launches, double* total_ms, int n);
int hieravg_kernel_classes(void);

/*
 * Mean duration in milliseconds of one launch of kernel class
 * `kernel_class` (see hieravg_kernel_class_name), from HIP events around one
 * launch of a graph of `reps` back-to-back launches of it (captured on the
 * handle's stream) with the arguments of step 0 of the current round.  For
 * measurement only: the launches act on the replicas as `reps` extra
 * applications of that kernel would.  HIERAVG_EINVAL for a class the workload
 * does not launch, for the index draw, or while profiling.  Synchronises.
 */
int hieravg_time_kernel(hieravg_t h, int kernel_class, int reps, double* mean_ms);
const char* hieravg_kernel_class_name(int c);

/* ------------------------------------------------------------------ tensor operators
 *
 * The last layer of a model with many classes, on tensors of the caller:
 * scores of given labels and their gradient, an optimizer step with two
 * moments, the norm of many gradients and their clipping, products in 8-bit
 * floating point, low-rank adapters of many requests beside such a product, and
 * the verification of drafted tokens.  The pointers are device
 * memory of the current device; `hip_stream` is a stream of it (a hipStream_t;
 * NULL: the device's default stream).  Calls enqueue their kernels there and
 * return: they neither synchronise nor allocate (hieravg_adamw_create, _steps,
 * _lr and _destroy excepted), so a HIP graph may capture them.  Calls on
 * different streams may overlap where their outputs and scratch differ.
 * Outputs overlap no input but where that is said.  No float atomics: equal
 * inputs give equal bits.
 */

/* Element types. */
#define HIERAVG_F32 0
#define HIERAVG_F16 1
#define HIERAVG_BF16 2

/*
 * Per row x of `rows` rows of `classes` logits (row_stride >= classes elements
 * apart; 1 <= classes <= 2^23), in float32:
 *   lse     log sum_j exp x_j
 *   logp    x_label - lse; 0 for a label < 0 (a row without one), NaN for a
 *           label >= classes.  `labels` holds integers of label_bytes = 4 or 8.
 *   entropy -sum_j p_j log p_j of p_j = exp(x_j - lse) (0 log 0 = 0)
 *   top_ids, top_logp [rows][top]  the `top` <= min(classes, HIERAVG_TOP_MAX)
 *           largest logits in falling order, of equal ones the lowest index
 *           first (-0 equals 0; NaN, if any, before everything), and their
 *           log probabilities.
 * A row that holds NaN or +infinity, or nothing but -infinity, has no
 * distribution: its values are NaN (logp stays 0 where there is no label),
 * its top_ids still those of the order.  Any of logp (then labels too may be
 * NULL), entropy, lse and the top pair (top = 0) may be NULL.  `scratch`: at
 * least hieravg_log_probs_scratch bytes (0: may be NULL), 16-byte aligned,
 * free to reuse when the call's kernels are done.
 */
#define HIERAVG_TOP_MAX 64
size_t hieravg_log_probs_scratch(int64_t rows, int64_t classes, int32_t top);
int hieravg_log_probs(const void* logits, int32_t type, int64_t rows, int64_t classes, int64_t row_stride,
                      const void* labels, int32_t label_bytes, int32_t top, float* logp, float* entropy, float* lse,
                      int32_t* top_ids, float* top_logp, void* scratch, size_t scratch_bytes, void* hip_stream);

/*
 * The gradient of sum_rows (g_logp * logp + g_entropy * entropy) in the
 * logits, with lse and entropy as the forward left them:
 *   grad_j = g_logp ([j = label] - p_j) - g_entropy p_j (log p_j + entropy),
 * the first term 0 for a label < 0, NaN for a label >= classes (whatever its
 * weight).  Other rows whose two weights are 0 (or absent) get zeros whatever
 * their logits; rows without a distribution NaN.  Past |lse| = 64, where float32
 * holds few digits of it, an lse that is the row's own to its rounding is taken
 * again from the row's logits; any other (that of a longer row, of which these
 * are a part) as it is.  p_j below 2^-126 count as 0.  g_logp (with labels) or g_entropy (with entropy) may be
 * NULL.  grad has the logits' type, rows grad_stride elements apart, each
 * value rounded once; it may be the logits themselves (same pointer and
 * stride), and is refused where its rows overlap theirs otherwise.
 */
int hieravg_log_probs_grad(const void* logits, int32_t type, int64_t rows, int64_t classes, int64_t row_stride,
                           const void* labels, int32_t label_bytes, const float* lse, const float* entropy,
                           const float* g_logp, const float* g_entropy, void* grad, int64_t grad_stride,
                           void* hip_stream);

/*
 * AdamW (decoupled weight decay) over many tensors at once.  Step t = 1, 2, ..:
 *   m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g g,
 *   w <- w (1 - lr decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * in float32 (each product and sum of the first line rounded by itself), w
 * rounded once to its type.  `copy` (optional): w rounded to copy_type
 * as well, the working copy of a float32 parameter.
 *
 * The moments of all tensors lie one after the other in m and v, each tensor's
 * at a multiple of 128 elements: element i of tensor k at s = 128 * sum_{j<k}
 * ceil(n_j / 128) + i, hieravg_adamw_state_size elements in all, zeroed by the
 * caller before the first step.  state_bits 32: float32.  state_bits 8: blocks
 * of 128 elements share one scale byte per moment, 2^(byte - 127) (255: NaN),
 * the least power of two that holds the block; m is E4M3 (sign, 4 exponent
 * bits of bias 7, 3 fraction bits); v is 4 exponent and 4 fraction bits, code
 * c = 16 e + f meaning (16 + f) 2^(e - 19), or f 2^-18 for e = 0.  Both are
 * rounded to a neighbour at random, with the odds that keep the mean (with
 * nearest rounding the slow average v would not move: at beta2 = 0.999 a step
 * changes it by less than half a step of any 8-bit format); a v above 0 keeps
 * a code above 0.  The random bits of step t are those of H(H(H(seed,
 * "hv.adamw"), t), s / 2) (the SplitMix64 counter of hieravg_config): its low
 * half for even s, its high half for odd s, 16 low bits for m, 16 for v.  The
 * step itself uses the moments before they are rounded.  A block with an
 * infinite or NaN moment becomes NaN.  The rest of a tensor's last block steps
 * like an element with gradient 0 (zeros stay zeros).
 *
 * create takes the tensors as they will be (parameters, copies, sizes, types;
 * nothing is read from them) and keeps the pointers, so their memory must
 * outlive the handle.  NULL on bad arguments: n < 1 tensors, sizes < 0,
 * lr or weight_decay not finite or negative, betas outside [0, 1), eps not a
 * float32 of at least 2^-126, state_bits other than 8 and 32, parameters or
 * copies that overlap.  One thread uses a handle at a time; the caller orders
 * the streams of its calls, and destroys it when their kernels are done.
 * step: grads[k] is tensor k's gradient of its grad_type, or NULL: the tensor
 * and its moments stay as they are.  Elements are addressed one after the
 * other (contiguous tensors, aligned to their element).  The count of steps
 * (one for all tensors) and lr live in device memory: a captured step counts
 * at every replay and takes the lr set last.  set_lr and set_steps are
 * ordered on their stream with the steps; steps and lr wait for the device.
 */
typedef struct hieravg_adamw* hieravg_adamw_t;
typedef struct hieravg_adamw_config {
  double lr, beta1, beta2, eps, weight_decay;
  uint64_t seed;
  int32_t state_bits;
} hieravg_adamw_config;
typedef struct hieravg_adamw_tensor {
  void* param;
  void* copy; /* or NULL */
  int64_t n;
  int32_t param_type, grad_type, copy_type;
} hieravg_adamw_tensor;
int64_t hieravg_adamw_state_size(const int64_t* n, int32_t count);
hieravg_adamw_t hieravg_adamw_create(const hieravg_adamw_config* cfg, const hieravg_adamw_tensor* tensors,
                                     int32_t count, void* m, void* v, uint8_t* m_scales, uint8_t* v_scales);
int hieravg_adamw_step(hieravg_adamw_t h, const void* const* grads, void* hip_stream);
/* The same on gradients times *factor (a float32 in device memory, as
 * hieravg_grad_norm leaves it; each product rounded to float32; NULL: 1).  Refused
 * where it lies in a parameter, a copy or a moment. */
int hieravg_adamw_step_scaled(hieravg_adamw_t h, const void* const* grads, const float* factor, void* hip_stream);
int hieravg_adamw_set_lr(hieravg_adamw_t h, double lr, void* hip_stream);
int hieravg_adamw_set_steps(hieravg_adamw_t h, int64_t t, void* hip_stream);
int64_t hieravg_adamw_steps(hieravg_adamw_t h);
int hieravg_adamw_lr(hieravg_adamw_t h, double* lr);
void hieravg_adamw_destroy(hieravg_adamw_t h);

/*
 * Matrices in 8-bit floating point (E4M3, largest value 448) with a scale for
 * each block of 128 along the rows.  Block form of an R x K matrix: codes
 * [R][Kp], Kp = K rounded up to 128 (the padding holds zeros), and scale bytes
 * [Rb][Sp] of one power of two 2^(byte - 127) per block, Sp = Kp / 128 rounded
 * up to 4 (padding 0); Rb = R (1 x 128 blocks) or, with tiles,
 * Rb = ceil(R / 128) (128 x 128 blocks).  Codes start at a multiple of 16 bytes, scales of 4.
 *
 * quantize_blocks: from x, R rows of K elements row_stride >= K apart.  A
 * block's scale is the least 2^e, -127 <= e <= 127, with |x| <= 448 * 2^e for its finite
 * values (1 if all are 0), its codes x / 2^e rounded to nearest even; NaN and
 * infinities become NaN.  `codes`, `scales`: the block form of x;
 * `codes_t`, `scales_t`: that of its transpose (blocks of 128 rows of x; with
 * tiles the same blocks), from the same reading of x.  Either pair may be
 * NULL.
 *
 * block_product: out[i][j] = sum_k a[i][k] b[j][k] over two block forms of m x
 * k and n x k, k <= 2^23: the products exact, their sums in float32, rounded
 * once to out_type, HIERAVG_F16 or HIERAVG_BF16, rows out_stride apart.  (The
 * values that codes and scales stand for are taken as bf16 holds them: exact
 * from 2^-126 on, infinite from 2^128 on, multiples of 2^-133 below.)  With x, W, dy of a layer y = x W^T in
 * block form: y = product(x, W), dx = product(dy, W transposed), dW =
 * product(dy transposed, x transposed).  `scratch` as for hieravg_log_probs.
 */
int hieravg_quantize_blocks(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t row_stride,
                            int32_t tiles, uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t,
                            void* hip_stream);
size_t hieravg_block_product_scratch(int64_t m, int64_t n, int64_t k);
int hieravg_block_product(const uint8_t* a, const uint8_t* a_scales, int32_t a_tiles, const uint8_t* b,
                          const uint8_t* b_scales, int32_t b_tiles, int64_t m, int64_t n, int64_t k, void* out,
                          int32_t out_type, int64_t out_stride, void* scratch, size_t scratch_bytes,
                          void* hip_stream);

/*
 * The norm of many gradients and their clipping.  A tensor: n >= 0 contiguous
 * elements, aligned to their element; data NULL counts as empty.
 *
 * grad_norm: norms[k] = sqrt(sum g^2) of tensor k, norm that of all together,
 * factor = 1 where norm <= max_norm, else max_norm / norm (NaN for a NaN norm, 0
 * for an infinite one past a finite max_norm).  Squares are added in
 * float32 by eights at most, off by 4 2^-24 of their sum, and these sums in 64 bits; the
 * results, off by 2 2^-24 so, are rounded once.  max_norm >= 0, or infinite.  Any of the
 * three results may be NULL, not all of them.  `scratch` as for
 * hieravg_log_probs.
 *
 * scale_tensors: out[k] = in[k] times *factor, rounded once to in[k]'s type (and
 * to float32 before that).  out[k] may be in[k].data, and is refused where it
 * overlaps any tensor otherwise, another result or factor.  out[k] of an empty tensor is not looked at.
 */
typedef struct hieravg_tensor {
  const void* data;
  int64_t n;
  int32_t type;
} hieravg_tensor;
size_t hieravg_grad_norm_scratch(const hieravg_tensor* grads, int32_t count);
int hieravg_grad_norm(const hieravg_tensor* grads, int32_t count, double max_norm, float* norms, float* norm,
                      float* factor, void* scratch, size_t scratch_bytes, void* hip_stream);
int hieravg_scale_tensors(const hieravg_tensor* in, void* const* out, int32_t count, const float* factor,
                          void* hip_stream);

/*
 * Verification of drafted tokens against a target model, from given random
 * numbers.  Per sequence s of `seqs`: n = lengths[s] drafts (clamped to [0, drafts];
 * NULL: `drafts` each), the target's logits of drafts + 1 rows, row i those
 * before draft i and row n those after the last, the draft model's of `drafts`
 * rows, and a temperature T (NULL: 1).  With p_i = softmax(target row i / T) and q_i
 * = softmax(draft row i / T), draft x_i is accepted while
 *   u_i q_i(x_i) < p_i(x_i),  u_i = uniforms[s][i] in [0, 1).
 * The first that is not is replaced by a token of the distribution
 * max(p_i - q_i, 0) / sum, and after the last accepted one comes one of p_n; the token is
 * the lowest class whose running sum of weights passes uniforms[s][drafts]
 * times their whole sum.  (Where p_i = q_i: of p_i.)  draft_logits NULL: q_i is 1 at x_i.
 * A T that is not above 0 and finite stands for its limit 0: a draft is accepted if it is
 * the row's largest class (of equal ones the lowest index), which is also the
 * token in its place, and the draft's logits are not looked at.
 *
 * tokens [seqs][drafts + 1]: the accepted drafts, the drawn token, then -1;
 * accepted [seqs]: how many; logp [seqs][drafts + 1]: log p_i of each token (0 at T = 0 and
 * beside -1).  A draft outside [0, classes) is not accepted.  Where a row that decides has
 * no distribution (NaN, +infinity, or nothing but -infinity), its draft is not
 * accepted and the token is -1.
 * All comparisons that float32 cannot settle and all draws are made in 64 bits, and
 * so is the drawn token's logp; that of an accepted draft comes from a float32 sum and
 * is off by (classes / 256 + 110) 2^-24 at most, beside its rounding.
 * Rows are row_stride (draft_stride) >= classes elements apart, those of a
 * sequence one after the other; classes <= 2^23; draft_tokens [seqs][drafts] of
 * token_bytes 4 or 8.  `scratch` as for hieravg_log_probs.
 */
#define HIERAVG_DRAFTS_MAX 64
size_t hieravg_verify_drafts_scratch(int64_t seqs, int32_t drafts, int64_t classes, int32_t draft_logits);
int hieravg_verify_drafts(const void* logits, int32_t type, int64_t seqs, int32_t drafts, int64_t classes,
                          int64_t row_stride, const void* draft_logits, int32_t draft_type, int64_t draft_stride,
                          const void* draft_tokens, int32_t token_bytes, const float* uniforms, const int32_t* lengths,
                          const float* temperature, int32_t* tokens, int32_t* accepted, float* logp, void* scratch,
                          size_t scratch_bytes, void* hip_stream);

/*
 * Low-rank adapters of many requests beside a shared projection.  Adapter a of
 * n: D = down[a] [rank][in], U = up[a] [rank][out] (both with the rank
 * outermost) in `type`, and a scale s (NULL: 1).  Row i takes that of ids[i], an
 * integer of id_bytes 4 or 8; below 0: none.
 *
 * adapter_product: h_i = x_i D^T,  out_i = base_i + s h_i U.
 * adapter_grad: of sum(grad * out) in x, D and U,
 *   dh_i = grad_i U^T,  dx_i = base_i + s dh_i D,
 *   ddown[a] = s sum_i dh_i^T x_i,  dup[a] = s sum_i h_i^T grad_i
 * over the adapter's rows; zeros for an adapter without rows.  (base there: the
 * gradient that comes through the shared projection.)
 *
 * x [rows][in] and grad [rows][out] are of `type`, rows their stride apart.  base
 * (NULL: zeros) and the result beside it are of out_type (dx_type), float32, `type`,
 * or any where `type` is float32; the result
 * may be base (same pointer and stride), and is refused where its rows overlap
 * those of base, x or grad otherwise, or another operand; so are hidden as a
 * result, ddown and dup where they overlap an operand or another result.  hidden [rows][rank], float32: h, written by adapter_product
 * if asked for (zeros for rows without an adapter), and taken by adapter_grad
 * in place of x D^T if given.  dx, ddown and dup may be NULL; ddown and dup are of
 * weight_type.  A row whose id is n or more gets NaN and adds to no
 * gradient; a row without an adapter gets base.
 * Sums are float32 and results rounded once; h and dh enter the second products to
 * 2^-23 of themselves or 2^-40 of their row's largest at least.  An infinite element
 * of down, up, x or grad, or an infinite h or dh, may give NaN where float32 arithmetic
 * has an infinity.  rows, in and out up to 2^24, rank up to HIERAVG_RANK_MAX, n up to
 * HIERAVG_ADAPTERS_MAX; refused are calls of 2^24 workgroups or more in a launch: tiles of
 * 64 rows by blocks of 128 to 512 columns, and for ddown and dup units of up to 4096 rows,
 * one at least for each adapter, by blocks of 64 or 128 columns and of 64 ranks.  `scratch` as for hieravg_log_probs; a gradient with ddown and
 * dup NULL needs hieravg_adapter_dx_scratch bytes only.
 */
#define HIERAVG_RANK_MAX 128
#define HIERAVG_ADAPTERS_MAX 8192
typedef struct hieravg_adapters {
  const void *down, *up;
  const float* scales;
  int64_t in, out;
  int32_t n, rank, type;
} hieravg_adapters;
size_t hieravg_adapter_product_scratch(int64_t rows, const hieravg_adapters* w);
int hieravg_adapter_product(const hieravg_adapters* w, const void* x, int64_t rows, int64_t x_stride, const void* ids,
                            int32_t id_bytes, const void* base, int64_t base_stride, void* out, int32_t out_type,
                            int64_t out_stride, float* hidden, void* scratch, size_t scratch_bytes, void* hip_stream);
size_t hieravg_adapter_grad_scratch(int64_t rows, const hieravg_adapters* w, int32_t hidden);
size_t hieravg_adapter_dx_scratch(int64_t rows, const hieravg_adapters* w);
int hieravg_adapter_grad(const hieravg_adapters* w, const void* grad, int64_t rows, int64_t grad_stride, const void* x,
                         int64_t x_stride, const void* ids, int32_t id_bytes, const float* hidden, const void* base,
                         int64_t base_stride, void* dx, int32_t dx_type, int64_t dx_stride, void* ddown, void* dup,
                         int32_t weight_type, void* scratch, size_t scratch_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* HIERAVG_H */
