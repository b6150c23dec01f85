/*
 * micro_sparsify.h -- C ABI of the MI355X (gfx950) implementation of MiCRO's
 * per-worker gradient sparsification step (Yoon & Oh, arXiv 2310.00967).
 *
 * One call of micro_sparsify_step is one worker's share of one iteration of
 * the paper's Algorithm 1, restricted to the worker's own partition:
 *
 *   Sec. 4.1  partition:  [s, e) = [floor(r*N/n), floor((r+1)*N/n))
 *   Sec. 2    error feedback accumulation:  acc_j = grad_j + residual_j
 *             (one binary32 addition, round to nearest even, no fused
 *             multiply-add, subnormals kept)
 *   Sec. 4.2  exclusive selection:  j is selected iff |acc_j| >= theta
 *             (the binary32 magnitude compared with the binary64 threshold)
 *   Alg. 1    the selected pairs (j, acc_j), in increasing j, go to
 *             out_idx / out_val; residual_j becomes +0 where j is selected
 *             and acc_j elsewhere in [s, e)
 *   Sec. 4.3  threshold scaling:  theta <- Estimate(d * P, k, theta), in
 *             binary64 on the host from the selected count k
 *
 * Every function is extern "C", takes plain pointers and sizes, and reports
 * failure through micro_status; no C++ exception crosses the ABI.  Pointers
 * documented as "device" are HIP device addresses on the device that was
 * current when the context was created; "host" pointers are ordinary host
 * memory.  The caller owns every buffer it passes.
 *
 * Typical use, one worker of `world` over a gradient of n values already in
 * device memory (error handling shortened):
 *
 *   micro_ctx *ctx;
 *   micro_sparsify_init(&ctx, n, stream, NULL);          // NULL: default rule
 *   double theta = theta0;                               // e.g. a calibrated start
 *   for (int64_t t = 0; t < steps; ++t) {
 *       int32_t part; int64_t k;
 *       micro_cycle(t, worker, world, &part);            // Algorithm 1's rotation
 *       micro_sparsify_step(ctx, grad, residual, part, world, density, &theta,
 *                           out_idx, out_val, &k);       // out_* hold k pairs
 *       ... exchange out_idx[0, k) / out_val[0, k) with the other workers ...
 *   }
 *   micro_sparsify_free(ctx);
 */
#ifndef MICRO_SPARSIFY_H
#define MICRO_SPARSIFY_H

#include <stdint.h>

#if defined(__GNUC__)
#define MICRO_API __attribute__((visibility("default")))
#else
#define MICRO_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct micro_ctx micro_ctx; /* opaque, owned by the library */

typedef enum micro_status {
    MICRO_OK = 0,
    MICRO_EINVAL = 1,    /* an argument is invalid; nothing was modified        */
    MICRO_ECAPACITY = 2, /* a size exceeds what the context was created for     */
    MICRO_ERANGE = 3,    /* n_total does not fit int32 global indices           */
    MICRO_ENOMEM = 4,    /* a device or pinned host allocation failed           */
    MICRO_EHIP = 5       /* a HIP runtime call failed (see micro_last_error)    */
} micro_status;

/* Threshold update rules (readings of Sec. 4.3, which gives no formula). */
#define MICRO_RULE_PROPORTIONAL 0 /* theta * clamp(1 + beta*(k - k*)/k*, lo, hi) */
#define MICRO_RULE_FIXED_STEP 1   /* theta * (1 + alpha) if k > k*,
                                     theta * (1 - alpha) if k < k*, else theta   */
#define MICRO_RULE_HARD_THRESHOLD 2 /* theta never changes: the hard-threshold
                                       sparsifier the paper compares with
                                       (Sec. 1, Sec. 5.2), a fixed threshold  */
#define MICRO_RULE_TOPK 3 /* the exact top-k sparsifier the paper compares
                             with (Sec. 1: the k largest gradients; its density
                             footnote: d = k / n_g).  Not a threshold rule: the
                             step selects the k = max(1, floor(d * P)) values
                             of [s, e) whose accumulated magnitude is largest,
                             equal magnitudes by lower index, NaN never (so
                             fewer than k when fewer than k are not NaN).  The
                             incoming theta is not checked and does not change
                             the result: when it is positive and finite it is
                             a hint for the k-th magnitude (pass on the theta
                             the last step returned) and sets where the step
                             looks first.  theta receives the smallest
                             selected magnitude (0 or +inf possible; unchanged
                             when nothing is selected).  Through
                             micro_sparsify_step and micro_ef_step only
                             (MICRO_EINVAL in micro_sweep_step,
                             micro_sparsify_step_noalloc and
                             micro_estimate_threshold).  The k-th magnitude is
                             found by a radix select: three histogram passes
                             over the keys and a one-workgroup select after
                             each.  With a hint (and k <= P / 8, STAGED or
                             AUTO) the threshold step runs first at 7/8 of it
                             or closer (up to 511/512, as the last steps' k-th
                             magnitudes allowed), the select runs over its
                             output list and a trim cuts that to the top k,
                             enqueued together; if that list holds
                             fewer than k values, they go back into the
                             residual and the select starts over on the
                             partition's residual.  Without one
                             the passes run over the partition first (waited
                             for), then the step at the k-th magnitude or at
                             the floor of its first digit, then the passes
                             left and the trim over its list.               */
#define MICRO_TOPK_ROUTE_FULL 1      /* micro_step_stats.topk_route: three passes over the partition, then the step */
#define MICRO_TOPK_ROUTE_LIST 2      /* one pass over the partition, the step, two passes over its list */
#define MICRO_TOPK_ROUTE_HINT_LIST 3 /* the step at the hint's bound, the select over its list */
#define MICRO_TOPK_ROUTE_HINT_PICK 4 /* the step at the hint's bound listed fewer than k: one pass over the
                                        residual, then the values from the k-th magnitude's first-digit bin
                                        up extracted and two passes over them (or the passes and a pick
                                        over the residual) */

/* Kernel schedules (both compute the same result). */
#define MICRO_VARIANT_AUTO 0   /* per call, the faster measured schedule: TICKET
                                  for partitions of up to 2^20 values, STAGED
                                  above, which up to 2^22 values keeps its staged
                                  pairs in local memory and places them in the
                                  same single launch; both scratch sets         */
#define MICRO_VARIANT_TICKET 1 /* one pass, one launch: each tile's offset by
                                  decoupled look-back; tiles in launch order up
                                  to 2^22 values of the partition, drawn from a
                                  ticket counter above                           */
#define MICRO_VARIANT_STAGED 2 /* a streaming pass that stages each tile's pairs
                                  (no inter-workgroup waits), a scan pass (look-
                                  back per chunk of a million values) and a
                                  balanced pass that places them, the first two
                                  in one launch (see MICRO_FLAG_SEPARATE_SCAN);
                                  scratch of about 2 bytes per value of the
                                  vector                                          */

/* Flags. */
#define MICRO_FLAG_TIME_KERNEL 1 /* record HIP events around each launch so
                                    micro_sparsify_last_kernel_ms can report it */
#define MICRO_FLAG_SEPARATE_SCAN 2 /* STAGED: launch the scan pass on its own;
                                      by default micro_sparsify_step runs the
                                      streaming and scan passes as one launch
                                      (same result)                            */

typedef struct micro_config {
    int32_t rule;    /* MICRO_RULE_*                                  (default 0)    */
    double beta;     /* proportional gain                             (default 0.1)  */
    double lo, hi;   /* clamp of the proportional scale factor        (0.5, 2.0)     */
    double alpha;    /* fixed-step size                               (default 0.05) */
    int32_t variant; /* MICRO_VARIANT_*                               (default 0)    */
    int32_t flags;   /* MICRO_FLAG_*                                  (default 0)    */
} micro_config;

/* What the last micro_sparsify_step on a context did. */
typedef struct micro_step_stats {
    float kernel_ms;        /* device time of its kernels from HIP events
                               (MICRO_FLAG_TIME_KERNEL), else -1               */
    int32_t one_launch;     /* 1 if its step on the partition was one launch,
                               placing included (whichever schedule `variant`
                               names), 2 if a full pass accumulated the rest of
                               the vector in the same launch, else 0           */
    int64_t redone_tiles;   /* STAGED: 1024-value tiles with more selected
                               values than their staging slot holds (256),
                               redone by the placing pass instead (AUTO's
                               single launch: counted, and placed from
                               registers where four of them hold over 1024)    */
    int32_t variant;        /* the schedule of the last step, MICRO_VARIANT_TICKET
                               or MICRO_VARIANT_STAGED (AUTO above 2^20 values:
                               STAGED, also where one_launch is not 0)         */
    int32_t fused;          /* 1 if its streaming and scan passes ran as one
                               launch (micro_sparsify_step, STAGED; also where
                               the placing pass was part of it), else 0        */
    int32_t topk_route;     /* MICRO_RULE_TOPK: how the step found the k-th
                               magnitude (MICRO_TOPK_ROUTE_*); 0 for the other
                               rules, or when nothing was selectable           */
    int32_t topk_passes;    /* MICRO_RULE_TOPK: 1 if histogram passes ran; 0 where
                               the select enqueued with a hinted step found the
                               k-th magnitude in its list, and for other rules  */
} micro_step_stats;

/* Fills *cfg with the defaults listed above. */
MICRO_API void micro_config_default(micro_config *cfg);

/*
 * Creates a context for flattened gradient vectors of n_total fp32 values on
 * the current HIP device, enqueuing all work on `hip_stream` (a hipStream_t;
 * NULL means the null stream).  cfg == NULL selects the defaults.
 * The context owns its device scratch (STAGED: a 256-pair staging slot and a
 * count per 1024 values of the vector plus look-back words, about 2 bytes per
 * value; TICKET: one look-back word per 4096 values and a few, 1026 tile claims
 * and a ticket counter; AUTO: both, and 1 KB of mapped host memory) and a pinned host word
 * for the selected count; it never owns the caller's buffers.
 * Returns MICRO_EINVAL (ctx NULL, n_total < 0, bad cfg), MICRO_ERANGE
 * (n_total > INT32_MAX: indices are int32), MICRO_EHIP (no usable device) or
 * MICRO_ENOMEM.  On failure *ctx is set to NULL.  Every context also holds
 * the top-k comparator's 8 KB of radix-select counters and 64 bytes of mapped
 * host memory, and one of MICRO_RULE_TOPK another 25 KB of counters and one
 * byte of look-back words per 128 values of the vector, at least 1 KB.
 */
MICRO_API micro_status micro_sparsify_init(micro_ctx **ctx, int64_t n_total,
                                 void *hip_stream, const micro_config *cfg);

/*
 * One worker's sparsify step on partition `rank` of `world` (the paper's
 * cyclic partition number: the caller rotates it).
 *   grad      device, n_total fp32, read only; only [s, e) is read.
 *   residual  device, n_total fp32, in/out: the local error; only [s, e) is
 *             read and written, everything outside is untouched.
 *   rank, world  0 <= rank < world, world >= 1.
 *   density   the user-set density d, 0 < d <= 1; the target count is d*P.
 *   theta     host, in/out: the threshold of this step in, the threshold of
 *             the next step out.  Must be finite and > 0.  (MICRO_RULE_TOPK:
 *             the selection is the top k instead; theta in is unchecked and
 *             only a hint for where to look, theta out the k-th magnitude,
 *             see there.)
 *   out_idx   device int32, capacity >= P = e - s: the first k entries
 *             receive the selected global indices, strictly increasing.
 *   out_val   device fp32, capacity >= P: the first k entries receive acc
 *             at those indices.
 *   k         host out: the selected count.
 * The buffers grad[s,e), residual[s,e), out_idx[0,P) and out_val[0,P) must
 * not overlap.  grad and residual must be 4-byte aligned; the fastest path
 * needs them to share the same 16-byte phase.
 * The call is synchronous: it returns after the device work has finished and
 * theta has been updated.  Empty partitions (P == 0) return MICRO_OK with
 * k = 0 and theta unchanged.  Invalid arguments return MICRO_EINVAL before
 * any device work, with nothing modified.  A HIP failure returns MICRO_EHIP;
 * the outputs and the residual slice are then unspecified.
 * One context must not be used from two threads at once.
 */
MICRO_API micro_status micro_sparsify_step(micro_ctx *ctx, const float *grad,
                                 float *residual, int32_t rank, int32_t world,
                                 double density, double *theta,
                                 int32_t *out_idx, float *out_val, int64_t *k);

/*
 * micro_sparsify_step for callers that cannot allocate memory (tight serving
 * loops, harnesses that forbid hipMalloc, code that must not allocate after
 * start-up): no context, and no device or host allocation in the call.
 * It runs the one-pass schedule (MICRO_VARIANT_TICKET) with its scratch in
 * one static device array per device (4 MiB + 12.3 KB, held from the first
 * call on a device until the process ends): the count, a ticket counter, one
 * look-back word per 4096 values of the partition and one per 512 of those, and
 * 1026 tile claims, enough for any partition of up to 2^31 - 1 values.
 *   grad, residual, rank, world, density, theta, out_idx, out_val, k:
 *              as micro_sparsify_step, over a vector of n_total values on
 *              the current HIP device; same results bit for bit.
 *   hip_stream a hipStream_t of the current device (NULL: the null stream);
 *              the call enqueues its kernel and the count readback there
 *              and waits for them.
 *   cfg        NULL for the defaults; only its threshold rule (rule, beta,
 *              lo, hi, alpha) is used.
 * Calls on one device share its scratch; the library serialises them (a lock
 * per device, held until the count is read back), so they never overlap on
 * it.  Returns MICRO_ERANGE for n_total above 2^31 - 1 (the most the scratch
 * covers), MICRO_EINVAL for the argument errors of micro_sparsify_step (and
 * an invalid cfg), MICRO_EHIP on a HIP failure; messages through
 * micro_last_error(NULL) on the calling thread.
 */
MICRO_API micro_status micro_sparsify_step_noalloc(const float *grad, float *residual, int64_t n_total,
                                                   int32_t rank, int32_t world, double density,
                                                   double *theta, int32_t *out_idx, float *out_val,
                                                   int64_t *k, void *hip_stream,
                                                   const micro_config *cfg);

/*
 * Every partition r of `world` (1 <= world <= 64) searched once over one
 * vector, each with its own threshold, in one set of launches (the streaming
 * and scan passes of all partitions as one launch for vectors of up to 64
 * scan chunks of a million values, unless MICRO_FLAG_SEPARATE_SCAN, then one
 * placing launch): the selections all n workers make at one iteration
 * (Sec. 4.2), with the local error of Sec. 2 / Eq. 1 reduced on the way.
 *   grad, residual  device, n_total fp32; residual in/out over all of it.
 *   theta      host double[world], in/out: theta[r] for partition r, then its
 *              next threshold (Sec. 4.3 over P_r).  Each finite and > 0.
 *   out_idx, out_val  device, n_total entries each: the selected (index, acc)
 *              pairs of all partitions, concatenated in index order, so
 *              partition r's pairs start at k[0] + ... + k[r-1].
 *   k          host int64[world], out: each partition's count.
 *   sumsq      host double[world] out, or NULL: the squared L2 norm of each
 *              partition's new residual, squares in binary64 added in a fixed
 *              order (within (P_r - 1) * 2^-53 relative of the exact sum);
 *              sqrt of their sum is the vector's local error norm.
 * The pairs, counts, thresholds and residual equal those of world calls of
 * micro_sparsify_step (rank 0 .. world-1) bit for bit.  Needs the staged
 * schedule.  Synchronous; errors as micro_sparsify_step (MICRO_EINVAL also
 * for world above 64 or the ticket variant).
 */
MICRO_API micro_status micro_sweep_step(micro_ctx *ctx, const float *grad, float *residual,
                                        int32_t world, double density, double *theta,
                                        int32_t *out_idx, float *out_val, int64_t *k,
                                        double *sumsq);

/* Algorithm 1 (cyclic assignment of partitions; Sec. 4.1): the partition
 * number that worker `worker` of `world` searches at iteration t,
 * ((t mod n) + worker) mod n (pure host arithmetic).  Returns MICRO_EINVAL
 * for NULL output, t < 0, world < 1 or worker outside [0, world). */
MICRO_API micro_status micro_cycle(int64_t t, int32_t worker, int32_t world, int32_t *cycle);

/*
 * Algorithm 1 for worker `worker` of `world` at iteration t over the whole
 * vector (the error-feedback accumulation of every element, then selection in
 * the worker's partition of this iteration only):
 *   c = micro_cycle(t, worker, world), [s, e) = partition c (Sec. 4.1);
 *   for every j in [0, n_total): acc = grad[j] + residual[j] (one binary32
 *   addition); j in [s, e) with |acc| >= theta is selected (its pair goes to
 *   the outputs, residual[j] = +0); every other j gets residual[j] = acc.
 *   theta <- Estimate(density * (e - s), k, theta) (Sec. 4.3).
 *   grad      device, n_total fp32, read only, all of it.
 *   residual  device, n_total fp32, in/out, all of it.
 *   out_idx, out_val, k, theta, density: as micro_sparsify_step, with
 *             P = e - s of partition c.
 *   cycle     host out (may be NULL): c.
 *   sumsq     host out (may be NULL): the squared L2 norm of the whole new
 *             residual, the worker's local error of Sec. 2 squared (Eq. 1
 *             averages its square root over the workers); squares in binary64
 *             added in a fixed order, within (n_total - 1) * 2^-53 relative of
 *             the exact sum (MICRO_RULE_TOPK with t values of the k-th
 *             magnitude left out of the selection: (n_total + t) * 2^-53).  Requesting it runs the pass through the sweep's
 *             kernels (the staged schedule; MICRO_EINVAL on a TICKET context).
 * grad[0, n), residual[0, n), out_idx[0, P) and out_val[0, P) must not
 * overlap.  Synchronous; errors as micro_sparsify_step.  A partition that is
 * empty (n_total < world) still accumulates every element, with k = 0 and
 * theta unchanged.
 */
MICRO_API micro_status micro_ef_step(micro_ctx *ctx, const float *grad, float *residual,
                                     int64_t t, int32_t worker, int32_t world, double density,
                                     double *theta, int32_t *out_idx, float *out_val,
                                     int64_t *k, int32_t *cycle, double *sumsq);

/*
 * Algorithm 1, after the all-gather of the selected indices: the worker's
 * accumulated values at the union of all workers' selections (its part of
 * the all-reduce) and their reset in its local error.
 *   residual   device, n_total fp32, in/out: the local error as
 *              micro_ef_step left it (acc at every unselected element).
 *   union_idx  device int32[m]: the union, distinct indices in [0, n_total);
 *              positions [own_first, own_first + own_count) hold this
 *              worker's own selection of the same iteration, in the order
 *              micro_ef_step wrote it (own_count = its k).
 *   own_val    device fp32[own_count]: micro_ef_step's out_val.
 *   out        device fp32[m], out: out[q] = acc at union_idx[q]
 *              (own_val[q - own_first] inside the own run).
 * Every union index outside the own run gets residual = +0 (those of the own
 * run already are).  An index outside [0, n_total) touches nothing and gives
 * out[q] = NaN.  Buffers must not overlap and must be 4-byte aligned.
 * Enqueued on the context's stream: the call returns after the launch (with
 * MICRO_FLAG_TIME_KERNEL it waits and records kernel_ms).  MICRO_EINVAL for
 * m outside [0, n_total], an own run outside [0, m), NULL or overlapping
 * buffers, before any device work.
 */
MICRO_API micro_status micro_union_gather(micro_ctx *ctx, float *residual, const int32_t *union_idx,
                                          int64_t m, int64_t own_first, int64_t own_count,
                                          const float *own_val, float *out);

/*
 * Algorithm 1 and Sec. 4.4, the model update with the averaged sums:
 * x[union_idx[q]] = x[union_idx[q]] - sums[q] / world for q in [0, m) (one
 * correctly rounded binary32 division by world, one binary32 subtraction;
 * the learning rate is inside the gradients).
 *   x          device, n_total fp32 model parameters, in/out.
 *   union_idx  device int32[m], distinct; indices outside [0, n_total) are
 *              skipped.
 *   sums       device fp32[m]: the all-reduced (summed) values.
 * Enqueued like micro_union_gather.  MICRO_EINVAL for m outside
 * [0, n_total], world < 1, NULL or overlapping buffers.
 */
MICRO_API micro_status micro_sparse_update(micro_ctx *ctx, float *x, const int32_t *union_idx,
                                           const float *sums, int64_t m, int32_t world);

/* Sec. 4.1 partition bounds (pure host arithmetic, no device needed):
 * *start = floor(rank*n_total/world), *len = floor((rank+1)*n_total/world)
 * - *start.  Returns MICRO_EINVAL for world < 1, rank outside [0, world),
 * n_total < 0 or NULL outputs. */
MICRO_API micro_status micro_partition(int64_t n_total, int32_t rank, int32_t world,
                             int64_t *start, int64_t *len);

/* Sec. 4.3 threshold update as the step applies it (pure host arithmetic):
 * *theta <- Estimate(density * part_len, k, *theta) under cfg (NULL =
 * defaults).  part_len == 0 leaves *theta unchanged.  Returns MICRO_EINVAL
 * for NULL theta, part_len < 0, k outside [0, part_len] or density outside
 * (0, 1]. */
MICRO_API micro_status micro_estimate_threshold(const micro_config *cfg, double density,
                                      int64_t part_len, int64_t k,
                                      double *theta);

/* The fp32 threshold the device compares with: the smallest binary32 value
 * >= theta (+inf when theta exceeds FLT_MAX).  For every binary32 x,
 * x >= *theta_f  <=>  (double)x >= theta, so the device's binary32 compare
 * selects exactly what the binary64 definition selects.  Returns
 * MICRO_EINVAL for NULL output or theta not finite and > 0. */
MICRO_API micro_status micro_threshold_f32(double theta, float *theta_f);

/* Copies the statistics of the last step on ctx (zeroes and kernel_ms = -1
 * before the first step or without MICRO_FLAG_TIME_KERNEL).  Returns
 * MICRO_EINVAL for NULL arguments. */
MICRO_API micro_status micro_sparsify_last_stats(const micro_ctx *ctx, micro_step_stats *stats);

/* Message of the last failure on ctx (or of the last failed init when ctx is
 * NULL); never NULL. */
MICRO_API const char *micro_last_error(const micro_ctx *ctx);

/* Static name of a status code. */
MICRO_API const char *micro_status_string(micro_status status);

/* Releases the context's scratch; NULL is a no-op.  Waits for the context's
 * stream first. */
MICRO_API void micro_sparsify_free(micro_ctx *ctx);

/* ------------------------------------------------------------------------
 * Around the step on a language model: the global norm and clipping of a
 * model's gradients into the flat vector that the step reads, the lookup of
 * token rows with its gradient, the softmax cross entropy over the token table
 * with its gradients, the draw of tokens from logits, and matrices in 4 bits.
 *
 * Every call below is enqueued on its handle's stream and returns after the
 * launches; device inputs must be ready on that stream and stay allocated
 * until it has run.  Messages of a refusal come from micro_last_error(NULL) on
 * the calling thread; a refusal (MICRO_EINVAL, MICRO_ECAPACITY, MICRO_ERANGE)
 * comes before any device work, with nothing modified.  One handle must not be
 * used from two threads at once.  Calls share their handle's scratch, those that a
 * graph has captured too: they must not run at once, and the handle must be freed
 * after the graph's last replay.  Results are the same on every run.
 * ------------------------------------------------------------------------ */

/* Types of the tensors' values. */
#define MICRO_TYPE_F32 0  /* IEEE binary32 */
#define MICRO_TYPE_F16 1  /* IEEE binary16 */
#define MICRO_TYPE_BF16 2 /* bfloat16      */

/*
 * A set of gradient tensors, in the order of the flat vector: tensor i holds
 * sizes[i] contiguous values of types[i] at tensors[i] (device, aligned to its
 * type; a tensor of no values may be NULL).  The set keeps the addresses: the
 * tensors stay where they are until micro_grads_free.  No two may share
 * memory.  `tensors`, `sizes` and `types` are host arrays of `count` entries,
 * read during the call, which waits for its upload.  Device scratch: 16 KB and
 * 24 bytes per 4,096 to 32,768 values.
 */
typedef struct micro_grads micro_grads; /* opaque, owned by the library */
MICRO_API micro_status micro_grads_init(micro_grads **grads, int32_t count, void *const *tensors,
                                        const int64_t *sizes, const int32_t *types, void *hip_stream);

/*
 * The global L2 norm: *sumsq = the sum of the squares of all values (device
 * double), *norm = its square root (device float); either may be NULL.
 * Squares and sums in binary64, in an order that only the sizes determine.
 * Workers that hold parts of one model add their sumsq before clipping.
 */
MICRO_API micro_status micro_grads_norm(micro_grads *grads, double *sumsq, float *norm);

/*
 * Every value times c = min(1, max_norm / (norm + 1e-6)), in place: c in
 * binary64, rounded to binary32 once; the product in binary32, rounded to the
 * tensor's type once.  c == 1 writes nothing.  A norm of +inf makes c 0, a
 * NaN makes it NaN (as the formula says).
 *   max_norm  > 0; +inf does not clip.
 *   sumsq     device double: the squared norm to clip by (of all workers);
 *             NULL: this set's own, computed first.
 *   norm      device float out: sqrt(sumsq); may be NULL.
 */
MICRO_API micro_status micro_grads_clip(micro_grads *grads, double max_norm, const double *sumsq, float *norm);

/*
 * The same values in binary32 into `flat` (device, as many floats as the set
 * has values, sharing no memory with the set), tensor after tensor; the
 * tensors stay as they are.  With max_norm = +inf and norm == NULL the values
 * are only converted, in one pass.
 */
MICRO_API micro_status micro_grads_flatten(micro_grads *grads, double max_norm, const double *sumsq, float *flat,
                                           float *norm);

/* Releases the set's scratch after waiting for its stream; NULL is a no-op.
 * The tensors are the caller's. */
MICRO_API void micro_grads_free(micro_grads *grads);

/*
 * A token table: `vocab` rows of `dim` values of one type, with the lookup of
 * rows, the loss over the table and the gradients of both.  Row arguments are
 * device addresses with a row stride in values (>= dim; the values of a row
 * are adjacent, the address aligned to the type); tokens' ids and targets are
 * int32 or int64 (MICRO_IDS_*), one after the other, aligned to their size.
 * No output may share a value with another argument (columns of one buffer, of
 * the same row stride, may be different arguments; rows of different strides may
 * not lie among each other): MICRO_EINVAL.
 */
#define MICRO_IDS_I32 0
#define MICRO_IDS_I64 1

typedef struct micro_table micro_table; /* opaque, owned by the library */

typedef struct micro_table_config {
    int64_t padding_id;  /* an id whose row gets no gradient from lookups; -1: none      (-1)   */
    int64_t ignored;     /* the target of a token that does not count                    (-100) */
    int64_t score_bytes; /* scratch for one token block's scores at most (at least one
                            block of 256 tokens is held)                         (2^31) */
} micro_table_config;

/* Fills *cfg with the defaults listed above. */
MICRO_API void micro_table_config_default(micro_table_config *cfg);

/*
 * A handle for a table of vocab x dim values of `type` and calls of up to
 * max_tokens tokens, enqueuing on hip_stream; cfg NULL: the defaults.  Holds
 * no scratch yet: the first call of each kind allocates what its kind needs
 * (of max_tokens, whatever the call's own: a lookup nothing; its gradient 16
 * bytes and dim/2 bytes a token; the loss 32 MB, a padded copy of the hidden
 * rows, 8 bytes a block's token for every 128 rows of the table (at least what
 * 768 tokens take), and a padded copy of the table where it cannot be read in
 * place: binary32, a dim that is no multiple of 64, or rows that are not aligned
 * to 16 bytes; its gradients the block's scores, 128 MB, and where max_tokens
 * exceeds a block 4 bytes for every value of the table, both sides rounded up to
 * multiples of 256).  A block is as many tokens as score_bytes holds at 2 bytes
 * a score (binary32: 10), in multiples of 256.  A call that is captured into a
 * graph must have its scratch: make one like it before.
 * MICRO_ERANGE for vocab above 2^31 - 2, dim above 65536 or max_tokens above
 * 2^22; MICRO_EINVAL for vocab < 1, dim < 1, max_tokens < 0 or an unknown
 * type.
 */
MICRO_API micro_status micro_table_init(micro_table **table, int64_t vocab, int32_t dim, int64_t max_tokens,
                                        int32_t type, void *hip_stream, const micro_table_config *cfg);

/*
 * out[t] = scale * weight[ids[t]] for t in [0, tokens): one binary32 product,
 * rounded to the type once.  An id outside [0, vocab) gives a row of NaN.
 * MICRO_ECAPACITY for tokens above max_tokens, here and below.
 */
MICRO_API micro_status micro_table_lookup(micro_table *table, const void *weight, int64_t weight_stride,
                                          const void *ids, int32_t ids_type, int64_t tokens, double scale,
                                          void *out, int64_t out_stride);

/*
 * The lookup's gradient: dweight[v] = scale * the sum of grad[t] over the
 * tokens t with ids[t] == v, in binary32 and an order that the ids alone
 * determine (ascending t, for more than 16 to 31 tokens in runs of 16 whose sums
 * are added), rounded to the type once.
 * accumulate != 0 adds that to dweight[v] before rounding and leaves rows
 * without a token untouched; else every row is written.  Tokens whose id is
 * padding_id or outside [0, vocab) have no part.
 */
MICRO_API micro_status micro_table_lookup_grad(micro_table *table, const void *grad, int64_t grad_stride,
                                               const void *ids, int32_t ids_type, int64_t tokens, double scale,
                                               int32_t accumulate, void *dweight, int64_t dweight_stride);

/*
 * The softmax cross entropy of hidden rows against the table: with the logits
 * l[t][v] = hidden[t] . weight[v], losses[t] = log(sum over v of exp(l[t][v]))
 * - l[t][targets[t]], and *loss their sum (mean == 0) or mean over the counted
 * tokens; 0 when none counts.  Products of the type's values are accumulated
 * in binary32; the logits are not stored.
 *   targets  int32 or int64; `ignored` marks a token that does not count (its
 *            losses[t] is 0).  Any other target outside [0, vocab) does not
 *            count either and makes losses[t] and *loss NaN.
 *   losses   device float[tokens];  loss  device float.
 * MICRO_ERANGE for a vocab above 2^22.
 */
MICRO_API micro_status micro_table_loss(micro_table *table, const void *hidden, int64_t hidden_stride,
                                        const void *weight, int64_t weight_stride, const void *targets,
                                        int32_t targets_type, int64_t tokens, int32_t mean, float *losses,
                                        float *loss);

/*
 * The loss with its gradients, scaled by `scale` (and by 1 / counted tokens
 * with mean != 0):
 *   dhidden[t] = factor * sum over v of (p[t][v] - [v == targets[t]]) weight[v]
 *   dweight[v] = factor * sum over t of (p[t][v] - [v == targets[t]]) hidden[t]
 * with p the softmax of the logits.  A token that does not count has a zero
 * row in dhidden and no part in dweight.  accumulate != 0 adds to dweight.
 * Both are of the table's type, rounded once; between the products p - [..] is
 * rounded to the table's type once (binary32: to 24 bits; binary16 keeps it times
 * 2^14, so that it loses bits below 2^-28 and is 0 below 2^-39), sums in
 * binary32.  In dhidden the label's p - 1 counts unrounded.  In dweight of 16-bit
 * types that rounding adds to the error what the output's own does not: where
 * more matters, binary32 has it.
 */
MICRO_API micro_status micro_table_loss_grad(micro_table *table, const void *hidden, int64_t hidden_stride,
                                             const void *weight, int64_t weight_stride, const void *targets,
                                             int32_t targets_type, int64_t tokens, int32_t mean, double scale,
                                             int32_t accumulate, float *losses, float *loss, void *dhidden,
                                             int64_t dhidden_stride, void *dweight, int64_t dweight_stride);

/*
 * Draws a token for each row of logits over the table's vocabulary.  With m the
 * row's largest logit and T its temperature a token's weight is w = exp((l - m) /
 * T); tokens are ordered by logit, the largest first, equal ones by index.
 *   top_k   the first top_k tokens of that order are kept (<= 0: all);
 *   top_p   of those the shortest prefix whose weights reach top_p of theirs (at
 *           least one token; >= 1: all);
 *   min_p   of those the ones with w >= min_p.
 * ids[t] is the first token, by index, at which the running sum of the kept
 * weights exceeds uniforms[t] times their sum, logprobs[t] the logarithm of its
 * share.  T == 0 takes the first largest logit.  Logits of -inf or NaN have no
 * part, and equal +inf ones share the row; where none is left ids[t] is -1 and
 * logprobs[t] NaN.  Weights are whole multiples of 2^-f in 64 bits, where the
 * vocabulary has at most 2^(62 - f) tokens and f is at most 50, and their sums are
 * exact: a token of less than that share of the largest is never drawn.
 *   logits    device, `rows` rows of `vocab` values of logits_type, any row stride
 *             >= vocab.
 *   uniforms  device float[rows] in [0, 1); below (or NaN) counts as 0, above as
 *             the largest below 1.
 *   sampling  host: the settings of all rows, or for any of the four a device
 *             array of one value a row in its place (float, top_k int32), where a
 *             temperature that is not above 0 counts as 0 and a NaN top_p or min_p
 *             as one that keeps all.
 *   ids       device, of ids_type;  logprobs  device float[rows]; may be NULL.
 * MICRO_ERANGE for a vocab above 2^22, MICRO_EINVAL for a setting out of range
 * (temperature < 0 or NaN, top_p outside (0, 1], min_p outside [0, 1]).
 */
typedef struct micro_sampling {
    double temperature, top_p, min_p;
    int64_t top_k;
    const float *temperatures, *top_ps, *min_ps; /* device, one a row; NULL: the value above */
    const int32_t *top_ks;
} micro_sampling;

MICRO_API micro_status micro_table_sample(micro_table *table, const void *logits, int32_t logits_type,
                                          int64_t logits_stride, int64_t rows, const float *uniforms,
                                          const micro_sampling *sampling, void *ids, int32_t ids_type,
                                          float *logprobs);

/* Releases the handle's scratch after waiting for its stream; NULL is a no-op. */
MICRO_API void micro_table_free(micro_table *table);

/*
 * Microscaled 4-bit matrices (OCP MX v1.0, MXFP4) and their products.  A matrix
 * of rows x cols values is held in blocks of 32 values along a row: a scale 2^e,
 * one byte e + 127, and a 4-bit code a value, sign and one of 0, 0.5, 1, 1.5, 2,
 * 3, 4, 6.  With a the block's largest magnitude e = floor(log2 a) - 2, at least
 * -127, and the code is that of value / 2^e, to nearest, ties to the even code,
 * at most 6.  A block that holds a NaN or an infinity is NaN (byte 255, codes 0).
 * A block of zeros has byte 0.
 * A row is divided into groups of 128 values, the last one filled up with zeros.
 *   codes   64 bytes for each group and row, the rows of a group one after the
 *           other: value c of row r in byte ((c / 128) * rows + r) * 64 + c % 128 /
 *           2, an even c in the lower half.  Aligned to 16 bytes.
 *   scales  the byte of block b of row r at ((b / 4) * rows + r) * 4 + b % 4.
 *           Aligned to 4 bytes.
 * Sides are at most 2^24 (MICRO_ERANGE).
 */
typedef struct micro_mx4_matrix {
    void *codes, *scales; /* device */
    int64_t rows, cols;
} micro_mx4_matrix;

/* Bytes of a matrix's codes and scales (host arithmetic).  MICRO_EINVAL for a
 * negative side or NULL outputs, MICRO_ERANGE for one above 2^24. */
MICRO_API micro_status micro_mx4_bytes(int64_t rows, int64_t cols, int64_t *codes, int64_t *scales);

/* A handle for calls on hip_stream and the current device, with scratch of 256 KB for
 * each compute unit (64 MB), which its products share: two of one handle, captured into
 * graphs too, must not run at once. */
typedef struct micro_mx4 micro_mx4; /* opaque, owned by the library */
MICRO_API micro_status micro_mx4_init(micro_mx4 **mx, void *hip_stream);

/*
 * Packs `rows` rows of `cols` values of `type` (row stride in values, >= cols)
 * into *packed (rows x cols), *turned (cols x rows, the transposed matrix, whose
 * blocks run along the rows of x), or both from one read; either may be NULL.
 * MICRO_EINVAL for sides that do not fit x or an output that shares memory.
 */
MICRO_API micro_status micro_mx4_pack(micro_mx4 *mx, const void *x, int32_t type, int64_t stride, int64_t rows,
                                      int64_t cols, const micro_mx4_matrix *packed, const micro_mx4_matrix *turned);

/* The values that a packed matrix stands for, rounded to `type` once (binary32 and
 * bfloat16 hold them exactly). */
MICRO_API micro_status micro_mx4_unpack(micro_mx4 *mx, const micro_mx4_matrix *packed, void *out, int32_t type,
                                        int64_t stride);

/*
 * out[i][j] = sum over k of a[i][k] b[j][k] (a: m x k, b: n x k, out: m rows of n
 * values of `type`): products of values are exact, sums in binary32 and an order
 * that only the sizes determine, rounded to the type once.  accumulate != 0 adds to
 * out before rounding.  A value of 0 times a NaN block is NaN.  With cols == 0 the
 * sum is 0.
 */
MICRO_API micro_status micro_mx4_product(micro_mx4 *mx, const micro_mx4_matrix *a, const micro_mx4_matrix *b,
                                         int32_t accumulate, void *out, int32_t type, int64_t stride);

/*
 * The product with an a that is packed on the way: x has a->rows rows of a->cols
 * values of x_type; *a is scratch for their packed form, whose contents are
 * undefined afterwards.
 */
MICRO_API micro_status micro_mx4_linear(micro_mx4 *mx, const void *x, int32_t x_type, int64_t x_stride,
                                        const micro_mx4_matrix *a, const micro_mx4_matrix *b, int32_t accumulate,
                                        void *out, int32_t type, int64_t stride);

/* Releases the handle's scratch after waiting for its stream; NULL is a no-op. */
MICRO_API void micro_mx4_free(micro_mx4 *mx);

#ifdef __cplusplus
}
#endif

#endif /* MICRO_SPARSIFY_H */
