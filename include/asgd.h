/*
 * asgd.h — C ABI of the MI355X (gfx950) ASGD mini-batch K-Means library.
 *
 * The library runs W independent SGD workers on one GPU.  Every worker streams its
 * own shard of fp32 samples through mini-batch K-Means steps (nearest prototype,
 * per-centroid gradient, update) and every E steps sends its state to one other
 * worker, whose next step merges it under the paper's Parzen-window rule.
 *
 * Conventions
 *   - every function returns ASGD_OK (0) or a negative ASGD_E* code; nothing throws
 *     or aborts across this boundary; asgd_strerror() names a code;
 *   - "device pointer" = HIP device memory of the current device, "host pointer" =
 *     ordinary host memory; the library never frees caller memory;
 *   - a context belongs to the device that was current in asgd_create(); calls on
 *     one context must not overlap in time (one context per host thread);
 *   - there is no CPU fallback: without a usable HIP device the calls fail.
 *
 * Notation: k centroids, d dimensions, W workers, b mini-batch size, eps step size,
 * E exchange interval, H = floor(N / W) shard length, S = floor(H / b) steps per
 * epoch, t = step counter (the same for all workers, it continues across epochs and
 * across calls), round r = floor(t / E).
 */
#ifndef ASGD_H
#define ASGD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct asgd_ctx asgd_ctx; /* opaque: worker states, exchange buffers, counters */

enum {
    ASGD_OK = 0,
    ASGD_EINVAL = -1,   /* bad argument (null pointer, size out of range, unknown option) */
    ASGD_ENOMEM = -2,   /* device or host allocation failed */
    ASGD_ESTATE = -3,   /* call out of order (e.g. run before load_shards) */
    ASGD_EHIP = -4,     /* a HIP runtime call failed; asgd_last_hip_error() has its code */
    ASGD_ESYNC = -5     /* a bounded wait inside a kernel expired (runs that are one launch of workgroups
                           which wait for each other's messages; all the waits of a workgroup draw on one
                           budget of polls that grows with the rounds of the launch, or, in the kernels
                           with fp16-split operands, every wait has a budget that covers the longest a
                           round can take, and after one expired wait there are no more; a launch covers
                           at most 1024 rounds, so it ends within a second plus a few milliseconds per
                           round of waiting, or plus a few such rounds).  The run is lost: the step counter is not advanced and later runs
                           fail with ASGD_ESTATE until asgd_load_shards(), or asgd_set_state() followed by
                           asgd_set_step(), have put the context back on a known footing. */
};

/* Keys of asgd_set_option().  Values are passed as double and rounded to integers
   where an integer is meant. */
enum {
    ASGD_OPT_EXCHANGE_EVERY = 1, /* E >= 0; 0 = never send: silent mode = SimuParallelSGD with
                                    mini-batches (Sec. 4, first paragraph; Sec. 5.4 "silent");
                                    E = 1 is Alg. 5 as printed.  Default 0. */
    ASGD_OPT_SEED = 2,           /* seed of the peer schedule (integer < 2^53).  Default 1. */
    ASGD_OPT_MODE = 3,           /* ASGD_MODE_*.  Default deterministic. */
    ASGD_OPT_PARZEN = 4,         /* 1 = gate merges with Eq. 4 (default), 0 = delta = 1 (Eq. 2) */
    ASGD_OPT_LR_MODE = 5,        /* ASGD_LR_*.  Default constant. */
    ASGD_OPT_DROP_RATE = 6,      /* test hook: probability in [0,1] that a message is lost on
                                    the way (Sec. 4.4: a lost message is harmless).  Default 0. */
    ASGD_OPT_KERNEL = 7,         /* ASGD_KERNEL_*: which implementation runs the steps.
                                    Default auto.  All give the same results to rounding.  The kernels keep
                                    messages in flight in different formats; when the kernel changes between
                                    two runs the library carries them over (see asgd_get_exchange). */
    ASGD_OPT_TUNE = 8,           /* launch-shape variant of the chosen kernel (0 = default; shape-agnostic kernel: bits 1 one
                                    workgroup per worker, 2 matrix cores, whatever the size, 4 several launches
                                    per step also where one launch would do); for
                                    performance experiments: the variants compute the same thing and may
                                    differ in the rounding of their sums */
    ASGD_OPT_COOPERATIVE = 9,    /* 1 (default): a run that needs all its workgroups resident at the
                                    same time is started with a cooperative launch, which refuses
                                    grids that cannot be; 0: plain launch of the same grid (for tools
                                    that cannot follow cooperative launches).  The in-kernel waits are
                                    bounded either way. */
    ASGD_OPT_BUFFERS = 10,       /* N of Eq. 3 / Eq. 6: external buffers per worker, 1 (default) .. 4.  A
                                    worker then sends every message to N different workers (copy n goes
                                    into the recipient's buffer n; deterministic schedule: a cyclic shift
                                    per round and copy, so every worker receives N messages per round from
                                    N different senders) and merges, of the buffers that hold a message,
                                    those that pass Eq. 4 on their own: w - (sum of them + w)/(their
                                    number + 1) is added to the step.  With ASGD_OPT_PARZEN = 0 every
                                    non-empty buffer takes part (Eq. 3).  Needs N < W at run time
                                    (ASGD_EINVAL otherwise); may only be set before the first step
                                    (ASGD_ESTATE after); reallocates the exchange buffers (2 * N * W states).
                                    Available in all three kernels. */
    ASGD_OPT_PARTS = 11          /* partial messages (Sec. 4.4, partitioned along the cluster centres):
                                    P in 1 .. k, default 1 = whole states.  With P > 1 part q is the set of
                                    centroid rows c with c mod P = q, and copy n of the message of round r
                                    to worker p carries part (r + p + n) mod P only (1/P of the bytes); the
                                    recipient treats every transmitted row as a unit of its own: empty iff
                                    all zero, tested by Eq. 4 over that row, merged by Eq. 6 with the other
                                    buffers' accepted copies of the same row; rows that did not travel take
                                    the plain step.  "received" then counts buffers with a non-empty row,
                                    "accepted" buffers with an accepted row.  May only be set before the
                                    first step (ASGD_ESTATE after).  Available in all three kernels; in the
                                    matrix-core kernel only while W*k*d <= ASGD_MFMA_PARTS_MAX_STATE (the sizes
                                    its tests cover: the only batch of larger runs of that combination ended in
                                    a device fault that was never explained).  Above that the automatic choice
                                    takes the shape-agnostic kernel and an explicit ASGD_KERNEL_MFMA fails with
                                    ASGD_EINVAL. */
};
enum { ASGD_MFMA_PARTS_MAX_STATE = 1 << 18 };
enum {
    ASGD_OPT_WAIT_POLLS = 12,       /* test hook: polls a workgroup may spend, in total, on the waits of one launch
                                       (0 = the library's default of some 10^5, i.e. a fraction of a second) */
    ASGD_OPT_DROP_UNANNOUNCED = 13, /* test hook: 1 = the recipient does not know which messages ASGD_OPT_DROP_RATE
                                       loses, so a run that is one launch waits for them until its poll budget is
                                       gone and then returns ASGD_ESYNC (every kernel still ends normally); 0 (default):
                                       a lost message is skipped at once */
    ASGD_OPT_REFUSE_ONE_LAUNCH = 14 /* test hook: 1 = runs that would be one launch of workgroups which wait for each other
                                       behave as if the runtime refused it; 2 (split kernels): as if one of its
                                       workgroups found no place on the device.  Either way the run is done with
                                       more launches and no waits inside them.  Default 0. */
};
enum { ASGD_MODE_DETERMINISTIC = 0, ASGD_MODE_FREE_RUNNING = 1 };
enum { ASGD_LR_CONST = 0, ASGD_LR_INV_COUNT = 1 };
enum { ASGD_KERNEL_AUTO = 0, ASGD_KERNEL_GENERIC = 1, ASGD_KERNEL_SMALL = 2, ASGD_KERNEL_MFMA = 3 };
/* Two of the kernels stand for a pair each, and asgd_last_run_form() says which of the pair ran: the fp32 kernel, or the one
   with fp16-split operands, as one launch or as several launches per step (phases). */
/* (SPLIT_LAUNCH also where that one launch was refused or the call is short, and one launch per round took its place.) */
enum { ASGD_FORM_NONE = 0, ASGD_FORM_FP32 = 1, ASGD_FORM_SPLIT_LAUNCH = 2, ASGD_FORM_SPLIT_PHASES = 3 };

typedef struct asgd_stats {
    int64_t steps;            /* value of the step counter t */
    int64_t samples;          /* samples processed so far = t * W * b */
    int64_t sent;             /* messages written, summed over workers (Alg. 5, send) */
    int64_t received;         /* messages found in a buffer and tested with Eq. 4 */
    int64_t accepted;         /* of those, messages with delta = 1 ("good" messages, Sec. 5.4) */
    int64_t parzen_near_ties; /* tested messages with |lhs - rhs| / rhs < 1e-6 in Eq. 4 */
    int64_t exact_rechecks;   /* samples whose two best fp32 scores were too close to call and
                                 whose assignment was therefore recomputed in fp64 */
    double last_run_ms;       /* device time of the last asgd_run_* call (HIP events) */
    int32_t kernel;           /* ASGD_KERNEL_* that the last run used */
    int32_t launches;         /* kernel launches of the last run */
} asgd_stats;

/*
 * Create a context for the problem of Sec. 5.1 (k prototypes for points in R^d) run by
 * Alg. 5 with W workers ("nodes"), mini-batch size b and step size eps = lr.
 * Requires k, d, W, b >= 1 and lr > 0 (Alg. 5 "Require"; W = 1 is allowed and equals
 * Alg. 4).  Allocates W*k*d floats of state, the exchange buffers and the operands of one state (Eq. 8; 4 bytes per
 * padded element, rows of 8 to 128 columns) on the current device.  More is allocated by the first call that needs it and kept until asgd_destroy():
 * 8 KB per column at the first asgd_load_shards() (d <= 8192; where the streaming kernel runs: at the first run of another; that
 * kernel takes 4 bytes per worker and mini-batch once it has met large elements, see asgd_load_shards()), and the operands and sums of the
 * kernels with fp16-split operands at a run, several times W*k*d floats and 32 GiB at most
 * (a kernel that needs none takes over where there is no room).  *out is set only on success and must be released with asgd_destroy().
 */
int asgd_create(asgd_ctx **out, int k, int d, int W, int b, float lr);

/* Set one option (see the key list).  Allowed at any time between runs. */
int asgd_set_option(asgd_ctx *ctx, int key, double value);

/*
 * Hand the samples to the workers (Sec. 4 "Initialization": the data is split into
 * packages, one per worker; Alg. 5 lines 1-2).
 *   x_dev       device pointer, N x d fp32 row-major, at least 8-byte aligned.  BORROWED:
 *               the caller keeps it alive and unchanged until asgd_destroy() or the
 *               next asgd_load_shards().
 *   N           number of rows; worker i owns rows [i*H, (i+1)*H), the last N mod W rows
 *               are not used by the optimisation.  Requires H >= max(k, b).
 *   hip_stream  a hipStream_t (0 = default stream) on which this and all later calls of
 *               the context enqueue their work.
 * Effects: every worker's state is set to the first k rows of its own shard, exchange
 * buffers, counters and the step counter are cleared.  Synchronises the stream.
 * Column maxima are formed over all rows, where the streaming kernel runs over a part of them: it looks out for larger elements
 * in the first epoch, forms the steps that hold one a second time, and knows them from then on.
 */
int asgd_load_shards(asgd_ctx *ctx, const float *x_dev, int64_t N, void *hip_stream);

/*
 * Overwrite worker states from host memory: w_host holds k*d floats (worker >= 0 sets
 * that worker, worker = -1 gives the same w0 to all workers, Sec. 4 "Initialization") or
 * W*k*d floats (worker = -2 sets each worker from its own block).  Needed to continue an
 * earlier run (Sec. 4: w0 may be the result of a run that was stopped early).
 */
int asgd_set_state(asgd_ctx *ctx, int worker, const float *w_host);

/* Set the step counter t (>= 0) when continuing an earlier run.  Exchange buffers are
   emptied: at a multiple of E the messages of the round just finished are in flight
   (Alg. 5: sent at the end of one step, looked at in the merge of the next), so a run resumed
   there equals the uninterrupted one only if asgd_set_exchange() hands them over too. */
int asgd_set_step(asgd_ctx *ctx, int64_t t);

/*
 * The messages in flight (Alg. 5 lines 5 and 9, Eq. 3 / Eq. 6: N external buffers per
 * worker; Sec. 4 "Initialization": a run may start from the result of an earlier one), in
 * a layout that does not depend on the kernel that ran:
 *   values_host  float [buffers][W][k][d], host memory: the rows waiting in buffer n of
 *                worker i; rows that a partial message (Sec. 4.4) does not carry, and
 *                empty buffers, are zeros.
 *   rounds_host  int32 [buffers][W], host memory: the round the message was sent in,
 *                -1 = nothing waiting.
 * Deterministic mode: messages wait exactly when t is a positive multiple of E, and all
 * carry round t/E - 1; anywhere else every entry is -1.  Free-running mode: whatever the
 * buffers hold at this moment (the newest message of a buffer; its rows only).
 * asgd_get_exchange() copies them out (sizes in bytes are checked: ASGD_EINVAL if too
 * small).  asgd_set_exchange() is called after asgd_set_state() and asgd_set_step(t) of a
 * continued run; the library keeps a host copy until the next run, which writes it into
 * the buffers in its kernel's format.  A deterministic run continued this way at a merge
 * point is bit-identical to the uninterrupted run.  ASGD_EINVAL: a round that cannot wait
 * at step t (deterministic mode: anything but -1 and t/E - 1 at a merge point).
 * The same conversion happens by itself when ASGD_OPT_KERNEL changes between two runs.
 */
int asgd_get_exchange(asgd_ctx *ctx, float *values_host, size_t values_bytes, int32_t *rounds_host, size_t rounds_bytes);
int asgd_set_exchange(asgd_ctx *ctx, const float *values_host, const int32_t *rounds_host);

/*
 * Run `epochs` passes over every shard: epochs * S steps of Alg. 5 lines 6-10 per
 * worker, mini-batch s of an epoch being rows [s*b, (s+1)*b) of the shard (the tail
 * H mod b is skipped).  A step = assignment s_i(w) (Sec. 5.1), gradient (Eq. 9 with
 * m' = b), merge of a buffered external state when t > 0 and t mod E == 0 (Eq. 4,
 * Eq. 7), update w <- w - eps * step (Alg. 5, update) and, when (t+1) mod E == 0, the
 * send of the new state to one other worker (Alg. 5, send).  Returns after the work
 * has finished on the device.  The result does not depend on how a run is cut into
 * calls (deterministic mode: bit for bit), the time does: with the streaming kernel, and
 * with the others where the workers fill the device and exchange every fourth step or less
 * often (or at any step, where a worker's state and two mini-batches fit a compute unit), a call of two communication rounds or more is ONE kernel launch for every 1024 rounds
 * it covers (the streaming kernel: a call of more than two epochs that begins with the first after loading or after asgd_set_step(), one more),
 * and the start and the tail of a launch are then paid once per launch, not once per epoch (asgd_stats.launches); else a round, or every phase of a step, is a launch over all
 * workers.
 */
int asgd_run_epochs(asgd_ctx *ctx, int epochs);

/* Same, for an arbitrary number of steps (continues inside an epoch). */
int asgd_run_steps(asgd_ctx *ctx, int64_t steps);

/*
 * Test aid: record the assignment s_i of every sample processed by later runs.
 *   assign_dev  device pointer to capacity int32 values, BORROWED, or NULL to stop.
 * A run of n steps writes n*W*b values, step-major, then worker, then position in the
 * mini-batch, and fails with ASGD_EINVAL if that exceeds `capacity`.
 */
int asgd_set_assign_dump(asgd_ctx *ctx, int32_t *assign_dev, size_t capacity);

/*
 * Copy states to host memory.  worker >= 0: that worker's k*d floats (worker 0 is the
 * result Alg. 5, return returns); worker = -1: all W states, W*k*d floats.
 * out_bytes must be at least the size copied.
 */
int asgd_get_state(asgd_ctx *ctx, int worker, float *out_host, size_t out_bytes);

/*
 * The mean of the W worker states (the alternative final aggregation of Sec. 4.3),
 * k*d floats, computed on the device in worker order.
 */
int asgd_get_mean_state(asgd_ctx *ctx, float *out_host, size_t out_bytes);

/*
 * Quantization error of Eq. 8, E(w) = sum_i 1/2 * min_k |x_i - w_k|^2, over all N loaded
 * rows for the state of `worker` (>= 0) or the mean state (worker = -1).  fp32: the nearest
 * centroid of a sample is found from expanded-form scores x.w_c - |w_c|^2/2 (any shape but the
 * smallest ones: on the matrix cores; where their operands are fp16 parts, candidates within the
 * rounding error of the scores are decided by their distances), the distance to it is then formed
 * directly as sum_j (x_j - w_cj)^2, so clusters far from the origin lose nothing to cancellation; the sum
 * over the samples is fp64 in a fixed order.  *out is host memory.
 */
int asgd_quant_error(asgd_ctx *ctx, int worker, double *out);

/*
 * Eq. 8 without a context and without any allocation, for callers that cannot call hipMalloc: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same kernels and the same result as
 * asgd_quant_error(); the partial sums of the reduction and the operands of the state live in a static device array of the library
 * (4.3 MB on every GPU the library runs on, held until the process ends) instead of a context's scratch.
 *   x_dev    device pointer, N x d fp32 row-major, at least 8-byte aligned (BORROWED for the duration of the work)
 *   w_dev    device pointer, k x d fp32 state
 *   out_dev  device pointer to ONE double, 8-byte aligned: receives E(w) when the work enqueued on `hip_stream`
 *            (a hipStream_t, 0 = default stream) has finished; the call itself does not wait
 * Limits: N <= 2^40, d <= 65536, k*d <= 2^24; anything larger, a null pointer or a misaligned one gives ASGD_EINVAL
 * and nothing is enqueued.  Calls neither hipMalloc/hipFree nor any routine that allocates (the first call on a
 * device looks up the address of the static array, nothing more).  All calls on one GPU share that array: calls that
 * overlap in time on one GPU (different streams or threads) race on it; calls on one stream are ordered and safe.
 * The array keeps the last call's numbers; every call overwrites all it reads, so nothing is cleared.
 */
int asgd_quant_error_noalloc(const float *x_dev, int64_t N, int k, int d, const float *w_dev, double *out_dev,
                             void *hip_stream);

/* ---- Routed experts --------------------------------------------------------------------------------------------------
 *
 * Beyond the one nearest centroid: a row of scores against E directions (a router; learned centroids serve as one) is
 * taken to the best k of them with weights, and every direction has a product ("expert") that only its own rows pass
 * through.  The products run in 8-bit floating point (e4m3) with a scale for each block of 128 along the contraction.
 *
 * These calls have no context.  Every pointer is a device pointer of the current device unless it is called a host
 * pointer; the structures themselves are host memory and read before the call returns.  The work is enqueued on
 * `hip_stream` (a hipStream_t, 0 = default stream) and not waited for; nothing is allocated, nothing is kept from one
 * call for another, and calls on different streams are independent as long as their buffers are.  Memory that a call
 * writes must not overlap what it reads.  Arguments that do not fit give ASGD_EINVAL and nothing is enqueued; a refused
 * launch gives ASGD_EHIP.  Results do not depend on timing: the same call on the same inputs gives the same bits.
 */
enum { ASGD_TYPE_F32 = 0, ASGD_TYPE_BF16 = 1, ASGD_TYPE_F16 = 2 };
enum { ASGD_SCORE_SOFTMAX = 0, ASGD_SCORE_SIGMOID = 1 };
enum { ASGD_GROUP_BEST = 0, ASGD_GROUP_BEST_TWO = 1 };
enum { ASGD_ROUTE_MAX_EXPERTS = 1024, ASGD_ROUTE_MAX_CHOSEN = 64, ASGD_ROUTE_MAX_GROUPS = 64 };

typedef struct asgd_route_rule {
    int32_t k;           /* experts per row, 1 .. min(ASGD_ROUTE_MAX_CHOSEN, experts in the kept groups) */
    int32_t score;       /* ASGD_SCORE_* */
    int32_t groups;      /* 1 .. ASGD_ROUTE_MAX_GROUPS, a divisor of E: groups of E / groups consecutive experts */
    int32_t kept;        /* groups that stay, 1 .. groups */
    int32_t group_by;    /* a group is judged by its best key, or by the sum of its two best (ASGD_GROUP_*; two: E / groups >= 2) */
    int32_t renormalize; /* 1: a row's weights add up to `scale`; 0: they are the scores times `scale` */
    float scale;
} asgd_route_rule;

/*
 * Best k of E experts for each of T rows.  logits: T x E of `type` (ASGD_TYPE_*), rows `stride` elements apart; bias: E
 * floats or NULL.  An expert is out for a row where its logit or its bias is -infinity.  With l the logits of the
 * experts that are in: score s = softmax(l) or 1 / (1 + exp(-l)); key = l without a bias, s + bias with one.  The groups
 * with the best keys stay (ASGD_GROUP_BEST_TWO: sums of two keys, without a bias of two scores; a group with one expert
 * left ranks last), of their experts those with the k largest keys are chosen, largest first, ties lowest index first.
 *   ids      int32 T x k: chosen experts, -1 where none is left
 *   weights  float T x k: scale * s, or with renormalize scale * s / (sum of the chosen s); 0 at ids of -1, and where
 *            that sum is 0
 * A row in which an expert that is in has a logit or a bias that is not a number gets weights that are not numbers; its
 * ids are valid.  Scores, keys and sums are 32-bit.  T >= 0.
 */
int asgd_route(const void *logits, int type, int64_t T, int E, int64_t stride, const float *bias, const asgd_route_rule *rule,
               int32_t *ids, float *weights, void *hip_stream);

/*
 * Gradient of the logits from that of the weights, the choice held fixed: d_logits (T x E of `type`, rows `d_stride`
 * elements apart) is written whole.  logits, bias, rule and ids are those of asgd_route(); d_weights is float T x k, of
 * which the places with ids of -1 are not looked at.
 */
int asgd_route_backward(const void *logits, int type, int64_t T, int E, int64_t stride, const float *bias,
                        const asgd_route_rule *rule, const int32_t *ids, const float *d_weights, void *d_logits,
                        int64_t d_stride, void *hip_stream);

/*
 * The order in which experts take their rows.  Slot t * k + j is choice j of row t; the slots with an expert are put in order of
 * expert, then of slot, and a slot's number in that order is its place.  All four arrays are int32 and device memory.
 */
typedef struct asgd_route_order {
    int64_t T;
    int32_t k, E;
    int32_t *offsets;  /* E + 1: the first place of an expert; [E] = places in use */
    int32_t *blocks;   /* E + 1: the first block of an expert when each begins a new block of 128 places; [E] = blocks in use */
    int32_t *slots;    /* T * k: the slot at a place; -1 at the places that are not in use */
    int32_t *places;   /* T * k: the place of a slot; -1 where it has no expert */
} asgd_route_order;

/* Fills the order from ids (T x k; entries outside 0 .. E - 1 have no expert).  T * k <= 2^30, E <= ASGD_ROUTE_MAX_EXPERTS.
   work: asgd_route_plan_bytes() of scratch, 16-byte aligned (may be NULL if that is 0). */
size_t asgd_route_plan_bytes(int64_t T, int k, int E);
int asgd_route_plan(const int32_t *ids, const asgd_route_order *order, void *work, size_t work_bytes, void *hip_stream);

/* Blocks of 128 that T * k places can need when every expert begins a new one (host arithmetic): T * k / 128 + min(E, T * k). */
int64_t asgd_route_max_blocks(int64_t T, int k, int E);

/*
 * A matrix in 8-bit blocks.  values: e4m3 bytes, `count` matrices of rows x (128 * kb) one after the other, kb =
 * ceil(cols / 128), zeros from column cols on; 16-byte aligned.  An element is its value times the scale of its block:
 *   ASGD_BLOCKS_ROWS     blocks of 1 x 128: scales[kb][rows] (block major; count = 1)
 *   ASGD_BLOCKS_SQUARES  blocks of 128 x 128: scales[count][ceil(rows / 128)][kb]
 *   ASGD_BLOCKS_RAW      not in 8 bits yet: values are rows x cols of `type`, rows `stride` elements apart, scales is
 *                        not used (count = 1); the product brings them to 8 bits as ASGD_BLOCKS_ROWS would on the way
 */
enum { ASGD_BLOCKS_ROWS = 0, ASGD_BLOCKS_SQUARES = 1, ASGD_BLOCKS_RAW = 2 };
typedef struct asgd_blocks {
    void *values;
    float *scales;
    int64_t rows, cols;
    int32_t form;      /* ASGD_BLOCKS_* */
    int32_t count;
    int32_t type;      /* ASGD_BLOCKS_RAW */
    int64_t stride;    /* ASGD_BLOCKS_RAW */
} asgd_blocks;

/*
 * x (count matrices of rows x cols of `type`, rows `stride` elements apart, matrices rows * stride apart) to 8 bits:
 * out's values and scales are written, its rows, cols, form and count say how.  A block with largest magnitude m (at least
 * 1e-30) gets the scale m * (1 / 448) and the values v * (448 * (1 / m)), each operation rounded to 32 bits, then to the nearest e4m3 number, ties to even.
 * A block that holds an infinity or something that is not a number gets a scale that is not a number.
 *   turned = 1   the transpose of x is brought to 8 bits: out has cols rows; blocks lie along x's rows
 *   order        (ASGD_BLOCKS_ROWS only, count = 1, or NULL) x has one row for each of the order's T rows; row p of what is
 *                brought to 8 bits is x's row of the slot at place p, times weights[slot] (float T x k, or NULL).  Not
 *                turned: out->rows = T * k, and the rows at places that are not in use are not written.  Turned: out->cols = 128 *
 *                asgd_route_max_blocks(), and column 128 * blocks[e] + i is place offsets[e] + i of expert e; columns of no
 *                place are zeros, and blocks from blocks[E] on are not written.
 */
int asgd_block_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, int turned,
                        const asgd_route_order *order, const float *weights, const asgd_blocks *out, void *hip_stream);

/* asgd_block_quantize() of the same x twice, not turned into `out` and turned into `out_turned` (both ASGD_BLOCKS_ROWS), from one
   reading of x: what a training step takes of its activations and gradients. */
int asgd_block_quantize_both(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, const asgd_route_order *order,
                             const float *weights, const asgd_blocks *out, const asgd_blocks *out_turned, void *hip_stream);

/*
 * out[i][j] = sum over the blocks of the contraction of (scale of a) * (scale of b) * (sum of a block's products of values); a and b
 * have the same cols.  out: `type`, rows `stride` elements apart.  Scales are applied and blocks added in 32 bits.
 *   exact = 0  a block's products are summed by the 8-bit matrix instruction: it aligns eight neighbours at a time to the
 *              largest of them and drops what lies more than 14 bits below.  The error (root mean square, of the result) is
 *              below 2e-5 where values are of one size and below 1e-4 where they spread over six octaves; no result is off
 *              by more than 7 * 2^-14 of the sum of its products' magnitudes, which is all of it where large products
 *              cancel.  A rounding to float16 costs 2e-4, one to bfloat16 1.7e-3
 *   exact = 1  they are summed in 32 bits, by the 16-bit instruction (half the rate), which holds every value and product
 *   ASGD_PRODUCT_ALL      out (a.rows x b.rows) = a b^T; order = NULL, both counts 1; a ROWS or RAW, b ROWS or SQUARES
 *   ASGD_PRODUCT_GATHER   a (ROWS or RAW) has the order's T rows, b (SQUARES) a matrix for each of its E experts: row p of out
 *                         (T * k x b.rows) is the row of a of the slot at place p times the matrix of the place's expert;
 *                         rows at places that are not in use are not written
 *   ASGD_PRODUCT_PLACES   the same with an `a` that has a row for each place already (ROWS)
 *   ASGD_PRODUCT_OVER     a and b (ROWS) are turned quantisations over the same order: out (E x a.rows x b.rows, matrices
 *                         a.rows * stride apart) = for each expert the product over its own places alone, zeros without any
 * a RAW: at most ASGD_PRODUCT_RAW_ROWS rows (ALL) or ASGD_PRODUCT_RAW_SLOTS slots (GATHER), and b SQUARES.  A matrix in 8-bit
 * blocks has at most 2^30 rows and 2^24 columns, b at most 2^24 rows, out at most 2^22 tiles of 128 x 128.
 */
enum { ASGD_PRODUCT_ALL = 0, ASGD_PRODUCT_GATHER = 1, ASGD_PRODUCT_PLACES = 2, ASGD_PRODUCT_OVER = 3 };
enum { ASGD_PRODUCT_RAW_ROWS = 16, ASGD_PRODUCT_RAW_SLOTS = 4096 };
int asgd_block_product(const asgd_blocks *a, const asgd_blocks *b, int mode, int exact, const asgd_route_order *order, void *out,
                       int type, int64_t stride, void *hip_stream);

/* The kernel that asgd_block_product() takes, from sizes and forms alone (host arithmetic): few rows, whose weights go from memory
   to registers, or tiles of so many rows of a and of b (FAR: of a gathered a of 2^32 bytes and more).  NONE: refused, or nothing to do. */
enum { ASGD_PRODUCT_FORM_NONE = 0, ASGD_PRODUCT_FORM_FEW = 1, ASGD_PRODUCT_FORM_TILES_64 = 2, ASGD_PRODUCT_FORM_TILES_128 = 3,
       ASGD_PRODUCT_FORM_TILES_128_FAR = 4, ASGD_PRODUCT_FORM_TILES_256 = 5 };
int asgd_block_product_form(const asgd_blocks *a, const asgd_blocks *b, int mode, int exact, const asgd_route_order *order);

/*
 * The experts of few rows in one launch, without an order: out[t] = sum over j of weights[t][j] * (x's row t times the
 * matrix ids[t][j] of w), ids outside 0 .. w->count - 1 left out.  x: RAW, at most ASGD_PRODUCT_RAW_ROWS rows; w: SQUARES;
 * ids and weights: rows x k.  Every row reads its experts' matrices for itself.
 */
int asgd_experts_direct(const asgd_blocks *x, const int32_t *ids, const float *weights, int k, const asgd_blocks *w, int exact,
                        void *out, int type, int64_t stride, void *hip_stream);

/*
 * out[t] = sum over j of weights[t][j] * y[place of slot (t, j)], in the order of j and 32-bit, slots without an expert left
 * out (a row that has none: zeros).  y: a row of n elements of y_type for each place, rows y_stride apart; weights: float
 * T x k, or NULL (ones); out: T x n of `type`.
 */
int asgd_experts_sum(const void *y, int y_type, int64_t n, int64_t y_stride, const asgd_route_order *order, const float *weights,
                     void *out, int type, int64_t stride, void *hip_stream);

/* Gradient of those weights: d_weights[t][j] = d_out[t] . y[place of slot (t, j)], 0 at slots without an expert. */
int asgd_experts_sum_backward(const void *d_out, int type, int64_t stride, const void *y, int y_type, int64_t n, int64_t y_stride,
                              const asgd_route_order *order, float *d_weights, void *hip_stream);

/* Device time in milliseconds of the last asgd_run_* call, measured with HIP events recorded on
   the context's stream around its kernel launches.  No device access. */
int asgd_last_run_ms(asgd_ctx *ctx, double *out);

/* ASGD_FORM_* of the last asgd_run_* call.  No device access. */
int asgd_last_run_form(asgd_ctx *ctx, int32_t *out);

/* Totals since asgd_load_shards(). */
int asgd_get_stats(asgd_ctx *ctx, asgd_stats *out);

/* Per-worker message counters (Sec. 5.4, "messages sent or received by a single CPU"):
   each array receives W values; any pointer may be NULL. */
int asgd_get_worker_counters(asgd_ctx *ctx, int64_t *sent, int64_t *received, int64_t *accepted);

/* Recipient of worker i's message of round r under the deterministic schedule
   (host-side copy of what the kernels compute; W >= 2); _n: of copy n of it, 0 <= n < W - 1
   (ASGD_OPT_BUFFERS; copy 0 is the one-buffer schedule).  -1 on invalid arguments. */
int64_t asgd_schedule_peer(uint64_t seed, int64_t r, int64_t i, int64_t W);
int64_t asgd_schedule_peer_n(uint64_t seed, int64_t r, int64_t i, int64_t W, int64_t n);

/* hipError_t of the last failed HIP call of this context (0 if none). */
int asgd_last_hip_error(asgd_ctx *ctx);

/* Release the context and everything it allocated (not the samples, not the dump). */
void asgd_destroy(asgd_ctx *ctx);

/* Static description of a return code. */
const char *asgd_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* ASGD_H */
