/*
 * rip.h -- C ABI of librip, a single-GPU (MI355X, gfx950) implementation of
 * Partial All-Reduce (P-Reduce) with a fused local update, the data-parallel
 * hot path of "Heterogeneity-Aware Asynchronous Decentralized Training"
 * (Ripples; arXiv 1909.08029).
 *
 * N model replicas ("workers") live in one GPU's memory.  One training step
 * of the algorithm of Fig. 4 is, for every worker i that computes this step:
 *   Step 2  x_i <- x_i - lr * grad_i            (optionally with momentum)
 *   Step 3  obtain a group G containing i        (rip_schedule_groups)
 *   Step 4  xbar = (1/|G|) sum_{g in G} x_g;  x_g <- xbar for all g in G
 *                                                (rip_preduce)
 * Groups that share no worker commute and run together in one launch
 * (Sec. 3.2, last paragraph).
 *
 * Conventions for every call below
 *  - Return value: RIP_OK (0) or a negative RIP_E_* code.  On error nothing
 *    is launched and no caller memory is written, except that the message
 *    returned by rip_last_error() is replaced (and except a HIP failure of
 *    the second launch of a split step; see rip_preduce).  No C++ exception
 *    crosses the boundary.
 *  - Host arrays passed in are read during the call only; the caller may
 *    reuse them as soon as the call returns.
 *  - Device buffers (parameters, gradients, momentum) belong to the caller.
 *    The library never allocates, frees or keeps them beyond the work it
 *    enqueues; the caller keeps them alive until the stream passes that work.
 *  - `stream` is a hipStream_t (NULL = the legacy default stream).  Device
 *    work is asynchronous on that stream.
 *  - Handles are not thread-safe; use one handle per thread or lock.
 *  - Graph capture: rip_local_step and rip_preduce enqueue one kernel
 *    launch (up to three for a step of several unit shapes, see rip_preduce;
 *    nothing when the step has no work), each with its part of the step --
 *    schedule, optimizer scalars, the handle's pointer table -- in the kernel
 *    argument, and no memset, copy or allocation.  They may be
 *    called on a stream under HIP graph capture; each replay re-applies the
 *    captured step to whatever the buffers hold then.  The replicas handle
 *    must outlive the graph.
 */
#ifndef RIP_H
#define RIP_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Changes where a declaration below changes what it was; a function that is only
 * added leaves it, as a caller built without that function still runs. */
#define RIP_ABI_VERSION 2

/* status codes */
enum {
  RIP_OK = 0,
  RIP_E_INVAL = -1,        /* bad argument: null pointer, size, id out of range,
                              group not strictly ascending, duplicate active id,
                              steps not consecutive, exhausted script */
  RIP_E_ALIGN = -2,        /* a device buffer is not 16-byte aligned */
  RIP_E_OVERLAP = -3,      /* one replica appears in two groups of one call,
                              or a registered buffer that a step writes
                              overlaps another registered buffer */
  RIP_E_UNSUPPORTED = -4,  /* unknown dtype or mode, or a size above a limit */
  RIP_E_HIP = -5,          /* HIP runtime error (text in rip_last_error) */
  RIP_E_NOMEM = -6         /* host or device allocation failed */
};

/* storage types of parameters, gradients and momentum; arithmetic is fp32 */
enum { RIP_FP32 = 0, RIP_BF16 = 1 };

/* Largest number of replicas one handle or scheduler accepts. */
#define RIP_MAX_REPLICAS 256

/* Message describing the last error on the calling thread ("" if none). */
const char* rip_last_error(void);
int32_t rip_abi_version(void);
/* Kernel launches the calling thread's last rip_preduce, rip_local_step or
 * rip_step enqueued: 0 (an error before any launch, or a step with no work),
 * 1, or 2 or 3 (a step split by its units' sizes; see rip_preduce).  For
 * accounting and tests; results never depend on it. */
int32_t rip_last_launch_count(void);

/* ------------------------------------------------------------------------
 * Group generation (Step 3 of Fig. 4; Sec. 4 and Sec. 5.1-5.3)
 *
 * The scheduler is a stepped model of the paper's Group Generator.  Each
 * worker keeps a request counter c_i (Sec. 5.3) and a Group Buffer, the
 * ordered list of groups that include it (Sec. 5.1).  One call per step t:
 *  1. Active workers = eligible this step and not blocked in a P-Reduce;
 *     they run their local update this step.
 *  2. Each active worker, in ascending id order (the Group Generator serves
 *     requests one at a time), asks for a group:
 *       TABLE / STATIC / RULE: the group of row (c_i - 1) mod period that
 *         contains it (a static schedule, Sec. 4.2, Fig. 8, Fig. 9); a worker
 *         with no group in that row skips synchronization (Sec. 4.2);
 *       RANDOM_GB / GD / INTER_INTRA / SCRIPTED: the head of its Group
 *         Buffer if that is not empty; else new groups are made and appended
 *         to the buffer of every member: one random group containing it
 *         (RANDOM_GB, Step 3 of Fig. 4), a random partition of all idle
 *         workers (Global Division, Sec. 5.1) admitting only workers w with
 *         c_i - c_w < c_thres when c_thres > 0 (Sec. 5.3), the two-phase
 *         Inter-Intra division (Sec. 5.2), or the next group of a script.
 *  3. A group runs when it heads every member's buffer and every member is
 *     blocked in it (serialization of conflicting groups, Sec. 4.1).  The
 *     groups that run are therefore disjoint.  Their members unblock.
 *
 * Random draws: SplitMix64 (Steele, Lea & Flood 2014) with keys folded as
 * k <- mix(k + 0x9E3779B97F4A7C15*(c+1)); bounded(n) = ((x>>32)*n)>>32.
 *   RANDOM_GB/GD/INTER_INTRA: one sequential stream from fold(seed, 3).
 *     RANDOM_GB group: k = min(kmin + bounded(kmax-kmin+1), N); the other
 *     k-1 members by a partial Fisher-Yates over the ascending ids != i
 *     (slot j swaps with j + bounded(N-1-j)).
 *     GD: Fisher-Yates over the ascending idle list (slot a swaps with
 *     bounded(a+1), a from the end), then consecutive chunks whose sizes are
 *     drawn as kmin + bounded(kmax-kmin+1) (the last chunk takes the rest).
 *   STATIC: row r of attempt a from its own stream fold(seed, 3, a, r): a
 *     Fisher-Yates shuffle of 0..N-1 cut into groups of group_size.  Attempts
 *     a = 0, 1, ... until the union of one period's groups connects all
 *     workers (the spectral-gap condition of Sec. 3.3); at most 1000.
 *   RULE: the rule table of Fig. 9: n_nodes nodes of 4 local workers, rank
 *     node*4 + local, period 4 (n_nodes = 1 or even).
 *   INTER_INTRA (Sec. 5.2): N/n_nodes consecutive workers per node.  A
 *     worker with an empty buffer divides the idle workers (same filter as
 *     GD): per node in ascending order a head = idle[bounded(count)]; the
 *     heads (ascending node order), then each node's other idle workers, are
 *     Fisher-Yates shuffled and cut into chunks as in GD (inter phase); then
 *     each node's idle workers form one group (intra phase).  Every idle
 *     worker thus gets its inter group, then its intra group, in its buffer.
 *   ADPSGD (the baseline of Fig. 3, for comparison on the same kernel): each
 *     active worker i draws x = bounded(N-1) and pairs with j = x (x < i) or
 *     x + 1; j is passive and need not be waiting.  Waiting requesters are
 *     then served oldest first; a pair runs unless one of its two workers
 *     is already in a pair of this step (the atomic averaging of Fig. 3),
 *     otherwise the requester keeps waiting.  Groups come out in request
 *     order; only requesters count requests and syncs.  N = 1: every
 *     request is a skip.
 * ---------------------------------------------------------------------- */
enum {
  RIP_SCHED_TABLE = 0,      /* caller's periodic table (FIXED = one row)   */
  RIP_SCHED_STATIC = 1,     /* seeded conflict-free periodic table         */
  RIP_SCHED_RANDOM_GB = 2,  /* random group per request + Group Buffers    */
  RIP_SCHED_GD = 3,         /* Global Division (+ slowdown filter)         */
  RIP_SCHED_SCRIPTED = 4,   /* Group Buffers fed by a caller's group list  */
  RIP_SCHED_RULE = 5,       /* the rule table of Fig. 9                    */
  RIP_SCHED_INTER_INTRA = 6,/* Inter-Intra division (Sec. 5.2)             */
  RIP_SCHED_ADPSGD = 7      /* AD-PSGD pairs with a passive partner (Fig. 3) */
};

typedef struct rip_sched rip_sched; /* opaque, library-owned */

typedef struct rip_sched_cfg {
  int32_t n_workers;   /* N, 1..RIP_MAX_REPLICAS */
  int32_t mode;        /* RIP_SCHED_* */
  uint64_t seed;       /* STATIC, RANDOM_GB, GD, INTER_INTRA, ADPSGD */
  int32_t group_size;  /* STATIC: N % group_size == 0, group_size >= 2 if N > 1 */
  int32_t period;      /* STATIC: rows per period (>= 1); TABLE: number of rows */
  int32_t kmin, kmax;  /* RANDOM_GB, GD, INTER_INTRA: 1 <= kmin <= kmax */
  int32_t c_thres;     /* GD, INTER_INTRA: slowdown threshold, <= 0 = off */
  int32_t n_nodes;     /* RULE: N == 4 * n_nodes; INTER_INTRA: N % n_nodes == 0 */
  /* TABLE: row r holds groups row_offsets[r] .. row_offsets[r+1]-1;
   * SCRIPTED: groups 0 .. n_groups-1 handed out in order.
   * Group g has members members[group_offsets[g] .. group_offsets[g+1]-1],
   * strictly ascending ids in [0, N); groups of one row are disjoint. */
  const int32_t* row_offsets;    /* TABLE: [period + 1], row_offsets[0] == 0 */
  const int32_t* group_offsets;  /* TABLE, SCRIPTED: [n_groups + 1] */
  const int32_t* members;        /* TABLE, SCRIPTED */
  int32_t n_groups;              /* TABLE, SCRIPTED */
} rip_sched_cfg;

/* Create a scheduler.  The configuration and its arrays are copied.
 * Errors: RIP_E_INVAL (sizes, table contents, a STATIC table with no
 * connected attempt), RIP_E_UNSUPPORTED (mode), RIP_E_NOMEM. */
int32_t rip_sched_create(const rip_sched_cfg* cfg, rip_sched** out);
void rip_sched_destroy(rip_sched* s); /* NULL is a no-op */

/* Schedule step `step`; steps must be 0, 1, 2, ... in order.
 *  eligible      [N] host bytes, nonzero = the worker finishes a local
 *                iteration this step if it is free; NULL = all eligible.
 *  active        out [N]: ascending ids of the workers updating this step
 *  n_active      out
 *  group_offsets out [N + 1], members out [N]: the groups that run this step
 *                as CSR, members ascending; ordered by creation (group-buffer
 *                modes) or by (iteration, position in the row) (table modes)
 *  n_groups      out
 * Output capacities are always enough: groups that run are disjoint.
 * Errors: RIP_E_INVAL (null handle or output, step out of order, a scripted
 * group that does not contain its requester, an exhausted script).  On an
 * error the scheduler state is unchanged. */
int32_t rip_schedule_groups(rip_sched* s, int64_t step, const uint8_t* eligible,
                            int32_t* active, int32_t* n_active,
                            int32_t* group_offsets, int32_t* members,
                            int32_t* n_groups);

typedef struct rip_worker_state {
  int64_t requests;  /* c_i: requests made (local iterations finished) */
  int64_t syncs;     /* groups of this worker that ran */
  int64_t skips;     /* requests with no group (table modes) */
  int32_t waiting;   /* 1 if blocked in a P-Reduce */
  int32_t gb_depth;  /* entries in its Group Buffer (ADPSGD: 1 while its pair waits) */
} rip_worker_state;

/* Counters of one worker; requests == syncs + skips + waiting always. */
int32_t rip_sched_worker(const rip_sched* s, int32_t worker, rip_worker_state* out);

/* ------------------------------------------------------------------------
 * Replicas: registered once, used by every step.
 *
 * Each replica r holds S segments (e.g. the layer tensors of a model; the
 * paper flattens them into one buffer per worker, Sec. 6.1 -- here they may
 * stay separate, or be views of one flat buffer).  Segment s has
 * seg_numel[s] elements in every replica.
 *  param  [N*S] host array of device pointers, param[r*S + s]
 *  grad   [N*S] or NULL (then only pure P-Reduce is possible)
 *  mom    [N*S] or NULL (momentum buffers, same storage type)
 * When every replica's non-empty segments lie back to back in memory (and
 * likewise for grad and mom), they are treated as one flat range and only
 * its first segment must be 16-byte aligned; otherwise every non-empty
 * segment must be.  Zero-length segments may be NULL.
 * Every non-empty segment must be device (or managed) memory of the current
 * device and lie inside the allocation holding its first byte; the buffers a
 * step writes (param, mom) must not overlap any other registered segment.
 * Gradient segments may overlap each other (replicas may share a gradient).
 * A step reads and writes the registered elements and nothing else, with one
 * exception: of a bf16 segment (or flat range) of odd length it reads the
 * whole aligned four bytes that hold the last element.  The two bytes after it
 * lie in the same page; no result depends on them, and they are not written.
 * The handle copies the pointer table to device memory (one allocation,
 * freed by rip_replicas_destroy) on the current device; calls using it must
 * run with that device current.  Destroy only after the work that uses it
 * has finished.
 * Errors: RIP_E_INVAL (also: not device memory of this device, or a
 * segment running past its allocation), RIP_E_ALIGN, RIP_E_OVERLAP (a
 * written segment overlapping another), RIP_E_UNSUPPORTED (dtype, N above
 * RIP_MAX_REPLICAS), RIP_E_NOMEM, RIP_E_HIP. */
typedef struct rip_replicas rip_replicas; /* opaque, library-owned */

int32_t rip_replicas_create(int32_t n_replicas, int32_t n_segments, int32_t dtype,
                            const int64_t* seg_numel, void* const* param,
                            void* const* grad, void* const* mom, rip_replicas** out);
void rip_replicas_destroy(rip_replicas* r); /* NULL is a no-op */

/* For callers that cannot allocate device memory (code that runs while a HIP
 * graph is being captured, tight serving loops, harnesses that forbid
 * hipMalloc): the same registration as rip_replicas_create, with the same
 * arguments, checks and errors, but the handle's device tables (pointer
 * table and segment tables) go into a fixed array of RIP_NOALLOC_TABLE_BYTES
 * that the library keeps on each device for the life of the process, copied
 * there with a blocking hipMemcpy.  It calls no hipMalloc or hipFree.
 * Size: the tables take 24*N*S' + 8*S' + 32*(S'+1) bytes, where S' is 1 when
 * the segments are back to back (one flat range) and S otherwise; above the
 * array's size the call fails with RIP_E_UNSUPPORTED and changes nothing
 * (a failure of the copy itself, RIP_E_HIP, still supersedes the previous
 * handle).
 * Sharing: every such handle on a device uses that device's one array, which
 * keeps the last registration's tables.  Creating another one supersedes the
 * previous handle on that device: its later calls fail with RIP_E_INVAL
 * (destroying it is still fine).  A registration that overlaps work still in
 * flight with the previous handle on that device races with that work:
 * finish it (synchronize) first.  The handle is used and destroyed like any
 * other; handles from rip_replicas_create are unaffected.  The registration
 * itself copies synchronously, so it is made outside a stream capture; the
 * rip_preduce / rip_local_step / rip_step launches that use the handle may
 * then be captured like any others. */
#define RIP_NOALLOC_TABLE_BYTES 65536
int32_t rip_replicas_create_noalloc(int32_t n_replicas, int32_t n_segments, int32_t dtype,
                                    const int64_t* seg_numel, void* const* param,
                                    void* const* grad, void* const* mom, rip_replicas** out);

/* ------------------------------------------------------------------------
 * Local update and P-Reduce (Steps 2 and 4 of Fig. 4; F^G of Sec. 3.2)
 *
 * Arithmetic (fp32, this exact order; no fused multiply-add):
 *   active worker r:  g' = g_r + wd*w_r when weight_decay != 0, else g' = g_r;
 *                     u_r = w_r - lr*g', or with momentum
 *                     v_r = mu*v_r + g' (stored) and u_r = w_r - lr*v_r
 *                     (Nesterov: u_r = w_r - lr*(g' + mu*v_r))
 *   other worker r:   u_r = w_r
 *   group m1 < ... < mk:  s = u_m1; s = s + u_mj (j = 2..k, ascending);
 *                     xbar = s * (float)(1.0/k); w_m = xbar for every member
 *   active worker in no group: w_r = u_r
 *   every other replica: not read, not written.
 * bf16 storage: values widen exactly to fp32 and are rounded to nearest-even
 * once, when stored.  Momentum buffers are never averaged (Step 4 averages
 * parameters only).  momentum == 0 is plain SGD and leaves mom untouched.
 * The paper's ResNet-50 runs use momentum 0.9 and weight decay 1e-4
 * (Sec. 7.1.2); its VGG-16 runs plain SGD.
 * ---------------------------------------------------------------------- */
typedef struct rip_sgd {
  float lr;            /* learning rate (eta in Fig. 4) */
  float momentum;      /* mu; 0 = plain SGD.  Needs mom buffers when nonzero. */
  float weight_decay;  /* wd, added to the gradient as wd*w; 0 = none */
  int32_t nesterov;    /* nonzero: Nesterov momentum (needs momentum != 0) */
} rip_sgd;

/* Step 2 alone for the `n_active` workers listed in `active` (distinct ids).
 * Same as rip_preduce with no groups.
 * Errors: RIP_E_INVAL (null handle/sgd, ids, no grad or needed mom buffers,
 * Nesterov without momentum, device mismatch), RIP_E_UNSUPPORTED, RIP_E_HIP
 * as rip_preduce. */
int32_t rip_local_step(const rip_replicas* r, const int32_t* active, int32_t n_active,
                       const rip_sgd* sgd, void* stream);

/* Steps 2 and 4 fused in one pass over memory, for one step of the schedule:
 * the local update of every listed active worker, then the P-Reduce of each
 * of the `n_groups` groups given as CSR (group g = members[group_offsets[g]
 * .. group_offsets[g+1]-1], strictly ascending).  Groups must be disjoint
 * (RIP_E_OVERLAP otherwise).  sgd == NULL is pure P-Reduce; then n_active
 * must be 0.  One kernel launch covers all groups and updates, with two
 * exceptions, each of which adds one, in a row on `stream`: groups above eight
 * run on a kernel of their own, beside other units in more than a small launch;
 * and where the units of up to eight members move 1 GiB or more and prefer
 * residency caps far apart (a Global Division step of pairs and groups of
 * eight, say), they are two launches, unless a cap is forced with
 * rip_set_blocks_per_cu.  The units are disjoint, so the result is the same
 * either way.  If a launch fails, those before it have been enqueued
 * (RIP_E_HIP).
 * Errors: RIP_E_INVAL (also: the current device is not the handle's),
 * RIP_E_OVERLAP, RIP_E_UNSUPPORTED (a step of 2^31 or more tiles), RIP_E_HIP
 * (launch failure). */
int32_t rip_preduce(const rip_replicas* r, const int32_t* group_offsets,
                    const int32_t* members, int32_t n_groups, const int32_t* active,
                    int32_t n_active, const rip_sgd* sgd, void* stream);

/* One whole step of the algorithm of Fig. 4 for every worker in one call:
 * group generation for `step` (Step 3, exactly as rip_schedule_groups with
 * the same arguments), then the fused local update and P-Reduce of the
 * groups that run (Steps 2 and 4, as rip_preduce with those groups and the
 * active workers).  Saves the host round trip between the two calls.
 *  s, r       scheduler and replicas handle with the same number of workers
 *  sgd        required (the workers that finish an iteration update); the
 *             handle needs gradient buffers, and momentum buffers when
 *             sgd->momentum != 0
 *  active .. n_groups  optional outputs, as in rip_schedule_groups (NULL =
 *             not wanted); written only on success
 * Atomic: on any error (including a failed launch) the scheduler is left as
 * it was, as if the call had not been made, and nothing is launched (a HIP
 * failure of the second launch of a split step leaves the first enqueued).
 * Errors: RIP_E_INVAL (null handle or sgd, worker counts differ, missing
 * buffers, Nesterov without momentum, device mismatch, a scheduling error),
 * RIP_E_HIP. */
int32_t rip_step(rip_sched* s, const rip_replicas* r, int64_t step, const uint8_t* eligible,
                 const rip_sgd* sgd, void* stream, int32_t* active, int32_t* n_active,
                 int32_t* group_offsets, int32_t* members, int32_t* n_groups);

/* Launch tuning (process-wide).  rip_set_max_blocks caps the workgroups of
 * one launch (0 = the default: one workgroup per tile up to 2^25
 * workgroups, beyond which workgroups loop over tiles); rip_set_blocks_per_cu
 * caps how many of the kernel's workgroups share a compute unit (0 = the
 * default: chosen per launch from its units' sizes, whether their members
 * update, momentum, and whether the handle has several segments: 4-14 per
 * compute unit, 16 in a launch of that many or fewer; 1-10 of the several-wave
 * workgroups of groups above eight).  Negative values are RIP_E_INVAL.
 * Results never depend on these settings. */
int32_t rip_set_max_blocks(int32_t max_blocks);
int32_t rip_set_blocks_per_cu(int32_t blocks_per_cu);

/* ------------------------------------------------------------------------
 * Operators that fill the gradient buffers of language-model replicas
 *
 * A replica's training pass begins at its embedding, keeps what its layers need
 * for the backward pass, and ends in a loss over the vocabulary.  These calls
 * write straight into registered gradient segments (rip_replicas_create), which
 * the next rip_step / rip_preduce reads.  Each works on one replica's buffers.
 *
 * Conventions beyond those at the top of this file
 *  - A matrix is a device pointer, its type (RIP_FP32 / RIP_BF16) and its row
 *    stride `ld` in elements (at least its width).  It need only be aligned to
 *    its elements; columns between the width and `ld` are not written (nor read,
 *    unless a call says so).  Indexes into it are 64-bit.
 *  - Arithmetic and every sum are fp32 (or wider); a result is rounded to bf16
 *    once, to nearest even.  Nothing is added atomically: a call's result is the
 *    same bits every time for the same sizes, strides and alignment (a loss adds
 *    a row's exponentials in an order that follows the sixteen-byte boundaries).
 *  - Token ids and targets are RIP_INT32 or RIP_INT64 device arrays.
 *  - `workspace` is device memory of at least the bytes that the call's
 *    _workspace function returns for the same sizes (0 = none needed; sizes that
 *    the call itself refuses also give 0), 16-byte aligned, free again when the
 *    stream has passed the call.  It need not be cleared.
 *  - A buffer that a call writes must not overlap any other of its buffers,
 *    except where a call says that it may be the same matrix.  Arrays of 32-bit
 *    numbers (offsets, log-probabilities, weights, a loss) are 4-byte aligned.
 *  - Empty inputs (no tokens) are no error; their pointers may be NULL.
 *  - All calls are only kernel launches on `stream` (no allocation, copy, memset
 *    or wait), so they may be captured into a HIP graph.
 * Errors of every call: RIP_E_INVAL (null pointer, size, row stride, workspace
 * too small, a scalar out of its range), RIP_E_ALIGN, RIP_E_OVERLAP,
 * RIP_E_UNSUPPORTED (type, size above a limit), RIP_E_HIP.
 * ---------------------------------------------------------------------- */
enum { RIP_INT32 = 0, RIP_INT64 = 1 };  /* types of token ids */

#define RIP_MAX_TOKENS (1 << 23)    /* tokens (rows) of one call */
#define RIP_MAX_WIDTH (1 << 24)     /* columns of a row; logits of a token */
#define RIP_MAX_FEATURES (1 << 18)  /* rows and columns of a layer's weight */
#define RIP_MAX_PAIRS (1 << 20)     /* pairs of sequences of one call */

/* Embedding lookup: out[t] = scale * table[ids[t]] for n_tokens rows of `width`.
 * An id outside 0 .. vocab-1 (padding) gives a row of zeros.  table and out may
 * have different types. */
int32_t rip_embed_lookup(const void* table, int32_t table_dtype, int64_t vocab, int64_t width,
                         int64_t ld_table, const void* ids, int32_t id_type, int64_t n_tokens,
                         float scale, void* out, int32_t out_dtype, int64_t ld_out, void* stream);

/* Its gradient: grad[v] = scale * sum of dout[t] over the tokens with ids[t] == v
 * (ascending t within fixed runs of tokens, whose sums are added in order), for
 * every row of the table: rows that no token names become zeros.  With
 * `accumulate` nonzero the sums are added to what grad holds and the other rows
 * are not touched.  Ids outside the vocabulary contribute nothing. */
int64_t rip_embed_grad_workspace(int64_t n_tokens, int64_t width);
int32_t rip_embed_grad(const void* dout, int32_t dout_dtype, int64_t ld_dout, const void* ids,
                       int32_t id_type, int64_t n_tokens, float scale, void* grad,
                       int32_t grad_dtype, int64_t vocab, int64_t width, int64_t ld_grad,
                       int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream);

/* Activations kept in 8 bits.  A checkpoint of `rows` rows of `width` columns is
 *   codes [rows][32 * ceil(width / 32)] int8, 16-byte aligned
 *   exps  [rows][ceil(width / 32)] uint8
 * A block is 32 columns of a row (the last may be short; its other codes are 0).
 * With e = exp - 127, code q stands for q * 2^e, q in -127 .. 127: e is the
 * smallest integer in -126 .. 121 for which the block's largest magnitude is at
 * most 127 * 2^e (121 for a magnitude beyond 127 * 2^121), and q is x / 2^e
 * rounded to nearest, ties to even, and cut to -127 .. 127.  A block with an
 * infinity or a NaN has exp 255 and codes 0 and stands for NaN throughout, so
 * that a diverged value is not lost.
 * rip_ckpt_unpack writes the values it stands for (exact in bf16 too). */
int32_t rip_ckpt_pack(const void* x, int32_t dtype, int64_t ld, int64_t rows, int64_t width,
                      int8_t* codes, uint8_t* exps, void* stream);
int32_t rip_ckpt_unpack(const int8_t* codes, const uint8_t* exps, int64_t rows, int64_t width,
                        void* x, int32_t dtype, int64_t ld, void* stream);

/* Gated unit of a feed-forward layer: h = silu(gate) * up, silu(z) = z / (1 +
 * e^-z), from the inputs as given; gate and up are kept as checkpoints in the
 * same pass.  gate and up may lie side by side in the rows of one buffer; h may
 * be the same matrix as gate or up. */
int32_t rip_gate_forward(const void* gate, int64_t ld_gate, const void* up, int64_t ld_up,
                         int32_t dtype, int64_t rows, int64_t width, void* h, int64_t ld_h,
                         int8_t* gate_codes, uint8_t* gate_exps, int8_t* up_codes,
                         uint8_t* up_exps, void* stream);

/* Its backward pass from the checkpoints' values g, u, with s = 1 / (1 + e^-g):
 *   dgate = dh * u * s * (1 + g * (1 - s)),   dup = dh * g * s
 * and, unless h_codes and h_exps are both NULL, a checkpoint of g * s * u: the
 * next layer's input, so that no forward pass need keep it.  dgate and dup may
 * lie side by side in the rows of one buffer; one of them may be dh. */
int32_t rip_gate_backward(const void* dh, int64_t ld_dh, int32_t dtype, const int8_t* gate_codes,
                          const uint8_t* gate_exps, const int8_t* up_codes,
                          const uint8_t* up_exps, int64_t rows, int64_t width, void* dgate,
                          int64_t ld_dgate, void* dup, int64_t ld_dup, int8_t* h_codes,
                          uint8_t* h_exps, void* stream);

/* Weight gradient of a linear layer y = x W^T from the checkpoint of x:
 *   grad[n][k] = sum_t dy[t][n] * x'[t][k]     (out_features x in_features)
 * added to what grad holds if `accumulate` is nonzero.  x' is what the
 * checkpoint stands for; products are exact and sums fp32 for either type of dy.
 * Of dy it also reads up to seven elements after a row but the last one; no
 * result depends on them.  Its row stride is at most RIP_MAX_WIDTH. */
int64_t rip_ckpt_wgrad_workspace(int32_t dy_dtype, int64_t rows, int64_t out_features,
                                 int64_t in_features);
int32_t rip_ckpt_wgrad(const void* dy, int32_t dy_dtype, int64_t ld_dy, int64_t rows,
                       int64_t out_features, const int8_t* codes, const uint8_t* exps,
                       int64_t in_features, void* grad, int32_t grad_dtype, int64_t ld_grad,
                       int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream);

/* Preference loss over pairs of sequences, and the gradient of the logits.
 *   logits   [n_tokens][vocab]; targets[t] is the token that row t predicts
 *   seq_offsets [2 * n_pairs + 1] int32 on the device, ascending: sequence q is
 *            the tokens seq_offsets[q] .. seq_offsets[q+1]-1; 2p is the chosen
 *            and 2p+1 the rejected one of pair p.  Offsets that are not so are cut
 *            to fit: to 0 .. n_tokens, and one below an earlier offset (of any
 *            pair) to the largest of those, so that no token is in two sequences.
 *   ref_logp [2 * n_pairs] log-probabilities of the sequences under the reference
 * A token counts unless its target lies outside 0 .. vocab-1 (prompt, padding),
 * it belongs to no sequence, or every logit of its row is -inf.  With
 *   logp[t] = log softmax(logits[t])[targets[t]]   (0 where it does not count)
 *   seq_logp[q] = sum of logp over sequence q (in 64 bits, then rounded)
 *   z_p = beta * ((seq_logp[2p] - ref_logp[2p]) - (seq_logp[2p+1] - ref_logp[2p+1]))
 *   loss = mean over p of -(1 - smoothing) log sigmoid(z_p) - smoothing log sigmoid(-z_p)
 * grad is grad_scale * d loss / d logits, zeros in the rows that do not count,
 * whatever those rows hold.  Outputs: loss [1], seq_logp [2 * n_pairs], logp
 * [n_tokens] or NULL, grad or NULL (only the loss), which may be the same matrix
 * as logits. */
int64_t rip_pref_loss_workspace(int64_t n_tokens, int64_t vocab, int32_t n_pairs);
int32_t rip_pref_loss(const void* logits, int32_t dtype, int64_t ld, int64_t n_tokens,
                      int64_t vocab, const void* targets, int32_t id_type,
                      const int32_t* seq_offsets, int32_t n_pairs, const float* ref_logp,
                      float beta, float smoothing, float grad_scale, float* loss, float* seq_logp,
                      float* logp, void* grad, int64_t ld_grad, void* workspace,
                      int64_t workspace_bytes, void* stream);

/* Clipped policy loss with a KL term, and the gradient of the logits.  logp and
 * which tokens count are as above (there are no sequences).  For a counted token
 *   r = e^(logp - old_logp),  c = min(max(r, 1 - clip_low), 1 + clip_high)
 *   loss_t = -min(r * advantage, c * advantage) + kl * (e^d - d - 1),  d = ref_logp - logp
 *   loss = sum over the counted t of weight[t] * loss_t
 * The derivative by logp of the first term is -r * advantage where r * advantage
 * <= c * advantage, else 0.  An advantage of 0 makes the first term and its
 * derivative 0 also where r is beyond fp32.  A token of weight 0 adds nothing to the
 * loss and its row of grad is zeros, whatever its other numbers are.  old_logp,
 * advantage, weight and ref_logp are fp32 [n_tokens]; weight NULL stands for
 * 1 / n_tokens, ref_logp may be NULL if kl is 0.  0 <= clip_low <= 1, clip_high >= 0.
 * Outputs as above. */
int64_t rip_policy_loss_workspace(int64_t n_tokens, int64_t vocab);
int32_t rip_policy_loss(const void* logits, int32_t dtype, int64_t ld, int64_t n_tokens,
                        int64_t vocab, const void* targets, int32_t id_type, const float* old_logp,
                        const float* advantage, const float* weight, const float* ref_logp,
                        float clip_low, float clip_high, float kl, float grad_scale, float* loss,
                        float* logp, void* grad, int64_t ld_grad, void* workspace,
                        int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RIP_H */
