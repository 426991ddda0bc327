/*
 * vie_head.h - C ABI of the exact LLM output head for GB300 (sm_103a).
 *
 * The head computes, for each decode query h (paper, Section 3):
 *     z = W_out h,            z_i = <w_i, h>        (W_out: V rows of width d)
 * selects the k rows with the largest z_i (exhaustive maximum inner product
 * search, Sections 2-3) and can write those k logits into a full-vocabulary
 * tensor that is -infinity everywhere else (Section 3, the sparse logit
 * tensor handed to standard logit processors).
 *
 * Conventions shared by every call:
 *   - Pointers marked "device" are CUDA device pointers of the device that is
 *     current on the calling thread; "host" pointers are ordinary memory.
 *   - A vie_stream is a cudaStream_t (NULL = the legacy default stream).  Calls
 *     that take a stream are asynchronous on it: they validate on the host,
 *     enqueue kernels and return without synchronising.
 *   - Every call returns a vie_status.  On anything but VIE_OK,
 *     vie_last_error() returns a message for the calling thread.  Argument
 *     errors are detected on the host before anything is enqueued; they leave
 *     no CUDA error behind.
 *   - Device-side problems (an out-of-range scatter index, a pipeline wait
 *     that ran past its time limit) never trap: the kernel records a flag and
 *     returns, and the next vie_device_status / vie_head_device_status call
 *     reports VIE_ERR_DEVICE.  The outputs of the call that recorded a wait
 *     time-out are unspecified (every write still stays inside them).
 *   - Logits are fp32.  Ranking is by logit descending; equal logits are
 *     ranked by ascending vocabulary index, and -0.0 ranks as +0.0 (and is
 *     returned as +0.0).  Inputs must be finite, and results for NaN or
 *     infinite inputs are unspecified, unless a call says otherwise.
 */
#ifndef VIE_HEAD_H
#define VIE_HEAD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct vie_head vie_head; /* opaque handle */
typedef void *vie_stream;         /* a cudaStream_t */

typedef enum {
    VIE_OK = 0,
    VIE_ERR_INVALID_ARG = 1, /* a pointer, size or enum value is out of range */
    VIE_ERR_UNSUPPORTED = 2, /* valid request beyond what this library serves */
    VIE_ERR_CUDA = 3,        /* a CUDA runtime call or a launch failed        */
    VIE_ERR_OOM = 4,         /* device memory could not be allocated          */
    VIE_ERR_DEVICE = 5       /* a kernel recorded a device-side problem       */
} vie_status;

typedef enum {
    VIE_DTYPE_BF16 = 0,
    VIE_DTYPE_F32 = 1 /* logits, tables and gradients below; heads hold bf16 or e4m3 rows */
} vie_dtype;

/* Limits of this library. */
#define VIE_K_MAX 1024     /* largest k of vie_head_topk                    */
#define VIE_BATCH_MAX 1024 /* largest batch of vie_head_topk                */
#define VIE_D_MAX 16384    /* largest hidden size d                         */
#define VIE_MANY_MAX (1 << 24)     /* largest n of vie_head_topk_many       */
#define VIE_RECALL_N_MAX (1 << 28) /* largest n of vie_recall_hits          */
#define VIE_RECALL_M_MAX (1 << 20) /* largest candidate count m             */
#define VIE_DISTILL_V_MAX (1 << 30) /* largest V of vie_distill_topk*       */
#define VIE_SAMPLE_V_MAX (1 << 22) /* largest V of vie_sample_logits        */
#define VIE_PREFERENCE_N_MAX (1 << 30) /* most tokens of vie_preference_loss* */
#define VIE_E2M1_N_MAX (1 << 28)   /* most rows of an e2m1 matrix           */

/* Read-only facts about a handle (for callers that size buffers or report). */
typedef struct {
    int64_t V;            /* vocabulary rows                                 */
    int32_t d;            /* hidden size                                     */
    int32_t d_pad;        /* row pitch in elements: d rounded up to 8        */
    int32_t ctas;         /* CTAs of one projection launch (one per SM max)  */
    int32_t device;       /* CUDA device ordinal the handle lives on         */
    int64_t weight_bytes; /* bytes of the owned padded copy of W_out         */
    int64_t scratch_bytes;/* bytes of per-handle scratch, query matrix and all
                             (not vie_head_topk_host's staging buffers)       */
} vie_head_props;

/*
 * vie_head_create - take a copy of W_out in the layout the kernels stream.
 * Section 3 treats the rows of W_out as a static database that is prepared
 * once and reused for every query; this is that preparation step.
 *
 *   W_out  device, bf16 (raw bit patterns), row-major [V, d], any alignment
 *          of 2 bytes.  Only read during the call; the caller may free it
 *          afterwards.
 *   V      1 <= V <= 2^31 - 2;   d   1 <= d <= VIE_D_MAX;
 *   dtype  VIE_DTYPE_BF16 (the only dtype that a head takes).
 *   out    host; receives the new handle.
 *
 * The handle owns a padded copy [V, d_pad] (d_pad = d rounded up to a
 * multiple of 8, pad = +0) plus its scratch.  The copy runs on the legacy
 * default stream of the current device and the call returns after the device
 * has finished it.  Errors: VIE_ERR_INVALID_ARG (null pointer, bad size,
 * W_out not device memory of the current device), VIE_ERR_UNSUPPORTED
 * (dtype), VIE_ERR_OOM, VIE_ERR_CUDA.
 */
vie_status vie_head_create(const void *W_out, int64_t V, int32_t d, vie_dtype dtype,
                           vie_head **out);

/*
 * vie_head_create_e4m3 - a head whose rows are stored as 8-bit floats: the
 * paper names weight quantisation as a bandwidth saving orthogonal to its
 * method (Section 4); this is that variant of the exact head, streaming half
 * the bytes of the bf16 head per decode step.
 *
 *   W_out   device, bf16, row-major [V, d], 2-byte aligned (as for
 *           vie_head_create); quantised on the device before the call returns.
 *   V, d    as for vie_head_create.
 *
 * Row i is stored as e4m3 codes (1 sign, 4 exponent bits with bias 7, 3
 * mantissa bits, largest finite value 448) and one fp32 scale:
 *   scale_i = max_j |w_ij| / 448 in fp32 (1 for an all-zero row);
 *   q_ij = w_ij / scale_i in fp32, rounded to the nearest e4m3 value (ties
 *          to even, saturated at +-448);
 * and every top-k call on the handle (vie_head_topk, _sparse, _host,
 * _sample) computes z_i = scale_i * sum_j e4m3(q_ij) * h_j with fp32
 * accumulation, then the same exact top-k.  Calls with k <= 128 on rows of
 * at least 128 codes run on the tensor cores (tcgen05 kind::f8f6f4; each
 * query enters as four e4m3 pieces with power-of-two scales, which keep it to
 * within 2^-16 |h_j| per entry), from batch 1 (vie_head_plan reports path
 * 1); other calls use the streaming CUDA-core kernel.  Same errors as
 * vie_head_create.
 */
vie_status vie_head_create_e4m3(const void *W_out, int64_t V, int32_t d, vie_head **out);

/* Copies an e4m3 handle's codes (device uint8 [V, d], row-major) and scales
 * (device fp32 [V]) to caller buffers, asynchronously on `stream`.
 * VIE_ERR_INVALID_ARG for a bf16 handle or NULL arguments. */
vie_status vie_head_export_e4m3(const vie_head *head, uint8_t *codes, float *scales,
                                vie_stream stream);

/* Frees the padded copy and the scratch.  NULL is accepted.  The caller must
 * make sure no work using the handle is still running (synchronise first). */
vie_status vie_head_destroy(vie_head *head);

/* Fills *props (host) with the handle's facts. */
vie_status vie_head_get_props(const vie_head *head, vie_head_props *props);

/* How a vie_head_topk / vie_head_topk_sparse call of this size runs.  Each
 * query group is one pass over W_out, but for bf16 batches of 256 queries or
 * more with k <= 128 (on vocabularies of 8192 rows or more whose sample fits the
 * handle's scratch): those run as a filtered GEMM on the tensor cores, in groups
 * of 128 queries, and read W_out about once per block of up to four groups (plus
 * every 8th to 64th row), five launches each: launches / 5 times. */
typedef struct {
    int32_t path;     /* 0: streaming CUDA-core kernel, 1: tensor-core kernel  */
    int32_t groups;   /* query groups (see above)                             */
    int32_t launches; /* kernel launches the call enqueues                    */
} vie_topk_plan;

/* Fills *plan (host) for a call with this batch and k; the same argument
 * checks as vie_head_topk.  Nothing is enqueued. */
vie_status vie_head_plan(const vie_head *head, int32_t batch, int32_t k, vie_topk_plan *plan);

/*
 * Launch options - a hook for tests and tuning; the paper has no counterpart.
 *
 * By default the path and launch shape of a call depend only on the call
 * (batch, k), the handle (V, d, bf16 or e4m3 rows) and the device: the
 * defaults below are the shapes that measured fastest on GB300 and that the
 * test suite covers.  An option changes how the work is laid out (which
 * kernel, stage sizes, work split), never the results: every setting gives
 * the same top-k under the same ranking rule.  Options are process-wide
 * (all handles, all threads) and are read when a call plans its launches, so
 * a change takes effect from the next call on; change them only while no
 * other thread is inside a call of this library.  Nothing is read from the
 * environment.
 */
typedef enum {
    VIE_OPT_STAGE_MIN_KB = 0,      /* smallest streaming weight stage, KB       (48)  */
    VIE_OPT_STATIC_PCT = 1,        /* % of W's pieces dealt round robin, rest
                                      drawn from a shared pool                   (85)  */
    VIE_OPT_POOL_DIV = 2,          /* pool pieces = one stage / this, 1..64      (1)   */
    VIE_OPT_TC_MIN_BATCH = 3,      /* smallest batch of a bf16 head sent to the
                                      tensor cores (k <= 128)                   (2)   */
    VIE_OPT_TC_KPS = 4,            /* most K-blocks per tensor-core stage, 1..4  (4)   */
    VIE_OPT_TC_MIN_BATCH_E4M3 = 5, /* the same threshold for e4m3 heads          (1)   */
    VIE_OPT_HALF_ROWS = 6,         /* streaming projection, one row per
                                      half-warp: 1 on, 0 off, -1 automatic       (-1)  */
    VIE_OPT_HOST_H_DIRECT = 7,     /* vie_head_topk_host reads page-locked
                                      queries in place: 1, or copies them: 0     (1)   */
    VIE_OPT_EARLY_MERGE = 8,       /* single-query streaming launches with
                                      k <= 64: one CTA merges the per-CTA lists
                                      while the others still stream: 1, or the
                                      last CTA to finish merges them all: 0      (1)   */
    VIE_OPT_COUNT = 9
} vie_launch_option;

#define VIE_OPT_DEFAULT INT32_MIN /* value that restores an option's default */

/* Sets one option (VIE_OPT_DEFAULT restores its default).  Errors:
 * VIE_ERR_INVALID_ARG for an unknown option or a value outside the range
 * given above (the option keeps its value). */
vie_status vie_set_launch_option(vie_launch_option option, int32_t value);

/* Reads one option's current value into *value (host). */
vie_status vie_get_launch_option(vie_launch_option option, int32_t *value);

/*
 * vie_head_topk - exact top-k of z = W_out h for a batch of queries
 * (Section 3: output projection followed by top-k selection, computed by
 * exhaustive MIPS over every row, Section 2).
 *
 *   h           device, fp32, row-major [batch, d] (4-byte aligned).
 *   batch       1 <= batch <= VIE_BATCH_MAX.
 *   k           1 <= k <= min(V, VIE_K_MAX).
 *   out_idx     device, int32 [batch, k]: vocabulary indices, best first.
 *   out_logits  device, fp32  [batch, k]: their logits (fp32 accumulation of
 *               the bf16 x fp32 products).
 *   stream      the stream the work is enqueued on.
 *
 * Batches on the tensor cores start by sharing a bound on the k-th logit
 * between all CTAs of the launch, one per SM, and wait at most 20 us for it; when
 * kernels of another stream hold some SMs, that wait runs out on every such
 * launch (the results are the same).
 * The full logit vector is never written to memory.  Calls using the same
 * handle share its scratch, so at most one vie_head_topk per handle may be
 * in flight at a time (calls on one stream are naturally serialised).
 * No allocation and no host synchronisation happen inside the call.
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_CUDA (launch failure).
 */
vie_status vie_head_topk(vie_head *head, const float *h, int32_t batch, int32_t k,
                         int32_t *out_idx, float *out_logits, vie_stream stream);

/*
 * vie_head_topk_sparse - vie_head_topk and the sparse full-vocabulary logit
 * tensor of Section 3 in one launch: besides out_idx / out_logits it writes
 *   out_sparse  device, fp32 [batch, V] (4-byte aligned): -inf (0xFF800000)
 *               everywhere except out_sparse[b, out_idx[b, j]] =
 *               out_logits[b, j] (the same bits).
 * The result equals vie_head_topk followed by vie_scatter_sparse_logits on
 * its outputs.  Same limits, sharing rule and errors as vie_head_topk.
 */
vie_status vie_head_topk_sparse(vie_head *head, const float *h, int32_t batch, int32_t k,
                                int32_t *out_idx, float *out_logits, float *out_sparse,
                                vie_stream stream);

/*
 * vie_head_topk_host - one whole decode step for a caller whose queries and
 * results live in host memory: copies h in, runs vie_head_topk_sparse (or
 * vie_head_topk when out_sparse is NULL), copies the top-k out and waits for
 * it.  The paper has no counterpart: it is the end-to-end form of the call.
 *
 *   h_host       host, fp32, row-major [batch, d].  Page-locked memory
 *                (cudaMallocHost / cudaHostRegister) keeps the copies
 *                asynchronous; pageable memory works, staged by the driver.
 *   idx_host     host, int32 [batch, k];  logits_host  host, fp32 [batch, k].
 *   out_sparse   device, fp32 [batch, V] (4-byte aligned), or NULL.
 *   batch, k, stream: as for vie_head_topk.
 *
 * Page-locked buffers (mapped into the device's address space) are used in
 * place: the kernels read page-locked queries straight from host memory, and
 * when idx_host and logits_host are both page-locked the kernel that merges
 * the top-k writes it there, with no copies.  Other buffers pass through
 * device buffers owned by the handle:
 * allocated by the first call that needs them (larger ones by a later call
 * that needs more, VIE_ERR_OOM if that fails), freed by vie_head_destroy.  The
 * call synchronises `stream` before it returns, so the host outputs are
 * ready; a device-side problem is reported by the next
 * vie_head_device_status, as for vie_head_topk.  At most one call per handle
 * at a time, as for vie_head_topk.
 */
vie_status vie_head_topk_host(vie_head *head, const float *h_host, int32_t batch, int32_t k,
                              int32_t *idx_host, float *logits_host, float *out_sparse,
                              vie_stream stream);

/*
 * vie_sample_topk - top-k sampling on the k candidates of each query
 * (Section 2: top-k sampling draws the next token from the k most probable
 * tokens; Section 3: top-p and min-p act as a second stage on the retrieved
 * logits; Section 4 samples with k = 50).  Per query, in fp32:
 *   p_j = softmax of logits[j] / temperature over the k candidates;
 *   top-p keeps the shortest prefix whose probability reaches top_p (at
 *   least one candidate); min-p keeps the candidates with p_j >= min_p * p_0;
 *   the kept set is the shorter prefix of the two;
 *   the token is the first kept candidate j whose cumulative probability
 *   exceeds u * (kept mass), where u in [0, 1) is the top 24 bits of the first
 *   output word of Philox4x32-10 (Salmon et al., SC 2011) at counter
 *   (step low, step high, query, 0) with key (seed low, seed high), times
 *   2^-24: the same (seed, step) gives the same draws, a new step new ones.
 *
 *   idx, logits  device, int32 / fp32 [batch, k]: candidates sorted by logit,
 *                best first, as vie_head_topk returns them (4-byte aligned).
 *   batch >= 1;  1 <= k <= VIE_K_MAX.
 *   temperature  > 0 and finite;  0 < top_p <= 1;  0 <= min_p <= 1.
 *   out_token    device, int32 [batch]: the drawn vocabulary index.
 *   out_prob     device, fp32 [batch]: its probability among the kept
 *                candidates.
 *   stream       the stream the work is enqueued on.
 *
 * The launch may start while the previous kernel on the stream finishes
 * (programmatic dependent launch); it reads idx and logits only after that
 * kernel has completed.  No allocation, no sync.
 */
vie_status vie_sample_topk(const int32_t *idx, const float *logits, int32_t batch, int32_t k,
                           float temperature, float top_p, float min_p, uint64_t seed,
                           uint64_t step, int32_t *out_token, float *out_prob, vie_stream stream);

/*
 * vie_head_topk_sample - vie_head_topk_sparse (or vie_head_topk when
 * out_sparse is NULL) followed by vie_sample_topk on its output: the whole
 * decode-step head with the next token drawn on the device.  Arguments as for
 * those two calls; k <= VIE_K_MAX.
 */
vie_status vie_head_topk_sample(vie_head *head, const float *h, int32_t batch, int32_t k,
                                float temperature, float top_p, float min_p, uint64_t seed,
                                uint64_t step, int32_t *out_idx, float *out_logits,
                                float *out_sparse, int32_t *out_token, float *out_prob,
                                vie_stream stream);

/*
 * vie_head_topk_many - the exact top-k of many hidden states, e.g. as the
 * ground truth against which an approximate head's Recall@k is measured
 * (Section 4.3 measures it over 20k hidden states).  The same results as
 * vie_head_topk on each block of up to VIE_BATCH_MAX consecutive states,
 * enqueued one block after the other on `stream`.
 *
 *   h          device, fp32 [n, d], row-major (4-byte aligned).
 *   n          1 <= n <= VIE_MANY_MAX;   k as for vie_head_topk.
 *   out_idx, out_logits  device, int32 / fp32 [n, k].
 *
 * Errors as for vie_head_topk; a block that fails to launch stops the call
 * (earlier blocks stay enqueued).
 */
vie_status vie_head_topk_many(vie_head *head, const float *h, int64_t n, int32_t k,
                              int32_t *out_idx, float *out_logits, vie_stream stream);

/*
 * vie_recall_hits - Recall@k bookkeeping (Section 4.3: recall is the share
 * of the exact head's top-k tokens that an approximate search also
 * retrieves).  For each query q:
 *   out_hits[q] = #{ j < k : exact[q, j] >= 0 and exact[q, j] is among
 *                            approx[q, 0], ..., approx[q, m - 1] },
 * the candidates taken as a set (a repeated candidate counts once) and
 * negative candidates as empty slots.  Recall@k over the n queries is
 * sum(out_hits) / (n k).  Integer work: the counts are exact.
 *
 *   exact     device, int32 [n, k]: the exact top-k indices (vie_head_topk,
 *             vie_head_topk_many).
 *   approx    device, int32 [n, m]: the approximate method's candidates.
 *   1 <= n <= VIE_RECALL_N_MAX;  1 <= k <= VIE_K_MAX;  1 <= m <= VIE_RECALL_M_MAX.
 *   out_hits  device, int32 [n].  All buffers 4-byte aligned.
 *
 * Asynchronous on `stream`, launched as a programmatic dependent of the
 * kernel before it (it reads its inputs only after that kernel completed).
 * Errors: VIE_ERR_INVALID_ARG (NULL, sizes, alignment), VIE_ERR_CUDA.
 */
vie_status vie_recall_hits(const int32_t *exact, int32_t k, const int32_t *approx, int32_t m,
                           int64_t n, int32_t *out_hits, vie_stream stream);

/*
 * vie_scatter_sparse_logits - the sparse full-vocabulary logit tensor of
 * Section 3: out[b, v] = -inf (bit pattern 0xFF800000) for every v, then
 * out[b, idx[b, j]] = logits[b, j] for j < k (values copied bit for bit).
 *
 *   idx     device, int32 [batch, k];   logits  device, fp32 [batch, k].
 *   batch   >= 1;  k >= 1;  V >= 1.
 *   out     device, fp32 [batch, V] (4-byte aligned).
 *
 * Indices within a row are expected to be distinct; if they repeat, which
 * value lands is unspecified.  An index outside [0, V) is skipped and sets
 * the device flag reported by vie_device_status.  No allocation, no sync.
 */
vie_status vie_scatter_sparse_logits(const int32_t *idx, const float *logits, int32_t batch,
                                     int32_t k, int64_t V, float *out, vie_stream stream);

/*
 * vie_head_topk_noalloc - vie_head_topk for callers that cannot allocate
 * device memory.  The paper has no counterpart: this is a deployment variant.
 *
 * Some callers are not allowed to call cudaMalloc at all: serving engines
 * whose device memory is carved out of one budget up front (a further
 * allocation could fail mid-request or take memory another model was
 * promised), and latency-critical decode loops that cannot afford the
 * implicit device synchronisation an allocation may bring.  A vie_head
 * allocates its padded weight copy and scratch in vie_head_create, so those
 * callers cannot make one.  This entry point takes the weights as they are
 * and keeps its scratch in a fixed array compiled into the library instead.
 *
 *   W_out       device memory of the current device (or managed memory),
 *               bf16 bit patterns, row-major [V, d], 16-byte aligned, d a
 *               multiple of 8 (rows must already be 16-byte vectors).
 *   V, d        1 <= V <= 2^31 - 2;  8 <= d <= VIE_D_MAX.
 *   h, batch, k, out_idx, out_logits, stream: as for vie_head_topk.
 *
 * Every batch runs on the streaming CUDA-core kernel, in query groups of up
 * to `cap` queries, one launch per group:
 *   cap = 8, halved (not below 1) while cap * d * 4 > 65536 or, for k > 64,
 *         while cap * c * 8 > 32768, where c = max(256, 2k rounded up to a
 *         multiple of 64) is the candidate buffer of one query.
 * Scratch: one 1 MiB array per device (every GPU that loads the library keeps
 * it until the process exits), of which the last 256 bytes hold counters, and
 * 80 KiB behind it for the bounds that the CTAs of a launch share.
 * A call needs
 *   8 * (round_up_even(slots * ctas * k) + slots * ctas * 8)
 * bytes of the rest, where ctas = min(SM count, ceil(V / 64), 1024) and
 * slots = the batch rounded up to a power of two, at most cap; larger
 * requests return VIE_ERR_UNSUPPORTED with the sizes in the message.  Groups
 * of one call run one after the other on `stream` and reuse the same lists
 * (the kernel re-arms its counters at the end of each launch).  The call clears
 * the counters and the bounds with cudaMemsetAsync on `stream` and allocates
 * nothing (no cudaMalloc, no cudaFree, no allocating library
 * routine).
 * The first call on a device looks up the array's device address with
 * cudaGetSymbolAddress (once per device); make that first call before any
 * stream capture.  Every call shares the one array, so calls whose work
 * overlaps on the GPU (other streams, other threads) race and corrupt each
 * other's results: serialise them.  Device-side problems set the flag read by
 * vie_device_status.  Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED,
 * VIE_ERR_CUDA.
 */
vie_status vie_head_topk_noalloc(const void *W_out, int64_t V, int32_t d, const float *h,
                                 int32_t batch, int32_t k, int32_t *out_idx, float *out_logits,
                                 vie_stream stream);

/*
 * Training and sampling around the head.  A small model that is trained on
 * what an exact head says (vie_head_topk_many: the teacher's top-k logits)
 * looks its tokens up in an embedding table (vie_embed), takes the loss of its
 * own full logits against the teacher's list and the gradient
 * (vie_distill_topk*), sums the table's gradient (vie_embed_grad), and draws
 * the tokens that it goes on with (vie_sample_logits).  These calls need no
 * handle.  Matrices are row-major with a row pitch in values ("ld", at least
 * the number of columns; rows need no alignment beyond a value's), bf16 or
 * fp32.  All arithmetic is fp32, each result rounded once to its type.  n = 0
 * is a valid call that does nothing (vie_embed_grad without accumulate still
 * clears its output).  No allocation and no host synchronisation happen inside
 * these calls, they may be captured in a graph, and calls on different streams
 * do not disturb each other (vie_embed_grad: with workspaces of their own).
 */

/*
 * vie_distill_topk - loss of a student's logits against a teacher's top-k
 * logits.  The teacher is the softmax of the sparse logit tensor (Section 3:
 * -inf except the k logits) over its k entries.  Per row, with z the
 * student's V logits, (i_j, t_j) the teacher's entries and T the temperature:
 *   p   = softmax(t / T) over the valid entries (i_j in [0, V), t_j > -inf);
 *   q   = softmax(z / T) over the vocabulary;
 *   loss = T^2 sum_j p_j (log p_j - log q[i_j])       (T^2 KL(p || q)).
 * Entries with an index outside [0, V) are empty slots, whatever their logit;
 * repeated indices add up.  A row without valid entries has loss 0 and stats
 * (0, 0), and its logits are not read.  Student logits of -inf have q = 0: the
 * loss is +inf where p > 0 there.  NaN or +inf logits give a NaN loss in
 * their row only.
 *
 *   logits      device, dtype [n, V], row pitch ld.
 *   n, V        0 <= n <= VIE_MANY_MAX;  1 <= V <= VIE_DISTILL_V_MAX.
 *   t_idx, t_logits  device, int32 / fp32 [n, k], in any order;
 *               1 <= k <= VIE_K_MAX.
 *   temperature > 0 and finite.  The loss is made of differences of fp32
 *               logarithms, times T^2: their roundings, some 2^-20 T^2, are what
 *               a large T leaves of a small loss.
 *   out_loss    device, fp32 [n].
 *   out_stats   device, fp32 [n, 2]: max z and sum_v exp((z_v - max z) / T), what
 *               vie_distill_topk_grad needs; may be NULL.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_distill_topk(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                            const int32_t *t_idx, const float *t_logits, int32_t k, float temperature,
                            float *out_loss, float *out_stats, vie_stream stream);

/*
 * vie_distill_topk_grad - the gradient of sum_i grad_loss[i] loss[i] with
 * respect to the student's logits:
 *   out_grad[i, v] = grad_loss[i] T (q_v - sum over j with i_j = v of p_j),
 * 0 in rows without valid entries.  Arguments as for vie_distill_topk, and
 *   stats       device, fp32 [n, 2]: out_stats of vie_distill_topk on the same
 *               logits and temperature.
 *   grad_loss   device, fp32 [n].
 *   out_grad    device, dtype [n, V], row pitch ld_grad; may be logits itself
 *               (with ld_grad = ld), but not overlap it in any other way.
 */
vie_status vie_distill_topk_grad(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                 const int32_t *t_idx, const float *t_logits, int32_t k, float temperature,
                                 const float *stats, const float *grad_loss, void *out_grad, int64_t ld_grad,
                                 vie_stream stream);

/*
 * vie_distill_topk_step - vie_distill_topk and vie_distill_topk_grad in one
 * call, for programs that know grad_loss beforehand.  Arguments as for those
 * two; out_stats may be NULL.
 */
vie_status vie_distill_topk_step(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                 const int32_t *t_idx, const float *t_logits, int32_t k, float temperature,
                                 const float *grad_loss, float *out_loss, float *out_stats, void *out_grad,
                                 int64_t ld_grad, vie_stream stream);

/*
 * vie_embed - rows of an embedding table, scaled (models with tied embeddings
 * look tokens up in the matrix that the head projects on):
 *   out[i, :] = scale * table[tokens[i], :].
 * Negative tokens are empty slots: a row of zeros.  A token of V or more gives
 * a row of zeros as well and sets the device flag that vie_device_status
 * reports.
 *
 *   table    device, dtype [V, d], row pitch ld;  1 <= V <= 2^31 - 2;
 *            1 <= d <= VIE_D_MAX.
 *   tokens   device, int32 [n];  0 <= n <= VIE_MANY_MAX.
 *   out      device, out_dtype [n, d], row pitch ld_out (fp32 rows are what
 *            vie_head_topk takes).
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_embed(const void *table, vie_dtype dtype, int64_t V, int32_t d, int64_t ld, const int32_t *tokens,
                     int64_t n, float scale, void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream);

/* Bytes of workspace that vie_embed_grad needs for n tokens (into *bytes, host). */
vie_status vie_embed_grad_workspace(int64_t n, int64_t V, int32_t d, int64_t *bytes);

/*
 * vie_embed_grad - the table's gradient:
 *   accumulate 0:  out[v, :]  = scale * sum over i with tokens[i] = v of grad[i, :]
 *                  (zeros for tokens that do not occur);
 *   otherwise:     out[v, :] += the same, for tokens that occur; the other rows
 *                  are not touched.  (In an fp32 table, results of magnitude
 *                  below 2^-126 become 0.)
 * The sum of a token's rows is fp32, in an order that depends on the tokens
 * alone: the same call gives the same bits.  Tokens outside [0, V) are left
 * out (V or more: the device flag, as in vie_embed).
 *
 *   tokens, n, V, d  as for vie_embed.
 *   grad     device, dtype [n, d], row pitch ld_grad.
 *   out      device, out_dtype [V, d], row pitch ld.
 *   workspace  device, 16-byte aligned, workspace_bytes bytes, at least what
 *            vie_embed_grad_workspace says; its contents need not be kept.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_embed_grad(const int32_t *tokens, int64_t n, const void *grad, vie_dtype dtype, int64_t ld_grad,
                          float scale, int64_t V, int32_t d, void *out, vie_dtype out_dtype, int64_t ld,
                          int32_t accumulate, void *workspace, int64_t workspace_bytes, vie_stream stream);

/*
 * vie_sample_logits - tokens drawn from full logits (dense ones, or the sparse
 * tensor of vie_head_topk_sparse after a program's own processors), each row
 * with its own settings and a uniform number that the caller gives.  Tokens
 * rank by (logit descending, index ascending).  Per row, with b = max z:
 *   w_v = floor(2^40 exp((z_v - b) (1 / T))), the products and the exp in fp32;
 *   top_k keeps the best top_k tokens (0 or less, or V and more: all), mass S;
 *   top_p keeps the shortest prefix of mass >= top_p S (1 or more: all);
 *   min_p keeps the tokens with w >= min_p 2^40 (0 or less: all);
 *   the shortest of these prefixes is kept, the best token always; mass M;
 *   the token is the first one whose running mass exceeds u M.
 * Weights are whole numbers, so their sums are exact in any order: a row's
 * token does not depend on how its work is split, nor on the rows beside it.
 * (A weight's last bits are those of the device's exp.)  u and top_p count in
 * steps of 2^-24 (u rounded down and held in [0, 1), top_p rounded up).  T of 0
 * (or anything not above 0) takes the best token.  Logits of -inf and NaN are
 * never drawn; a row that has no others gives token -1 and probability 0.
 * Logits of +inf share the whole mass.
 *
 *   logits   device, dtype [batch, V], row pitch ld;  0 <= batch <= VIE_MANY_MAX;
 *            1 <= V <= VIE_SAMPLE_V_MAX.
 *   u        device, fp32 [batch].
 *   temperature, top_k, top_p, min_p  device, fp32 / int32 / fp32 / fp32
 *            [batch]; each may be NULL (1, 0, 1, 0).
 *   out_token  device, int32 [batch].
 *   out_prob   device, fp32 [batch]: w / M of the token.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_sample_logits(const void *logits, vie_dtype dtype, int64_t batch, int64_t V, int64_t ld, const float *u,
                             const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                             int32_t *out_token, float *out_prob, vie_stream stream);

/*
 * vie_token_logprobs - log-probabilities of given tokens under full logits, e.g.
 * of tokens that vie_sample_logits has drawn.  Per row, z its V logits, t its
 * token, T the temperature:
 *   m = max z,  s = sum_v exp((z_v - m) / T),  logprob = (z_t - m) / T - log s.
 * Negative tokens are empty slots (a prompt's, padding): logprob 0 and stats
 * (0, 0), and the row's logits are not read.  A token of V or more is taken as
 * one and sets the device flag that vie_device_status reports.  A token whose
 * logit is -inf has logprob -inf, also where no logit is above it.  A row with a
 * NaN or +inf logit has logprob NaN, and no other row has.
 *
 *   logits      device, dtype [n, V], row pitch ld.
 *   n, V        0 <= n <= VIE_MANY_MAX;  1 <= V <= VIE_DISTILL_V_MAX.
 *   tokens      device, int32 [n].
 *   temperature > 0 and finite.
 *   out_logprob device, fp32 [n].
 *   out_stats   device, fp32 [n, 2]: m and s, what the gradients need; may be NULL.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_token_logprobs(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                              const int32_t *tokens, float temperature, float *out_logprob, float *out_stats,
                              vie_stream stream);

/*
 * vie_token_logprobs_grad - the gradient of sum_i grad_logprob[i] logprob[i] with
 * respect to the logits, q = softmax(z / T) (0 where no logit is above -inf):
 *   out_grad[i, v] = grad_logprob[i] ([v = t] - q_v) / T,
 * 0 in empty rows and in rows whose grad_logprob is 0, whose logits are not read.
 * Arguments as for vie_token_logprobs, and
 *   stats        device, fp32 [n, 2]: out_stats on the same logits and temperature.
 *   grad_logprob device, fp32 [n].
 *   out_grad     device, dtype [n, V], row pitch ld_grad; may be logits itself
 *                (with ld_grad = ld), but not overlap it in any other way.
 */
vie_status vie_token_logprobs_grad(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                   const int32_t *tokens, float temperature, const float *stats,
                                   const float *grad_logprob, void *out_grad, int64_t ld_grad, vie_stream stream);

/*
 * vie_policy_loss - clipped policy loss of drawn tokens with a KL term against a
 * reference policy.  Per row, lp as of vie_token_logprobs, A the advantage:
 *   r    = exp(lp - old_logprob)
 *   loss = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *          + kl_coef (exp(x) - x - 1),  x = ref_logprob - lp.
 * Empty rows (a token outside [0, V)) have loss, logprob and stats 0, and nothing
 * of them is read.  An advantage of 0 has no first term, whatever r; the second
 * is +inf where x is infinite.
 *
 *   logits, dtype, n, V, ld, tokens, temperature  as for vie_token_logprobs.
 *   old_logprob, advantage  device, fp32 [n]: of the policy that drew the tokens.
 *   ref_logprob device, fp32 [n]; may be NULL with a kl_coef of 0, which does not
 *               read it.
 *   clip_low    in [0, 1];  clip_high, kl_coef: finite, not negative.
 *   out_loss, out_logprob  device, fp32 [n].
 *   out_stats   as for vie_token_logprobs.  Results do not overlap the terms.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_policy_loss(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                           const int32_t *tokens, float temperature, const float *old_logprob, const float *advantage,
                           const float *ref_logprob, float clip_low, float clip_high, float kl_coef, float *out_loss,
                           float *out_logprob, float *out_stats, vie_stream stream);

/*
 * vie_policy_loss_grad - the gradient of sum_i grad_loss[i] loss[i] with respect
 * to the logits:
 *   slope = -A r where r A is the smaller one (also where both are the same),
 *           else 0, + kl_coef (1 - exp(x));
 *   out_grad[i, v] = grad_loss[i] slope ([v = t] - q_v) / T,
 * 0 in empty rows, where grad_loss is 0 and where slope is 0 (a clipped token
 * without a KL term); the logits of those are not read.  It is not finite where
 * slope is not.
 * Arguments as for vie_policy_loss, and
 *   logprob, stats  device, fp32 [n] and [n, 2]: out_logprob and out_stats of
 *               vie_policy_loss on the same logits and temperature.
 *   grad_loss   device, fp32 [n].
 *   out_grad    as for vie_token_logprobs_grad.
 */
vie_status vie_policy_loss_grad(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                const int32_t *tokens, float temperature, const float *old_logprob,
                                const float *advantage, const float *ref_logprob, float clip_low, float clip_high,
                                float kl_coef, const float *logprob, const float *stats, const float *grad_loss,
                                void *out_grad, int64_t ld_grad, vie_stream stream);

/*
 * vie_policy_loss_step - vie_policy_loss and vie_policy_loss_grad in one call, for
 * programs that know grad_loss beforehand.  Arguments as for those two;
 * out_stats may be NULL.
 */
vie_status vie_policy_loss_step(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                const int32_t *tokens, float temperature, const float *old_logprob,
                                const float *advantage, const float *ref_logprob, float clip_low, float clip_high,
                                float kl_coef, const float *grad_loss, float *out_loss, float *out_logprob,
                                float *out_stats, void *out_grad, int64_t ld_grad, vie_stream stream);

/*
 * vie_preference_loss - loss of preferred over rejected sequences from their
 * tokens' log-probabilities (vie_token_logprobs).  Sequence j holds the tokens
 * offsets[j] to offsets[j + 1] - 1 and may be empty; D_j is its sum of logprob -
 * ref_logprob.  Pair p is sequence 2p, the chosen one, and 2p + 1, the rejected:
 *   margin = beta (D_2p - D_2p+1)
 *   loss   = -(1 - label_smoothing) log sigmoid(margin) - label_smoothing log sigmoid(-margin).
 * Sums are fp32, in an order that depends on the sequence's place and length, n
 * and pairs alone: the same call gives the same bits.
 *
 *   logprob     device, fp32 [n];  0 <= n <= VIE_PREFERENCE_N_MAX.
 *   ref_logprob device, fp32 [n], or NULL (no reference: 0).
 *   offsets     device, int32 [2 pairs + 1], 0 <= offsets[0] <= offsets[1] ... <= n;
 *               tokens before the first and from the last on belong to no
 *               sequence.  Offsets that decrease or leave [0, n] are held inside
 *               (the results of their pairs are unspecified) and set the device
 *               flag that vie_device_status reports.
 *   pairs       0 <= pairs <= VIE_MANY_MAX.
 *   beta        finite;  label_smoothing in [0, 1].
 *   out_loss, out_margin  device, fp32 [pairs]; must not overlap the inputs.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_CUDA.
 */
vie_status vie_preference_loss(const float *logprob, const float *ref_logprob, int64_t n, const int32_t *offsets,
                               int64_t pairs, float beta, float label_smoothing, float *out_loss, float *out_margin,
                               vie_stream stream);

/*
 * vie_preference_loss_grad - the gradient of sum_p grad_loss[p] loss[p] with
 * respect to each token's logprob: beta grad_loss (label_smoothing -
 * sigmoid(-margin)) for the tokens of a chosen sequence, the negative for those
 * of a rejected one, 0 for the others (all n are written) and where grad_loss is 0.  It is what
 * vie_token_logprobs_grad takes as grad_logprob.
 *   margin      device, fp32 [pairs]: out_margin.
 *   grad_loss   device, fp32 [pairs].
 *   out_grad    device, fp32 [n]; must not overlap the inputs.
 * The other arguments as for vie_preference_loss.
 */
vie_status vie_preference_loss_grad(const float *margin, int64_t n, const int32_t *offsets, int64_t pairs, float beta,
                                    float label_smoothing, const float *grad_loss, float *out_grad,
                                    vie_stream stream);

/* vie_preference_loss and vie_preference_loss_grad in one call. */
vie_status vie_preference_loss_step(const float *logprob, const float *ref_logprob, int64_t n, const int32_t *offsets,
                                    int64_t pairs, float beta, float label_smoothing, const float *grad_loss,
                                    float *out_loss, float *out_margin, float *out_grad, vie_stream stream);

/*
 * Matrices in microscaled 4-bit floating point (e2m1), e.g. a head's rows: 4.5
 * bits per value.  Each row x of d values has a power of two s = 2^E, E the least
 * whole number (-126 at the least) with max |x| <= 2688 s; each block of 16 values
 * has a scale sigma = e4m3(max |x| over the block / (6 s)); a value's code is
 * e2m1(x / (s sigma)), at most 6 in magnitude (0 where sigma is 0), and stands for
 * code * sigma * s.  Roundings are to nearest, ties to even; what rounds to 0 has the
 * code 0 whatever its sign (never 8).  The same values in bf16 and in fp32 have the same
 * codes, scales and row scales.  A row that holds a
 * NaN or an infinity has s = NaN and codes of 0: all that is made of it is NaN.
 *   codes       uint8 [n, ceil(d / 32) * 16]: two codes to a byte, the even column
 *               in the low four bits; columns from d on are 0.
 *   scales      e4m3 [ceil(n / 128), ceil(d / 64), 32, 4, 4]: tiles of 128 rows by 4
 *               blocks; element [a, b, c] of a tile belongs to its row 32 b + a and
 *               block c.  Scales beyond the matrix are 0.
 *   row_scales  fp32 [n]: s.
 * vie_e2m1_bytes gives the sizes of codes and scales; both are 16-byte aligned.
 * 0 <= n <= VIE_E2M1_N_MAX;  1 <= d <= VIE_D_MAX.
 */
vie_status vie_e2m1_bytes(int64_t n, int32_t d, int64_t *code_bytes, int64_t *scale_bytes);

/*
 * vie_e2m1_quantize - rows to e2m1.
 *   x           device, dtype [n, d], row pitch ld.
 *   out_codes, out_scales, out_row_scales  device, as above; do not overlap x or each other.
 *   out_values  device, values_dtype [n, d], row pitch ld_values, or NULL: what the
 *               codes stand for, e.g. the weights that a training step computes
 *               with (exact in fp32, and in bf16 above its subnormal numbers); may
 *               be x itself (with its type and pitch), but not overlap it in any
 *               other way.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_e2m1_quantize(const void *x, vie_dtype dtype, int64_t n, int32_t d, int64_t ld, void *out_codes,
                             void *out_scales, float *out_row_scales, void *out_values, vie_dtype values_dtype,
                             int64_t ld_values, vie_stream stream);

/*
 * vie_e2m1_dequantize - out[i, j] = what the codes stand for (out_dtype [n, d], row pitch ld_out);
 * out does not overlap them.
 */
vie_status vie_e2m1_dequantize(const void *codes, const void *scales, const float *row_scales, int64_t n, int32_t d,
                               void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream);

/*
 * vie_e2m1_logits - full logits of a head whose rows are e2m1, for hidden states
 * that are e2m1 as well:
 *   out[i, v] = sum_j x[i, j] w[v, j],
 * products exact, sums fp32, rounded once to out_dtype (results below 2^-126 to fp32
 * before that), whatever the rows' powers of two.
 * vie_sample_logits draws from them, vie_token_logprobs scores them.
 *   x_*         device, n rows of d values;  0 <= n <= VIE_MANY_MAX.
 *   w_*         device, V rows of d values;  1 <= V <= VIE_E2M1_N_MAX.
 *   out         device, out_dtype [n, V], row pitch ld_out; does not overlap x_* and w_*.
 *
 * Errors: VIE_ERR_INVALID_ARG, VIE_ERR_UNSUPPORTED (dtype), VIE_ERR_CUDA.
 */
vie_status vie_e2m1_logits(const void *x_codes, const void *x_scales, const float *x_row_scales, int64_t n,
                           const void *w_codes, const void *w_scales, const float *w_row_scales, int64_t V, int32_t d,
                           void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream);

/*
 * vie_e2m1_quantize_logits - vie_e2m1_quantize of x (device, dtype [n, d], row pitch
 * ld) into x_* and vie_e2m1_logits of those, in one call: the head's rows are
 * fetched while x is quantised.  x_* do not overlap w_* or x.  Arguments and errors as
 * for those two.
 */
vie_status vie_e2m1_quantize_logits(const void *x, vie_dtype dtype, int64_t n, int64_t ld, void *x_codes,
                                    void *x_scales, float *x_row_scales, const void *w_codes, const void *w_scales,
                                    const float *w_row_scales, int64_t V, int32_t d, void *out, vie_dtype out_dtype,
                                    int64_t ld_out, vie_stream stream);

/*
 * vie_device_status - synchronises `stream`, then reads and clears the
 * library's device-side flag word of the current device.  Returns VIE_OK when
 * no kernel recorded a problem, VIE_ERR_DEVICE otherwise (vie_last_error()
 * names the problem), VIE_ERR_CUDA if the synchronisation itself failed.
 */
vie_status vie_device_status(vie_stream stream);

/* Same as vie_device_status for the handle's device, and also re-arms the
 * handle's scratch counters after a device-side problem. */
vie_status vie_head_device_status(vie_head *head, vie_stream stream);

/* Message for the last failing call on this thread ("" if none). */
const char *vie_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* VIE_HEAD_H */
