// vie_distill.cu - distillation from a teacher's top logits: the loss of a
// student's full logits against the top-k logits of an exact head, and its
// gradient (paper, Section 3: the sparse logit tensor, -inf except k logits,
// is what a head hands on; its softmax is the teacher here).
//
// Per row, z the V student logits, (i_j, t_j) the teacher's k entries, those
// with i_j in [0, V) and t_j > -inf valid, T the temperature:
//   p_j  = exp((t_j - max t) / T) / sum over the valid entries
//   q_v  = exp((z_v - m) / T) / s,   m = max z,  s = sum_v exp((z_v - m) / T)
//   loss = T^2 sum_j p_j (log p_j - log q_{i_j})
//   d loss / d z_v = T (q_v - sum over i_j = v of p_j)
// A row without valid entries has loss 0 and gradient 0 and its logits are
// not read.  All arithmetic is fp32; a bf16 gradient is rounded once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"
#include "vie_row_softmax.cuh"

namespace vie {

struct DistillParams {
    const void *logits;
    const int32_t *t_idx;
    const float *t;
    const float *stats_in;   // backward alone: m and s of each row
    const float *grad_loss;  // backward
    float *loss;             // forward
    float *stats_out;        // forward, or NULL
    void *grad;              // backward
    int64_t ld, ld_grad;
    int V, k;
    float T;
    uint32_t *flag;
};

// Vectors in flight per thread: eight, but for loss and gradient on bf16 logits,
// where a thread's 64 registers hold six (151936 x 4096: 450 us; 497 with eight).
template <typename T, bool FWD, bool BWD>
constexpr int kUnroll = FWD && BWD && sizeof(T) == 2 ? 6 : 8;
constexpr int kTeacherEntries = 4;  // of a teacher, per thread of the warps that deal with it
static_assert(VIE_K_MAX <= 32 * kTeacherEntries * kRowWarps, "warps for all entries");

struct DistillSmem : RowSmem {
    float3 teacher[kRowWarps];  // per teacher warp: max t, the sum of exp((t - max t) / T), part of the loss
    int repeats;
};

// Slots of the hash table of a slice's entries: a power of two, at least
// twice the entries.
__host__ __device__ inline int seen_slots(int k) {
    int slots = 64;
    while (slots < 2 * k) slots <<= 1;
    return slots;
}

// The teacher's entries of a row in shared memory, and the warps of the CTA that
// deal with them: `me` is a thread's number among theirs, below 0 in the
// others, which call nothing but mine().
struct Teacher {
    int32_t *idx;   // -1 where the entry does not count
    float *p;       // its logit, then the softmax
    float *z;       // the student's logit there
    int32_t *seen;  // hash table of the slice's entries
    int k, warps, me;
    bool repeats;

    __device__ __forceinline__ Teacher(int k_, int warps_, int me_, int32_t *list, float *z_, int32_t *seen_)
        : idx(list), p(reinterpret_cast<float *>(list + k_)), z(z_), seen(seen_), k(k_), warps(warps_), me(me_),
          repeats(false) {}
    __device__ __forceinline__ bool mine() const { return me >= 0; }
    __device__ __forceinline__ int step() const { return 32 * warps; }
    __device__ __forceinline__ void barrier() const {
        if (warps > 1) named_barrier_sync(1, 32 * warps);
        else __syncwarp();
    }
    // Entry j as it was read: whether it counts.
    __device__ __forceinline__ bool validate(const DistillParams &a, int j) const {
        if (idx[j] >= 0 && idx[j] < a.V && p[j] != -INFINITY) return true;
        idx[j] = -1;
        return false;
    }
    // The student's logits at the entries from value e0 (which may be below 0) to
    // e1 of the row: read into registers, which nothing waits for, and kept in z.
    template <typename T>
    __device__ __forceinline__ void read_logits(const T *row, int e0, int e1, T (&raw)[kTeacherEntries]) const {
#pragma unroll
        for (int u = 0; u < kTeacherEntries; ++u) {
            const int j = me + u * step(), i = j < k ? idx[j] : -1;
            if (i >= max(e0, 0) && i < e1) raw[u] = row[i];
        }
    }
    template <typename T>
    __device__ __forceinline__ void keep_logits(const T (&raw)[kTeacherEntries]) const {
#pragma unroll
        for (int u = 0; u < kTeacherEntries; ++u)
            if (me + u * step() < k) z[me + u * step()] = load_value(&raw[u]);
    }
    // p: from logits to the softmax.
    __device__ __forceinline__ void softmax(DistillSmem &sm, float inv_T) const {
        const int warp = me >> 5, lane = me & 31;
        float tm = -INFINITY, ts = 0.0f;
#pragma unroll 4
        for (int j = me; j < k; j += step())
            if (idx[j] >= 0) tm = fmaxf(tm, p[j]);
        tm = warp_max(tm);
        if (warps > 1) {
            if (lane == 0) sm.teacher[warp].x = tm;
            barrier();
            for (int w = 0; w < warps; ++w) tm = fmaxf(tm, sm.teacher[w].x);
        }
#pragma unroll 4
        for (int j = me; j < k; j += step()) {
            const float e = idx[j] >= 0 ? expf((p[j] - tm) * inv_T) : 0.0f;
            p[j] = e;
            ts += e;
        }
        ts = warp_sum(ts);
        if (warps > 1) {
            if (lane == 0) sm.teacher[warp].y = ts;
            barrier();
            ts = 0.0f;
            for (int w = 0; w < warps; ++w) ts += sm.teacher[w].y;
        }
        const float inv = 1.0f / ts;
#pragma unroll 4
        for (int j = me; j < k; j += step()) p[j] *= inv;
        barrier();
    }
    // Indices seldom repeat: a hash table finds out whether those of this slice do.
    __device__ __forceinline__ void find_repeats(DistillSmem &sm, int e0, int e1) {
        const int slots = seen_slots(k);
        for (int i = me; i < slots; i += step()) seen[i] = -1;
        if (me == 0) sm.repeats = 0;
        barrier();
        for (int j = me; j < k; j += step()) {
            const int32_t i = idx[j];
            if (i < e0 || i >= e1 || i < 0) continue;
            uint32_t h = (static_cast<uint32_t>(i) * 0x9E3779B1u) >> 16 & (slots - 1);
            while (true) {  // ends: at most half the slots are taken
                const int32_t old = atomicCAS(&seen[h], -1, i);
                if (old == i) sm.repeats = 1;
                if (old == -1 || old == i) break;
                h = (h + 1) & (slots - 1);
            }
        }
        barrier();
        repeats = sm.repeats != 0;
    }
    // T^2 sum p (log p - log q) over all entries, in all of the warps; m, s: the student's statistics.
    // One T is taken into the sum, log q = (z - m) / T - log s, and the other if it
    // is below 1: neither T^2 nor a difference of logits over T need be within fp32
    // (masks of the type's lowest value), and +inf stays +inf.
    __device__ __forceinline__ float loss(DistillSmem &sm, float T, float m, float s) const {
        float cost = 0.0f;
        const float log_s = logf(s), m0 = finite_max(m), inside = fminf(T, 1.0f);
#pragma unroll 4
        for (int j = me; j < k; j += step())
            if (p[j] != 0.0f) cost += p[j] * (inside * (T * (logf(p[j]) + log_s) - (z[j] - m0)));
        cost = warp_sum(cost);
        if (warps > 1) {
            if ((me & 31) == 0) sm.teacher[me >> 5].z = cost;
            barrier();
            cost = 0.0f;
            for (int w = 0; w < warps; ++w) cost += sm.teacher[w].z;
        }
        return s == 0.0f ? INFINITY : fmaxf(T, 1.0f) * cost;  // (no softmax: no logit above -inf)
    }
    // q - p over what the slice's loop has written at its entries; the first
    // entry of an index takes off the sum of all.
    template <typename T>
    __device__ __forceinline__ void store_gradient(T *g, int e0, int e1, const Exponent &e, float cg, float inv) const {
        for (int j = me; j < k; j += step()) {
            const int32_t i = idx[j];
            if (i < e0 || i >= e1 || i < 0) continue;
            float take = p[j];
            bool leads = true;
            if (repeats) {
                take = 0.0f;
                for (int x = 0; x < k; ++x)
                    if (idx[x] == i) {
                        leads &= x >= j;
                        take += p[x];
                    }
            }
            if (leads) store_value(g + i, cg * (e(z[j]) * inv - take));
        }
    }
};

__device__ __forceinline__ void write_row(const DistillParams &a, int64_t row, float loss, float m, float s) {
    a.loss[row] = loss;
    if (a.stats_out != nullptr) {
        a.stats_out[2 * row] = m;
        a.stats_out[2 * row + 1] = s;
    }
}

// Loss and statistics (FWD) or the gradient (BWD) or both.
//
// A row is a cluster's, a slice of it a CTA's; each thread keeps kUnroll 16-byte
// vectors in flight, its running maximum and sum, and the slices' (m, s) go to
// all CTAs of the row by asynchronous stores that count on their mbarriers (a
// cluster barrier with release would wait for the gradients written before).
// The teacher's softmax is worked out meanwhile.  For both, the slice is read
// again: from L2, as long as the slices in progress, four CTAs per SM of them,
// fit it.  They are 80 KB or less each up to rows of 640 KB, 50 MB in all, and an
// eighth of the row beyond: 80 MB at 262144 fp32 values (0.83 below); at a million
// 300 MB, which do not fit (0.61).
// (Keeping slices in shared memory measured the same at 50 entries per row, and
// twice the time at 1000, where too few threads were left for the teacher.)
//
// Bound by bytes.  Measured on bf16 logits, 50 to 64 entries per row, and as a
// share of the time that a copy of the bytes read and written once would take:
//   loss and statistics  262144 x 2048: 151 us (0.94)
//   gradient             128256 x 2048: 154 us (0.95)
//   both                 151936 x 4096: 450 us (0.78), 262144 x 1024: 196 (0.77), 32000 x 4096:
//                        104 (0.71); fp32 128256 x 1024: 173 (0.85), 262144 x 1024: 363 (0.83),
//                        1000003 x 128: 235 (0.61)
// What is left in the last: a row's exchange and its entries, which the CTAs'
// other rows hide only in part (61 % of issue slots used, DRAM 55 % busy).
// Dynamic shared memory: the teacher's entries (indices, logits, the student's
// logits there), the hash table (BWD).
template <typename T, bool FWD, bool BWD>
__global__ void __launch_bounds__(kRowThreads, 4) distill_kernel(const DistillParams a, int log2_slices) {
    constexpr int NT = kRowThreads, U = kUnroll<T, FWD, BWD>;
    extern __shared__ __align__(16) unsigned char distill_smem[];
    __shared__ DistillSmem sm;
    int32_t *const list = reinterpret_cast<int32_t *>(distill_smem);
    const int tid = threadIdx.x, warp = tid >> 5;
    // the first warps deal with the teacher, besides their part of the row
    const int t_warps = (a.k + 32 * kTeacherEntries - 1) / (32 * kTeacherEntries);
    Teacher tea(a.k, t_warps, tid < 32 * t_warps ? tid : -1, list, reinterpret_cast<float *>(list + 2 * a.k),
                list + 3 * a.k);
    const int slices = 1 << log2_slices, rank = blockIdx.x & (slices - 1);
    const int64_t row = blockIdx.x >> log2_slices;
    if (FWD) {
        if (tid == 0) sm.init();
        __syncwarp();
        cluster_arrive_relaxed();  // all CTAs of the cluster run and wait, before their memory is written
    }
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one

    bool any = false;
    for (int j = tid; j < a.k; j += NT) {
        tea.idx[j] = a.t_idx[row * a.k + j], tea.p[j] = a.t[row * a.k + j];
        any |= tea.validate(a, j);
    }
    const bool has = __syncthreads_or(any);
    const Slice<T> sl(static_cast<const T *>(a.logits) + row * a.ld, a.V, log2_slices, rank);
    const GradSlice<T> out(static_cast<T *>(a.grad) + row * a.ld_grad, sl);
    if (FWD) cluster_wait();
    if (!has) {
        if (BWD) clear_gradient(sl, out);
        if (FWD && rank == 0 && tid == 0) write_row(a, row, 0.0f, 0.0f, 0.0f);
        return;
    }
    const float inv_T = fminf(1.0f / a.T, 3.4e38f);
    const float c = exponent_factor(a.T);
    // The entries' logits, before a gradient may overwrite them; the loss (rank
    // 0) needs those of the whole row.
    const bool whole = FWD && rank == 0;
    T z_entries[kTeacherEntries] = {};
    const bool keeps = tea.mine() && (BWD || whole);
    if (keeps) tea.read_logits(sl.z, whole ? 0 : sl.e0, whole ? a.V : sl.e1, z_entries);
    float m, s;
    if (FWD) {
        slice_statistics<T, U, BWD>(sl, c, sm);
        if (keeps) tea.keep_logits(z_entries);
        __syncthreads();
        if (warp == 0) send_partial(sm, slices, rank, c);
        if (keeps) tea.softmax(sm, inv_T);  // while the partials travel
        join_partials(a.flag, sm, slices, c, &m, &s);
    } else {
        m = a.stats_in[2 * row];
        s = a.stats_in[2 * row + 1];
        if (keeps) tea.keep_logits(z_entries);
        __syncthreads();  // (grad may be logits: the entries' logits are read before it is written)
    }
    if (BWD) {
        const Exponent e{finite_max(m), c};
        const float cg = a.T * a.grad_loss[row], inv = s == 0.0f ? 0.0f : 1.0f / s, coef = cg * inv;
        store_softmax<T, U>(sl, out, e, coef);
        if (keeps) {
            if (!FWD) tea.softmax(sm, inv_T);
            tea.find_repeats(sm, sl.e0, sl.e1);
        }
        __syncthreads();
        if (keeps) tea.store_gradient(out.g, sl.e0, sl.e1, e, cg, inv);
    }
    if (FWD && rank == 0 && tea.mine()) {
        const float loss = tea.loss(sm, a.T, m, s);
        if (tid == 0) write_row(a, row, loss, m, s);
    }
}

template <typename T, bool FWD, bool BWD>
static cudaError_t start_distill(const DistillParams &p, int64_t n, int slices, cudaStream_t s) {
    auto kernel = distill_kernel<T, FWD, BWD>;
    const size_t smem = 12 * static_cast<size_t>(p.k) + (BWD ? 4 * seen_slots(p.k) : 0);  // 20 KB at most
    if (FWD && slices > kSlices) {
        static PerDevice prepared;
        const cudaError_t e =
            prepared.once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); });
        if (e != cudaSuccess) return e;
    }
    RowLaunch l(n * slices, FWD ? slices : 0, smem, s);
    return cudaLaunchKernelEx(&l.cfg, kernel, p, log2_of(slices));
}

// Bytes of a slice that one CTA takes, at most.  Gradient alone (128256 x 2048):
// 155 us in slices of 128 KB, 163 of 256; each CTA reads the teacher's entries.
constexpr int64_t kSliceBytes = 128 * 1024;
// Loss and gradient, while a cluster can have more CTAs (fp32 128256 x 1024: 174 us in
// slices of 64 KB, 186 of 128; bf16 151936 x 4096: 450 in slices of 76 KB, 556 of 38).
constexpr int64_t kSliceStep = 80 * 1024;

// CTAs per row of n rows of this many bytes.
static int slices_of(bool fwd, bool bwd, int64_t bytes, int64_t n) {
    int slices = 1;
    if (!fwd) {  // no partials to join
        while (bytes / slices > kSliceBytes && n * slices < (1 << 30)) slices *= 2;
        return slices;
    }
    if (bwd)
        while (slices < kSlices && bytes / slices > kSliceStep) slices *= 2;
    // enough CTAs for the chip, of 32 KB of the row or more
    while (slices < (n <= kFewRows ? kMaxSlices : kSlices) && n * slices < 1024 && bytes / slices > 32768) slices *= 2;
    return slices;
}

template <bool FWD, bool BWD>
static cudaError_t launch_distill(const DistillParams &p, vie_dtype dtype, int64_t n, cudaStream_t s) {
    const int slices = slices_of(FWD, BWD, static_cast<int64_t>(p.V) * dtype_size(dtype), n);
    return dtype == VIE_DTYPE_BF16 ? start_distill<__nv_bfloat16, FWD, BWD>(p, n, slices, s)
                                   : start_distill<float, FWD, BWD>(p, n, slices, s);
}

static vie_status check_distill(const char *fn, const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                const int32_t *t_idx, const float *t, int32_t k, float T) {
    if (n < 0 || n > VIE_MANY_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_MANY_MAX);
    if (V < 1 || V > VIE_DISTILL_V_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: V=%lld outside [1, %d]", fn, static_cast<long long>(V), VIE_DISTILL_V_MAX);
    if (k < 1 || k > VIE_K_MAX) return fail(VIE_ERR_INVALID_ARG, "%s: k=%d outside [1, %d]", fn, k, VIE_K_MAX);
    if (!(T > 0.0f) || std::isinf(T))
        return fail(VIE_ERR_INVALID_ARG, "%s: temperature=%g must be positive and finite", fn, static_cast<double>(T));
    if (n > 0 && (t_idx == nullptr || t == nullptr)) return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(t_idx, 4) || !aligned_to(t, 4))
        return fail(VIE_ERR_INVALID_ARG, "%s: buffers must be 4-byte aligned", fn);
    return check_matrix(fn, "logits", logits, dtype, n, V, ld);
}

static vie_status check_floats(const char *fn, int64_t n, const float *p, bool may_be_null) {
    if (p == nullptr && n > 0 && !may_be_null) return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(p, 4)) return fail(VIE_ERR_INVALID_ARG, "%s: buffers must be 4-byte aligned", fn);
    return VIE_OK;
}

}  // namespace vie

using namespace vie;

extern "C" {

vie_status vie_distill_topk(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                            const int32_t *t_idx, const float *t_logits, int32_t k, float temperature,
                            float *out_loss, float *out_stats, vie_stream stream) {
    const char *fn = "vie_distill_topk";
    vie_status st = check_distill(fn, logits, dtype, n, V, ld, t_idx, t_logits, k, temperature);
    if (st == VIE_OK) st = check_floats(fn, n, out_loss, false);
    if (st == VIE_OK) st = check_floats(fn, n, out_stats, true);
    if (st != VIE_OK || n == 0) return st;
    DistillParams p = {};
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    p.logits = logits, p.t_idx = t_idx, p.t = t_logits, p.loss = out_loss, p.stats_out = out_stats;
    p.ld = ld, p.V = static_cast<int>(V), p.k = k, p.T = temperature;
    e = launch_distill<true, false>(p, dtype, n, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_distill_topk_grad(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                 const int32_t *t_idx, const float *t_logits, int32_t k, float temperature,
                                 const float *stats, const float *grad_loss, void *out_grad, int64_t ld_grad,
                                 vie_stream stream) {
    const char *fn = "vie_distill_topk_grad";
    vie_status st = check_distill(fn, logits, dtype, n, V, ld, t_idx, t_logits, k, temperature);
    if (st == VIE_OK) st = check_floats(fn, n, stats, false);
    if (st == VIE_OK) st = check_floats(fn, n, grad_loss, false);
    if (st == VIE_OK) st = check_matrix(fn, "out_grad", out_grad, dtype, n, V, ld_grad);
    if (st != VIE_OK || n == 0) return st;
    DistillParams p = {};
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    p.logits = logits, p.t_idx = t_idx, p.t = t_logits, p.stats_in = stats, p.grad_loss = grad_loss;
    p.grad = out_grad, p.ld = ld, p.ld_grad = ld_grad, p.V = static_cast<int>(V), p.k = k, p.T = temperature;
    e = launch_distill<false, true>(p, dtype, n, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_distill_topk_step(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                 const int32_t *t_idx, const float *t_logits, int32_t k, float temperature,
                                 const float *grad_loss, float *out_loss, float *out_stats, void *out_grad,
                                 int64_t ld_grad, vie_stream stream) {
    const char *fn = "vie_distill_topk_step";
    vie_status st = check_distill(fn, logits, dtype, n, V, ld, t_idx, t_logits, k, temperature);
    if (st == VIE_OK) st = check_floats(fn, n, grad_loss, false);
    if (st == VIE_OK) st = check_floats(fn, n, out_loss, false);
    if (st == VIE_OK) st = check_floats(fn, n, out_stats, true);
    if (st == VIE_OK) st = check_matrix(fn, "out_grad", out_grad, dtype, n, V, ld_grad);
    if (st != VIE_OK || n == 0) return st;
    DistillParams p = {};
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    p.logits = logits, p.t_idx = t_idx, p.t = t_logits, p.grad_loss = grad_loss, p.loss = out_loss;
    p.stats_out = out_stats, p.grad = out_grad, p.ld = ld, p.ld_grad = ld_grad;
    p.V = static_cast<int>(V), p.k = k, p.T = temperature;
    e = launch_distill<true, true>(p, dtype, n, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

}  // extern "C"
