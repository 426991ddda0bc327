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
};

constexpr int kDistillThreads = 256;

// The teacher's row in shared memory: p (0 for entries that do not count) and
// the entropy part sum p log p in every thread; false if no entry is valid.
struct Teacher {
    float p[VIE_K_MAX];
    int32_t idx[VIE_K_MAX];  // -1: not valid
    float scratch[32];
};

__device__ __forceinline__ bool load_teacher(Teacher &tea, const DistillParams &a, int64_t row, float *plogp) {
    float mx = -INFINITY;
    bool any = false;
    for (int j = threadIdx.x; j < a.k; j += kDistillThreads) {
        const int32_t i = a.t_idx[row * a.k + j];
        const float t = a.t[row * a.k + j];
        const bool valid = i >= 0 && i < a.V && t != -INFINITY;
        tea.idx[j] = valid ? i : -1;
        tea.p[j] = t;
        any |= valid;
        if (valid) mx = fmaxf(mx, t);
    }
    if (!__syncthreads_or(any)) return false;
    mx = block_max<kDistillThreads>(mx, tea.scratch);
    float sum = 0.0f;
    for (int j = threadIdx.x; j < a.k; j += kDistillThreads)
        if (tea.idx[j] >= 0) sum += expf((tea.p[j] - mx) / a.T);
    sum = block_sum<kDistillThreads>(sum, tea.scratch);
    float ent = 0.0f;
    for (int j = threadIdx.x; j < a.k; j += kDistillThreads) {
        float p = 0.0f;
        if (tea.idx[j] >= 0) {
            const float x = (tea.p[j] - mx) / a.T;
            p = expf(x) / sum;
            if (p != 0.0f) ent += p * (x - logf(sum));
        }
        tea.p[j] = p;
    }
    *plogp = block_sum<kDistillThreads>(ent, tea.scratch);
    return true;
}

// One CTA per row.
template <typename T, bool FWD, bool BWD>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams a) {
    __shared__ Teacher tea;
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits) + row * a.ld;
    T *g = static_cast<T *>(a.grad) + row * a.ld_grad;
    float plogp;
    if (!load_teacher(tea, a, row, &plogp)) {
        if (FWD && threadIdx.x == 0) {
            a.loss[row] = 0.0f;
            if (a.stats_out != nullptr) a.stats_out[2 * row] = a.stats_out[2 * row + 1] = 0.0f;
        }
        if (BWD)
            for (int v = threadIdx.x; v < a.V; v += kDistillThreads) store_value(g + v, 0.0f);
        return;
    }
    float m = -INFINITY, s = 0.0f;
    if (FWD) {
        for (int v = threadIdx.x; v < a.V; v += kDistillThreads) m = fmaxf(m, load_value(z + v));
        m = block_max<kDistillThreads>(m, tea.scratch);
    } else {
        m = a.stats_in[2 * row];
        s = a.stats_in[2 * row + 1];
    }
    const float m0 = m == -INFINITY ? 0.0f : m;  // no finite logit: every exp is 0
    if (FWD) {
        for (int v = threadIdx.x; v < a.V; v += kDistillThreads) s += expf((load_value(z + v) - m0) / a.T);
        s = block_sum<kDistillThreads>(s, tea.scratch);
        float cross = 0.0f;
        for (int j = threadIdx.x; j < a.k; j += kDistillThreads)
            if (tea.p[j] != 0.0f) {
                const float logq = s == 0.0f ? -INFINITY : (load_value(z + tea.idx[j]) - m0) / a.T - logf(s);
                cross += tea.p[j] * logq;
            }
        cross = block_sum<kDistillThreads>(cross, tea.scratch);
        if (threadIdx.x == 0) {
            a.loss[row] = a.T * a.T * (plogp - cross);
            if (a.stats_out != nullptr) {
                a.stats_out[2 * row] = m;
                a.stats_out[2 * row + 1] = s;
            }
        }
    }
    if (BWD) {
        const float c = a.T * a.grad_loss[row], inv = s == 0.0f ? 0.0f : 1.0f / s;
        // each entry's gradient, before the logits may be overwritten (grad
        // may be logits): its first position takes the sum of its repeats
        float own[VIE_K_MAX / kDistillThreads];
#pragma unroll
        for (int u = 0; u < VIE_K_MAX / kDistillThreads; ++u) {
            const int j = threadIdx.x + u * kDistillThreads;
            if (j < a.k && tea.idx[j] >= 0)
                own[u] = expf((load_value(z + tea.idx[j]) - m0) / a.T) * inv;
        }
        __syncthreads();
        for (int v = threadIdx.x; v < a.V; v += kDistillThreads)
            store_value(g + v, c * (expf((load_value(z + v) - m0) / a.T) * inv));
        __syncthreads();
#pragma unroll
        for (int u = 0; u < VIE_K_MAX / kDistillThreads; ++u) {
            const int j = threadIdx.x + u * kDistillThreads;
            if (j >= a.k || tea.idx[j] < 0) continue;
            bool first = true;
            float p = 0.0f;
            for (int i = 0; i < a.k; ++i)
                if (tea.idx[i] == tea.idx[j]) {
                    first &= i >= j;
                    p += tea.p[i];
                }
            if (first) store_value(g + tea.idx[j], c * (own[u] - p));
        }
    }
}

template <bool FWD, bool BWD>
cudaError_t launch_distill(const DistillParams &p, vie_dtype dtype, int64_t n, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(n);
    if (dtype == VIE_DTYPE_BF16)
        distill_kernel<__nv_bfloat16, FWD, BWD><<<grid, kDistillThreads, 0, s>>>(p);
    else
        distill_kernel<float, FWD, BWD><<<grid, kDistillThreads, 0, s>>>(p);
    return cudaGetLastError();
}

static vie_status check_distill(const char *fn, const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                const int32_t *t_idx, const float *t, int32_t k, float T) {
    if (n < 0 || n > VIE_MANY_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_MANY_MAX);
    if (V < 1 || V > INT32_MAX - 1)
        return fail(VIE_ERR_INVALID_ARG, "%s: V=%lld outside [1, 2^31-2]", fn, static_cast<long long>(V));
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
    p.logits = logits, p.t_idx = t_idx, p.t = t_logits, p.loss = out_loss, p.stats_out = out_stats;
    p.ld = ld, p.V = static_cast<int>(V), p.k = k, p.T = temperature;
    const cudaError_t e = launch_distill<true, false>(p, dtype, n, static_cast<cudaStream_t>(stream));
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
    p.logits = logits, p.t_idx = t_idx, p.t = t_logits, p.stats_in = stats, p.grad_loss = grad_loss;
    p.grad = out_grad, p.ld = ld, p.ld_grad = ld_grad, p.V = static_cast<int>(V), p.k = k, p.T = temperature;
    const cudaError_t e = launch_distill<false, true>(p, dtype, n, static_cast<cudaStream_t>(stream));
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
    p.logits = logits, p.t_idx = t_idx, p.t = t_logits, p.grad_loss = grad_loss, p.loss = out_loss;
    p.stats_out = out_stats, p.grad = out_grad, p.ld = ld, p.ld_grad = ld_grad;
    p.V = static_cast<int>(V), p.k = k, p.T = temperature;
    const cudaError_t e = launch_distill<true, true>(p, dtype, n, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

}  // extern "C"
