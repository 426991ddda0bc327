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
    uint32_t *flag;
};

// A row is cut into 16-byte vectors at 16-byte addresses; its first and last
// one may reach over its ends.  The `slices` CTAs of a row take consecutive
// runs of vectors.
constexpr int kDistillThreads = 256;
constexpr int kDistillEntries = VIE_K_MAX / kDistillThreads;  // teacher entries per thread
constexpr int kDistillUnroll = 8;                             // vectors in flight per thread
constexpr int kMaxSlices = 16;

// What a CTA knows of its slice: the maximum m, the sum of exp((z - m) / T),
// and over the teacher's entries in it the sums of p (z - m) / T and of p.
struct Partial {
    float m, s, cross, p;
};

// exp2((z - m) c) = exp((z - m) / T).  The difference comes first: the type's
// lowest value is a usual mask, and z c - m c overflows there.
struct Exponent {
    float m, c;
    __device__ __forceinline__ float operator()(float z) const { return exp2_approx((z - m) * c); }
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

// Two partials as one, relative to the larger maximum.
__device__ __forceinline__ Partial join(const Partial &a, const Partial &b, float c, float inv_T) {
    Partial r;
    r.m = fmaxf(a.m, b.m);
    const float m0 = finite_max(r.m);
    const float da = finite_max(a.m) - m0, db = finite_max(b.m) - m0;
    r.s = (a.s != 0.0f ? a.s * exp2_approx(da * c) : 0.0f) + (b.s != 0.0f ? b.s * exp2_approx(db * c) : 0.0f);
    r.p = a.p + b.p;
    r.cross = (a.p != 0.0f ? a.cross + a.p * (da * inv_T) : 0.0f) + (b.p != 0.0f ? b.cross + b.p * (db * inv_T) : 0.0f);
    return r;
}

struct DistillSmem {
    float4 gathered[kMaxSlices];  // the row's partials, by slice
    float4 warp_part[kDistillThreads / 32];
    float scratch[32];
    float entropy[kDistillThreads / 32];
    uint64_t bar;
    int abort;
};

// Slots of the hash table of a slice's entries: a power of two, at least
// twice the entries.
__host__ __device__ inline int seen_slots(int k) {
    int slots = 64;
    while (slots < 2 * k) slots <<= 1;
    return slots;
}

// FWD: loss and statistics; BWD: the gradient.  RESIDENT: the CTA's slice stays
// in shared memory between the two, so the logits are read once; otherwise
// each of them reads the slice again.
// Dynamic shared memory: the slice (RESIDENT); from entries_at on (BWD) p and
// the indices of the teacher's entries and the hash table.
template <typename T, bool FWD, bool BWD, bool RESIDENT>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams a, int slices, uint32_t entries_at) {
    constexpr int kVec = Vec16<T>::kVec;
    extern __shared__ __align__(16) unsigned char distill_slice[];
    __shared__ DistillSmem sm;
    float *const sp = reinterpret_cast<float *>(distill_slice + entries_at);
    int32_t *const sidx = reinterpret_cast<int32_t *>(sp + a.k), *const seen = sidx + a.k;
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / slices;
    const int rank = blockIdx.x - static_cast<int>(row) * slices;
    if (FWD && slices > 1) cluster_arrive_relaxed();  // all CTAs of the cluster run, before their memory is written

    // the teacher's entries: kDistillEntries per thread
    int32_t idx[kDistillEntries];
    float t[kDistillEntries];
    bool any = false;
    float tm = -INFINITY;
#pragma unroll
    for (int u = 0; u < kDistillEntries; ++u) {
        const int j = tid + u * kDistillThreads;
        idx[u] = -1, t[u] = -INFINITY;
        if (j < a.k) {
            idx[u] = a.t_idx[row * a.k + j];
            t[u] = a.t[row * a.k + j];
            if (idx[u] < 0 || idx[u] >= a.V || t[u] == -INFINITY) idx[u] = -1, t[u] = -INFINITY;
        }
        any |= idx[u] >= 0;
        tm = fmaxf(tm, t[u]);
    }
    const bool has = __syncthreads_or(any);

    const T *z = static_cast<const T *>(a.logits) + row * a.ld;
    T *g = static_cast<T *>(a.grad) + row * a.ld_grad;
    // vector i holds the values first + i kVec .. + kVec - 1 of the row
    const int first = -static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
    const int vectors = (a.V - first + kVec - 1) / kVec;
    const int per = (vectors + slices - 1) / slices;
    const int v0 = min(rank * per, vectors), nv = min(per, vectors - v0);
    const int e0 = first + v0 * kVec;  // the slice's first value (may be below 0) and its end
    const int e1 = e0 + nv * kVec;
    const bool same_phase = BWD && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
    auto store_vector = [&](int i, const float *v) {  // of the gradient
        const int e = e0 + i * kVec;
        if (same_phase && e >= 0 && e + kVec <= a.V) {
            *reinterpret_cast<uint4 *>(g + e) = Vec16<T>::pack(v);
        } else {
#pragma unroll
            for (int x = 0; x < kVec; ++x)
                if (e + x >= 0 && e + x < a.V) store_value(g + e + x, v[x]);
        }
    };
    if (!has) {
        if (BWD) {
            const float zero[kVec] = {};
            for (int i = tid; i < nv; i += kDistillThreads) store_vector(i, zero);
        }
        if (FWD && rank == 0 && tid == 0) {
            a.loss[row] = 0.0f;
            if (a.stats_out != nullptr) a.stats_out[2 * row] = a.stats_out[2 * row + 1] = 0.0f;
        }
        __syncwarp();
        if (FWD && slices > 1) cluster_wait();
        return;
    }
    auto load_vector = [&](int i) {  // values outside the row: -inf
        const int e = e0 + i * kVec;
        if (e >= 0 && e + kVec <= a.V) return __ldcs(reinterpret_cast<const uint4 *>(z + e));
        float v[kVec];
#pragma unroll
        for (int x = 0; x < kVec; ++x) v[x] = e + x >= 0 && e + x < a.V ? load_value(z + e + x) : -INFINITY;
        return Vec16<T>::pack(v);
    };
    const uint4 *slice = reinterpret_cast<const uint4 *>(distill_slice);
    if (RESIDENT) {  // one bulk copy of the vectors inside the row; the others by hand
        const int lo = e0 < 0 ? 1 : 0, hi = e1 > a.V ? nv - 1 : nv;
        if (tid == 0) {
            sm.abort = 0;
            mbar_init(&sm.bar, 1);
            fence_mbar_init();
            const uint32_t bytes = hi > lo ? static_cast<uint32_t>(hi - lo) * 16u : 0u;
            mbar_arrive_expect_tx(&sm.bar, bytes);
            if (bytes > 0) bulk_g2s(distill_slice + lo * 16, z + e0 + lo * kVec, bytes, &sm.bar, l2_evict_first_policy());
        }
        if (tid < 2 && nv > 0) {
            const int i = tid == 0 ? 0 : nv - 1;
            if (i < lo || i >= hi) reinterpret_cast<uint4 *>(distill_slice)[i] = load_vector(i);
        }
    }

    // the teacher's softmax
    const float inv_T = fminf(1.0f / a.T, 3.4e38f);
    const float c = fminf(1.44269504f / a.T, 3.4e38f);  // log2 e / T
    tm = block_max<kDistillThreads>(tm, sm.scratch);
    float ts = 0.0f;
#pragma unroll
    for (int u = 0; u < kDistillEntries; ++u)
        if (idx[u] >= 0) ts += expf((t[u] - tm) * inv_T);
    ts = block_sum<kDistillThreads>(ts, sm.scratch);
    float p[kDistillEntries], plogp = 0.0f;
#pragma unroll
    for (int u = 0; u < kDistillEntries; ++u) {
        const int j = tid + u * kDistillThreads;
        p[u] = 0.0f;
        if (idx[u] >= 0) {
            const float x = (t[u] - tm) * inv_T;
            p[u] = expf(x) / ts;
            if (FWD && rank == 0 && p[u] != 0.0f) plogp += p[u] * (x - logf(ts));
        }
        if (BWD && j < a.k) sp[j] = p[u], sidx[j] = idx[u];
        if (idx[u] < e0 || idx[u] >= e1) idx[u] = -1;  // from here on: the slice's entries
    }
    float zt[kDistillEntries];  // the entries' logits, before a gradient may overwrite them
    if (RESIDENT) {
        __syncthreads();
        if (!mbar_wait(&sm.bar, 0, &sm.abort) && tid == 0)
            atomicOr(a.flag, kErrWaitTimeout);
    }
#pragma unroll
    for (int u = 0; u < kDistillEntries; ++u) {
        zt[u] = 0.0f;
        if (idx[u] >= 0)
            zt[u] = load_value(RESIDENT ? reinterpret_cast<const T *>(distill_slice) + (idx[u] - e0) : z + idx[u]);
    }

    float m, s;
    if (FWD) {
        Partial mine = {-INFINITY, 0.0f, 0.0f, 0.0f};
        for (int i0 = tid; i0 < nv; i0 += kDistillThreads * kDistillUnroll) {
            uint4 raw[kDistillUnroll];
            float mx = mine.m;
#pragma unroll
            for (int u = 0; u < kDistillUnroll; ++u) {
                const int i = i0 + u * kDistillThreads;
                if (i < nv) raw[u] = RESIDENT ? slice[i] : load_vector(i);
            }
#pragma unroll
            for (int u = 0; u < kDistillUnroll; ++u) {
                if (i0 + u * kDistillThreads >= nv) continue;
                float v[kVec];
                Vec16<T>::unpack(raw[u], v);
#pragma unroll
                for (int x = 0; x < kVec; ++x) mx = fmaxf(mx, v[x]);
            }
            const Exponent e{finite_max(mx), c};
            if (mine.s != 0.0f) mine.s *= e(finite_max(mine.m));
            mine.m = mx;
#pragma unroll
            for (int u = 0; u < kDistillUnroll; ++u) {
                if (i0 + u * kDistillThreads >= nv) continue;
                float v[kVec];
                Vec16<T>::unpack(raw[u], v);
                float part = 0.0f;
#pragma unroll
                for (int x = 0; x < kVec; ++x) part += e(v[x]);
                mine.s += part;
            }
        }
#pragma unroll
        for (int u = 0; u < kDistillEntries; ++u)
            if (idx[u] >= 0 && p[u] != 0.0f) {
                mine.cross += p[u] * ((zt[u] - finite_max(mine.m)) * inv_T);
                mine.p += p[u];
            }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
            const Partial other = {__shfl_xor_sync(0xFFFFFFFFu, mine.m, o), __shfl_xor_sync(0xFFFFFFFFu, mine.s, o),
                                   __shfl_xor_sync(0xFFFFFFFFu, mine.cross, o),
                                   __shfl_xor_sync(0xFFFFFFFFu, mine.p, o)};
            // the same order in both lanes: the result is the same in all
            mine = (lane & o) ? join(other, mine, c, inv_T) : join(mine, other, c, inv_T);
        }
        if (lane == 0) sm.warp_part[warp] = make_float4(mine.m, mine.s, mine.cross, mine.p);
        plogp = warp_sum(plogp);
        if (lane == 0) sm.entropy[warp] = plogp;
        __syncthreads();
        auto take = [](const float4 &v) { return Partial{v.x, v.y, v.z, v.w}; };
        Partial all = take(sm.warp_part[0]);
#pragma unroll
        for (int w = 1; w < kDistillThreads / 32; ++w) all = join(all, take(sm.warp_part[w]), c, inv_T);
        if (slices > 1) {
            cluster_wait();
            if (tid < slices)
                cluster_store(cluster_addr(&sm.gathered[rank], tid), make_float4(all.m, all.s, all.cross, all.p));
            __syncwarp();
            cluster_arrive();
            cluster_wait();
            all = take(sm.gathered[0]);
            for (int r = 1; r < slices; ++r) all = join(all, take(sm.gathered[r]), c, inv_T);
        }
        m = all.m, s = all.s;
        if (rank == 0 && tid == 0) {
            plogp = 0.0f;
            for (int w = 0; w < kDistillThreads / 32; ++w) plogp += sm.entropy[w];
            const float logs = s == 0.0f ? -INFINITY : logf(s);
            const float kl = s == 0.0f ? INFINITY : plogp - all.cross + all.p * logs;
            a.loss[row] = a.T * a.T * kl;
            if (a.stats_out != nullptr) {
                a.stats_out[2 * row] = m;
                a.stats_out[2 * row + 1] = s;
            }
        }
    } else {
        m = a.stats_in[2 * row];
        s = a.stats_in[2 * row + 1];
    }

    if (BWD) {
        const Exponent e{finite_max(m), c};
        const float cg = a.T * a.grad_loss[row], inv = s == 0.0f ? 0.0f : 1.0f / s, coef = cg * inv;
        const int slots = seen_slots(a.k);
        for (int i = tid; i < slots; i += kDistillThreads) seen[i] = -1;
        __syncthreads();  // (grad may be logits: the entries' logits are read before it is written)
        for (int i0 = tid; i0 < nv; i0 += kDistillThreads * kDistillUnroll) {
            uint4 raw[kDistillUnroll];
#pragma unroll
            for (int u = 0; u < kDistillUnroll; ++u) {
                const int i = i0 + u * kDistillThreads;
                if (i < nv) raw[u] = RESIDENT ? slice[i] : load_vector(i);
            }
#pragma unroll
            for (int u = 0; u < kDistillUnroll; ++u) {
                const int i = i0 + u * kDistillThreads;
                if (i >= nv) continue;
                float v[kVec];
                Vec16<T>::unpack(raw[u], v);
#pragma unroll
                for (int x = 0; x < kVec; ++x) v[x] = coef * e(v[x]);
                store_vector(i, v);
            }
        }
        __syncthreads();
        // The teacher's entries: q - p over what the loop above has written.
        // Indices seldom repeat; where the table finds one that does, the
        // entries before and after are looked through.
        bool repeats = false;
#pragma unroll
        for (int u = 0; u < kDistillEntries; ++u) {
            if (idx[u] < 0) continue;
            uint32_t h = (static_cast<uint32_t>(idx[u]) * 0x9E3779B1u) >> 16 & (slots - 1);
            while (true) {  // ends: at most half the slots are taken
                const int32_t old = atomicCAS(&seen[h], -1, idx[u]);
                if (old == -1) break;
                if (old == idx[u]) {
                    repeats = true;
                    break;
                }
                h = (h + 1) & (slots - 1);
            }
        }
        repeats = __syncthreads_or(repeats);
#pragma unroll
        for (int u = 0; u < kDistillEntries; ++u) {
            if (idx[u] < 0) continue;
            float sum = p[u];
            bool leads = true;
            if (repeats) {
                const int j = tid + u * kDistillThreads;
                sum = 0.0f;
                for (int i = 0; i < a.k; ++i)
                    if (sidx[i] == idx[u]) {
                        leads &= i >= j;
                        sum += sp[i];
                    }
            }
            if (leads) store_value(g + idx[u], cg * (e(zt[u]) * inv - sum));
        }
    }
}

template <typename T, bool FWD, bool BWD, bool RESIDENT>
static cudaError_t start_distill(const DistillParams &p, int64_t n, int slices, int64_t slice, cudaStream_t s) {
    auto kernel = distill_kernel<T, FWD, BWD, RESIDENT>;
    const size_t smem = static_cast<size_t>(slice) + (BWD ? 8 * static_cast<size_t>(p.k) + 4 * seen_slots(p.k) : 0);
    cudaError_t e = cudaSuccess;
    if (smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e == cudaSuccess && slices > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(n * slices));
    cfg.blockDim = dim3(kDistillThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(slices);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = FWD && slices > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p, slices, static_cast<uint32_t>(slice));
}

// Bytes of a slice that leave room for four CTAs per SM beside it, and the
// most that one CTA holds.
constexpr int64_t kSliceGood = 48 * 1024, kSliceMost = 200 * 1024;

template <bool FWD, bool BWD>
static cudaError_t launch_distill(const DistillParams &p, vie_dtype dtype, int64_t n, cudaStream_t s) {
    const int64_t bytes = static_cast<int64_t>(p.V) * dtype_size(dtype) + 32;  // with both ends' overhang
    int slices = 1;
    if constexpr (FWD && BWD) {
        const auto slice_of = [&](int c) { return (bytes / 16 + c - 1) / c * 16; };
        while (slices < kMaxSlices && slice_of(slices) > kSliceGood) slices *= 2;
        if (slice_of(slices) <= kSliceMost)
            return dtype == VIE_DTYPE_BF16
                       ? start_distill<__nv_bfloat16, FWD, BWD, true>(p, n, slices, slice_of(slices), s)
                       : start_distill<float, FWD, BWD, true>(p, n, slices, slice_of(slices), s);
    } else if constexpr (FWD) {
        // enough CTAs for the chip, of 32 KB of the row or more
        while (slices < kMaxSlices && n * slices < 1024 && bytes / slices > 32768) slices *= 2;
    } else {
        // no partials to join: all of a thread's vectors in flight at once
        while (bytes / slices > 16 * kDistillThreads * kDistillUnroll && n * slices < (1 << 30)) slices *= 2;
    }
    return dtype == VIE_DTYPE_BF16 ? start_distill<__nv_bfloat16, FWD, BWD, false>(p, n, slices, 0, s)
                                   : start_distill<float, FWD, BWD, false>(p, n, slices, 0, s);
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
