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
constexpr int kMaxSlices = 16;

// exp2((z - m) c) = exp((z - m) / T).  The difference comes first: the type's
// lowest value is a usual mask, and z c - m c overflows there.
struct Exponent {
    float m, c;
    __device__ __forceinline__ float operator()(float z) const { return exp2_approx((z - m) * c); }
};
// The maximum that exponents are taken from: 0 where no logit is above -inf.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

constexpr int kDistillThreads = 256;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kEntries = VIE_K_MAX / kDistillThreads;  // teacher entries per thread of a teacher warp, at most

struct DistillSmem {
    float4 gathered[kMaxSlices];      // per slice: max z and the sums of exp((z - m) / T), p (z - m) / T and p
    float4 teacher[kDistillWarps];    // per teacher warp: the sums of p (z - m) / T, p and p log p
    float2 t_part[kDistillWarps];     // per teacher warp: max t and the sum of exp((t - max t) / T)
    float row_max[kDistillWarps], row_sum[kDistillWarps];
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
// The first warps (one per 128 entries) deal with the teacher while the others
// wait for the slice: a thread's share of the row is small, and what every
// thread does besides counts (27 instructions per logit when all warps took
// part in the teacher's sums, 14 are the row's own).
// Dynamic shared memory: the slice (RESIDENT); from entries_at on (BWD) p and
// the indices of the teacher's entries and the hash table.
template <typename T, bool FWD, bool BWD, bool RESIDENT>
__global__ void __launch_bounds__(kDistillThreads, RESIDENT ? 5 : 4)
    distill_kernel(const DistillParams a, int log2_slices, uint32_t entries_at) {
    constexpr int NT = kDistillThreads, U = RESIDENT ? 2 : 8;  // U: vectors in flight per thread
    constexpr int kVec = Vec16<T>::kVec;
    extern __shared__ __align__(16) unsigned char distill_slice[];
    __shared__ DistillSmem sm;
    float *const sp = reinterpret_cast<float *>(distill_slice + entries_at);
    int32_t *const sidx = reinterpret_cast<int32_t *>(sp + a.k), *const seen = sidx + a.k;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int slices = 1 << log2_slices, rank = blockIdx.x & (slices - 1);
    const int64_t row = blockIdx.x >> log2_slices;
    const int t_warps = (a.k + 32 * kEntries - 1) / (32 * kEntries);
    const bool teaches = warp < t_warps;
    if (FWD && slices > 1) cluster_arrive_relaxed();  // all CTAs of the cluster run, before their memory is written
    if (RESIDENT && tid == 0) {
        sm.abort = 0;
        mbar_init(&sm.bar, 1);
        fence_mbar_init();
    }
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one

    // a teacher warp's entries: idx -1 where there is none
    int32_t idx[kEntries];
    float t[kEntries];
    bool any = false;
    if (teaches) {
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            const int j = tid + u * 32 * t_warps;
            idx[u] = -1, t[u] = -INFINITY;
            if (j < a.k) {
                idx[u] = a.t_idx[row * a.k + j];
                t[u] = a.t[row * a.k + j];
                if (idx[u] < 0 || idx[u] >= a.V || t[u] == -INFINITY) idx[u] = -1, t[u] = -INFINITY;
            }
            any |= idx[u] >= 0;
        }
    }
    const bool has = __syncthreads_or(any);

    const T *z = static_cast<const T *>(a.logits) + row * a.ld;
    T *g = static_cast<T *>(a.grad) + row * a.ld_grad;
    // vector i holds the values first + i kVec .. + kVec - 1 of the row; this
    // slice has nv of them, from value e0 (may be below 0) to e1; those
    // from lo to hi lie inside the row
    const int first = -static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
    const int vectors = (a.V - first + kVec - 1) / kVec;
    const int per = (vectors + slices - 1) >> log2_slices;
    const int v0 = min(rank * per, vectors), nv = min(per, vectors - v0);
    const int e0 = first + v0 * kVec, e1 = e0 + nv * kVec;
    const int lo = e0 < 0 ? 1 : 0, hi = e1 > a.V ? nv - 1 : nv;
    const int edge = tid == 0 ? 0 : nv - 1;  // threads 0 and 1: the vector that is not, if there is one
    const bool has_edge = tid < min(nv, 2) && (edge < lo || edge >= hi);
    auto load_edge = [&]() {  // values outside the row: -inf
        const int e = e0 + edge * kVec;
        float v[kVec];
#pragma unroll
        for (int x = 0; x < kVec; ++x) v[x] = e + x >= 0 && e + x < a.V ? load_value(z + e + x) : -INFINITY;
        return Vec16<T>::pack(v);
    };
    auto store_some = [&](int i, const float *v) {  // of the gradient: value by value, those inside the row
        const int e = e0 + i * kVec;
#pragma unroll
        for (int x = 0; x < kVec; ++x)
            if (e + x >= 0 && e + x < a.V) store_value(g + e + x, v[x]);
    };
    const bool same_phase = BWD && ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
    const uint4 *const zv = reinterpret_cast<const uint4 *>(z + e0);  // (only lo .. hi are read)
    uint4 *const gv = reinterpret_cast<uint4 *>(g + e0);
    if (!has) {
        if (BWD) {
            const float zero[kVec] = {};
            if (same_phase)
                for (int i = lo + tid; i < hi; i += NT) gv[i] = make_uint4(0, 0, 0, 0);
            else
                for (int i = lo + tid; i < hi; i += NT) store_some(i, zero);
            if (has_edge) store_some(edge, zero);
        }
        if (FWD && rank == 0 && tid == 0) {
            a.loss[row] = 0.0f;
            if (a.stats_out != nullptr) a.stats_out[2 * row] = a.stats_out[2 * row + 1] = 0.0f;
        }
        __syncwarp();
        if (FWD && slices > 1) cluster_wait();
        return;
    }
    uint4 *const slice = reinterpret_cast<uint4 *>(distill_slice);
    if (RESIDENT) {  // one bulk copy of the vectors inside the row; the others by hand
        if (tid == 0) {
            const uint32_t bytes = hi > lo ? static_cast<uint32_t>(hi - lo) * 16u : 0u;
            mbar_arrive_expect_tx(&sm.bar, bytes);
            if (bytes > 0) bulk_g2s(slice + lo, zv + lo, bytes, &sm.bar, l2_evict_first_policy());
        }
        if (has_edge) slice[edge] = load_edge();
    }

    const float inv_T = fminf(1.0f / a.T, 3.4e38f);
    const float c = fminf(1.44269504f / a.T, 3.4e38f);  // log2 e / T
    float p[kEntries];   // the teacher's softmax, of the entries before the sums over repeats
    float take[kEntries];  // what the gradient takes off at the entry's index
    bool repeats = false;
    if (teaches) {
        float tm = -INFINITY, ts = 0.0f;
#pragma unroll
        for (int u = 0; u < kEntries; ++u) tm = fmaxf(tm, t[u]);
        tm = warp_max(tm);
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            p[u] = idx[u] >= 0 ? expf((t[u] - tm) * inv_T) : 0.0f;
            ts += p[u];
        }
        ts = warp_sum(ts);
        if (t_warps > 1) {
            if (lane == 0) sm.t_part[warp] = make_float2(tm, ts);
            named_barrier_sync(1, 32 * t_warps);
            const float own = tm;
            for (int w = 0; w < t_warps; ++w) tm = fmaxf(tm, sm.t_part[w].x);
            ts = 0.0f;
            for (int w = 0; w < t_warps; ++w)
                if (sm.t_part[w].y != 0.0f) ts += sm.t_part[w].y * expf((sm.t_part[w].x - tm) * inv_T);
            const float scale = own == -INFINITY ? 0.0f : expf((own - tm) * inv_T);
#pragma unroll
            for (int u = 0; u < kEntries; ++u) p[u] = idx[u] >= 0 ? p[u] * scale : 0.0f;
        }
        const float log_ts = logf(ts);
        float plogp = 0.0f;
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            const int j = tid + u * 32 * t_warps;
            if (u > 0 && u * 32 * t_warps >= a.k) continue;
            p[u] /= ts;
            if (FWD && rank == 0 && p[u] != 0.0f) plogp += p[u] * ((t[u] - tm) * inv_T - log_ts);
            if (BWD && j < a.k) sp[j] = p[u], sidx[j] = idx[u];
            if (idx[u] < e0 || idx[u] >= e1) idx[u] = -1;  // from here on: the slice's entries
        }
        if (FWD && rank == 0) {
            plogp = warp_sum(plogp);
            if (lane == 0) sm.teacher[warp].z = plogp;
        }
        if (BWD) {
            // Indices seldom repeat; where the table finds one that does, the
            // first entry of an index takes the sum of all.
            const int slots = seen_slots(a.k);
            for (int i = tid; i < slots; i += 32 * t_warps) seen[i] = -1;
            named_barrier_sync(1, 32 * t_warps);
#pragma unroll
            for (int u = 0; u < kEntries; ++u) {
                take[u] = p[u];
                if (idx[u] < 0) continue;
                uint32_t h = (static_cast<uint32_t>(idx[u]) * 0x9E3779B1u) >> 16 & (slots - 1);
                while (true) {  // ends: at most half the slots are taken
                    const int32_t old = atomicCAS(&seen[h], -1, idx[u]);
                    repeats |= old == idx[u];
                    if (old == -1 || old == idx[u]) break;
                    h = (h + 1) & (slots - 1);
                }
            }
            // (of a repeated index, some thread has found the slot taken: all of them look)
            if (t_warps > 1) {
                if (lane == 0) sm.t_part[warp].x = 0.0f;
                named_barrier_sync(1, 32 * t_warps);
            }
            repeats = __any_sync(0xFFFFFFFFu, repeats);
            if (t_warps > 1) {
                if (lane == 0 && repeats) sm.t_part[0].x = 1.0f;
                named_barrier_sync(1, 32 * t_warps);
                repeats = sm.t_part[0].x != 0.0f;
            }
        }
    }
    if (RESIDENT) {
        __syncthreads();  // the vectors that were copied by hand
        if (!mbar_wait(&sm.bar, 0, &sm.abort) && tid == 0) atomicOr(a.flag, kErrWaitTimeout);
    }
    float zt[kEntries];  // the entries' logits, before a gradient may overwrite them
    if (teaches) {
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            zt[u] = 0.0f;
            if (idx[u] >= 0) zt[u] = load_value(RESIDENT ? reinterpret_cast<const T *>(slice) + (idx[u] - e0) : z + idx[u]);
        }
        if (BWD && repeats) {
#pragma unroll
            for (int u = 0; u < kEntries; ++u) {
                if (idx[u] < 0) continue;
                const int j = tid + u * 32 * t_warps;
                bool leads = true;
                take[u] = 0.0f;
                for (int i = 0; i < a.k; ++i)
                    if (sidx[i] == idx[u]) {
                        leads &= i >= j;
                        take[u] += sp[i];
                    }
                if (!leads) take[u] = -1.0f;  // (no sum of probabilities: nothing to store)
            }
        }
    }

    float m, s;
    if (FWD) {
        m = -INFINITY, s = 0.0f;  // of this thread, then of the CTA, then of the row
        auto add = [&](const Exponent &e, const uint4 &raw) {
            float v[kVec], part = 0.0f;
            Vec16<T>::unpack(raw, v);
#pragma unroll
            for (int x = 0; x < kVec; ++x) part += e(v[x]);
            s += part;
        };
        if (RESIDENT) {
            for (int i = tid; i < nv; i += NT) m = fmaxf(m, Vec16<T>::max_of(slice[i]));
            m = block_max<NT>(m, sm.row_max);
            const Exponent e{finite_max(m), c};
#pragma unroll 2
            for (int i = tid; i < nv; i += NT) add(e, slice[i]);
        } else {
            auto raise = [&](float mx) {  // the thread's maximum, and its sum with it
                if (s != 0.0f) s *= Exponent{finite_max(mx), c}(finite_max(m));
                m = mx;
            };
            for (int i = lo + tid; i < hi; i += U * NT) {
                uint4 raw[U];
                float mx = m;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * NT < hi) raw[u] = __ldcs(zv + i + u * NT);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * NT < hi) mx = fmaxf(mx, Vec16<T>::max_of(raw[u]));
                raise(mx);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * NT < hi) add(Exponent{finite_max(m), c}, raw[u]);
            }
            if (has_edge) {
                const uint4 raw = load_edge();
                raise(fmaxf(m, Vec16<T>::max_of(raw)));
                add(Exponent{finite_max(m), c}, raw);
            }
            const float top = block_max<NT>(m, sm.row_max);
            raise(top);
        }
        s = warp_sum(s);
        if (lane == 0) sm.row_sum[warp] = s;
        if (teaches) {
            float cross = 0.0f, mass = 0.0f;
#pragma unroll
            for (int u = 0; u < kEntries; ++u)
                if (idx[u] >= 0 && p[u] != 0.0f) {
                    cross += p[u] * ((zt[u] - finite_max(m)) * inv_T);
                    mass += p[u];
                }
            cross = warp_sum(cross), mass = warp_sum(mass);
            if (lane == 0) sm.teacher[warp].x = cross, sm.teacher[warp].y = mass;
        }
        __syncthreads();
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < kDistillWarps; ++w) s += sm.row_sum[w];
        float4 mine = make_float4(m, s, 0.0f, 0.0f);
        if (warp == 0)
            for (int w = 0; w < t_warps; ++w) mine.z += sm.teacher[w].x, mine.w += sm.teacher[w].y;
        if (slices > 1) {
            cluster_wait();
            if (tid < slices) cluster_store(cluster_addr(&sm.gathered[rank], tid), mine);
            __syncwarp();
            cluster_arrive();
            cluster_wait();
            // lane r: slice r; every warp joins them all, in the same order
            mine = lane < slices ? sm.gathered[lane] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
            m = warp_max(mine.x);
            const float m0 = finite_max(m), mr = finite_max(mine.x);
            s = warp_sum(mine.y != 0.0f ? mine.y * Exponent{m0, c}(mr) : 0.0f);
            if (rank == 0 && warp == 0) {
                mine.z = warp_sum(mine.w != 0.0f ? mine.z + mine.w * ((mr - m0) * inv_T) : 0.0f);
                mine.w = warp_sum(mine.w);
            }
        }
        if (rank == 0 && tid == 0) {
            float plogp = 0.0f;
            for (int w = 0; w < t_warps; ++w) plogp += sm.teacher[w].z;
            const float kl = s == 0.0f ? INFINITY : plogp - mine.z + mine.w * logf(s);
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
        if (!FWD) __syncthreads();  // (grad may be logits: the entries' logits are read before it is written)
        auto grad_of = [&](const uint4 &raw, float *v) {
            Vec16<T>::unpack(raw, v);
#pragma unroll
            for (int x = 0; x < kVec; ++x) v[x] = coef * e(v[x]);
        };
        auto store = [&](int i, const uint4 &raw) {
            float v[kVec];
            grad_of(raw, v);
            if (same_phase) gv[i] = Vec16<T>::pack(v);
            else store_some(i, v);
        };
        if (RESIDENT) {
#pragma unroll 2
            for (int i = lo + tid; i < hi; i += NT) store(i, slice[i]);
        } else {
            for (int i = lo + tid; i < hi; i += U * NT) {
                uint4 raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * NT < hi) raw[u] = __ldcs(zv + i + u * NT);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * NT < hi) store(i + u * NT, raw[u]);
            }
        }
        if (has_edge) {
            float v[kVec];
            grad_of(RESIDENT ? slice[edge] : load_edge(), v);
            store_some(edge, v);
        }
        __syncthreads();
        if (teaches) {  // q - p over what the loop above has written at the entries
#pragma unroll
            for (int u = 0; u < kEntries; ++u)
                if (idx[u] >= 0 && !(take[u] < 0.0f)) store_value(g + idx[u], cg * (e(zt[u]) * inv - take[u]));
        }
    }
}

template <typename T, bool FWD, bool BWD, bool RESIDENT>
static cudaError_t start_distill(const DistillParams &p, int64_t n, int slices, int64_t slice, cudaStream_t s) {
    auto kernel = distill_kernel<T, FWD, BWD, RESIDENT>;
    int log2_slices = 0;
    while ((1 << log2_slices) < slices) ++log2_slices;
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
    return cudaLaunchKernelEx(&cfg, kernel, p, log2_slices, static_cast<uint32_t>(slice));
}

// Bytes of a slice that leave room for four CTAs per SM beside it, and the
// most that one CTA holds.
constexpr int64_t kSliceGood = 48 * 1024, kSliceMost = 200 * 1024;
constexpr int64_t kSliceStream = 128 * 1024;

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
        while (bytes / slices > kSliceStream && n * slices < (1 << 30)) slices *= 2;
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
