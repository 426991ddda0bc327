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

// Slices per row: up to 8; up to 16 for a few rows alone (clusters of 16 find
// fewer places to run: 64 rows of 151936 take 18.9 us with them, 13.5 with 8).
constexpr int kSlices = 8, kMaxSlices = 16;
constexpr int kFewRows = 8;

// exp2((z - m) c) = exp((z - m) / T), with c = log2(e) / T.  The difference comes
// first: the type's lowest value is a usual mask, and z c - m c overflows there.
struct Exponent {
    float m, c;
    __device__ __forceinline__ float operator()(float z) const { return exp2_approx((z - m) * c); }
};
// The maximum that exponents are taken from: 0 where no logit is above -inf.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

constexpr int kDistillThreads = 256;
constexpr int kDistillWarps = kDistillThreads / 32;
// Vectors in flight per thread: eight, but for loss and gradient on bf16 logits,
// where a thread's 64 registers hold six (151936 x 4096: 450 us; 497 with eight).
template <typename T, bool FWD, bool BWD>
constexpr int kUnroll = FWD && BWD && sizeof(T) == 2 ? 6 : 8;
constexpr int kTeacherEntries = 4;  // of a teacher, per thread of the warps that deal with it
static_assert(VIE_K_MAX <= 32 * kTeacherEntries * kDistillWarps, "warps for all entries");

struct DistillSmem {
    float2 gathered[kMaxSlices];    // per slice of the row: max z and the sum of exp((z - max z) / T)
    uint64_t gather_bar;
    float2 part[kDistillWarps];     // the same per warp of a slice
    float3 teacher[kDistillWarps];  // per teacher warp: max t, the sum of exp((t - max t) / T), part of the loss
    int repeats, abort;
};

// Slots of the hash table of a slice's entries: a power of two, at least
// twice the entries.
__host__ __device__ inline int seen_slots(int k) {
    int slots = 64;
    while (slots < 2 * k) slots <<= 1;
    return slots;
}

// Where a slice's gradient goes: by vectors if its rows lie to 16-byte
// addresses as the logits' do, else value by value.
template <typename T>
struct GradSlice {
    static constexpr int kVec = Vec16<T>::kVec;
    T *g;
    int e0, V;
    bool by_vector;

    __device__ __forceinline__ GradSlice(const DistillParams &a, int64_t row, const Slice<T> &sl)
        : g(static_cast<T *>(a.grad) + row * a.ld_grad), e0(sl.e0), V(sl.V),
          by_vector(((reinterpret_cast<uintptr_t>(sl.z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0) {}
    __device__ __forceinline__ void store_values(int i, const float *v) const {  // those inside the row
        const int e = e0 + i * kVec;
#pragma unroll
        for (int x = 0; x < kVec; ++x)
            if (e + x >= 0 && e + x < V) store_value(g + e + x, v[x]);
    }
    __device__ __forceinline__ void store(int i, const float *v) const {
        if (by_vector) reinterpret_cast<uint4 *>(g + e0)[i] = Vec16<T>::pack(v);
        else store_values(i, v);
    }
};

template <typename T>
__device__ __forceinline__ void clear_gradient(const Slice<T> &sl, const GradSlice<T> &out) {
    const float zero[Slice<T>::kVec] = {};
    for (int i = sl.lo + threadIdx.x; i < sl.hi; i += kDistillThreads) out.store(i, zero);
    if (sl.has_edge()) out.store_values(sl.edge(), zero);
}

template <typename T>
__device__ __forceinline__ void gradient_of(const Exponent &e, float coef, const uint4 &raw, float *v) {
    Vec16<T>::unpack(raw, v);
#pragma unroll
    for (int x = 0; x < Slice<T>::kVec; ++x) v[x] = coef * e(v[x]);
}
// Running sums of exponentials, one per position of a vector: chains that do
// not wait for one another.
template <typename T>
struct Sums {
    float v[Slice<T>::kVec] = {};
    __device__ __forceinline__ void add(const Exponent &e, const uint4 &raw) {
        float x[Slice<T>::kVec];
        Vec16<T>::unpack(raw, x);
#pragma unroll
        for (int i = 0; i < Slice<T>::kVec; ++i) v[i] += e(x[i]);
    }
    __device__ __forceinline__ float total() const {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < Slice<T>::kVec; i += 2) s += v[i] + v[i + 1];
        return s;
    }
};

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

// One warp: the maximum and sum of this CTA's slice, joined from its warps'
// (sm.part, written before the last barrier), to all CTAs of the row.
__device__ __forceinline__ void send_partial(DistillSmem &sm, int slices, int rank, float c) {
    const int lane = threadIdx.x & 31;
    const float2 part = lane < kDistillWarps ? sm.part[lane] : make_float2(-INFINITY, 0.0f);
    const float m = warp_max(part.x);
    const float s = warp_sum(part.y != 0.0f ? part.y * Exponent{finite_max(m), c}(finite_max(part.x)) : 0.0f);
    if (lane == 0) mbar_arrive_expect_tx(&sm.gather_bar, 8u * slices);
    if (lane < slices)
        cluster_send(cluster_addr(&sm.gathered[rank], lane), make_float2(m, s),
                     cluster_addr(&sm.gather_bar, lane));
    __syncwarp();
}
// The row's, from those of all its slices, in the same order in every warp.
__device__ __forceinline__ void join_partials(const DistillParams &a, DistillSmem &sm, int slices, float c, float *m,
                                              float *s) {
    if (!mbar_wait(&sm.gather_bar, 0, &sm.abort) && threadIdx.x == 0) atomicOr(a.flag, kErrWaitTimeout);
    const int lane = threadIdx.x & 31;
    const float2 part = lane < slices ? sm.gathered[lane] : make_float2(-INFINITY, 0.0f);
    *m = warp_max(part.x);
    *s = warp_sum(part.y != 0.0f ? part.y * Exponent{finite_max(*m), c}(finite_max(part.x)) : 0.0f);
}

__device__ __forceinline__ void init_smem(DistillSmem &sm) {
    sm.abort = 0;
    mbar_init(&sm.gather_bar, 1);
    fence_mbar_init();
}

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
__global__ void __launch_bounds__(kDistillThreads, 4) distill_kernel(const DistillParams a, int log2_slices) {
    constexpr int NT = kDistillThreads, U = kUnroll<T, FWD, BWD>;
    extern __shared__ __align__(16) unsigned char distill_smem[];
    __shared__ DistillSmem sm;
    int32_t *const list = reinterpret_cast<int32_t *>(distill_smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // the first warps deal with the teacher, besides their part of the row
    const int t_warps = (a.k + 32 * kTeacherEntries - 1) / (32 * kTeacherEntries);
    Teacher tea(a.k, t_warps, tid < 32 * t_warps ? tid : -1, list, reinterpret_cast<float *>(list + 2 * a.k),
                list + 3 * a.k);
    const int slices = 1 << log2_slices, rank = blockIdx.x & (slices - 1);
    const int64_t row = blockIdx.x >> log2_slices;
    if (FWD) {
        if (tid == 0) init_smem(sm);
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
    const GradSlice<T> out(a, row, sl);
    if (FWD) cluster_wait();
    if (!has) {
        if (BWD) clear_gradient(sl, out);
        if (FWD && rank == 0 && tid == 0) write_row(a, row, 0.0f, 0.0f, 0.0f);
        return;
    }
    const float inv_T = fminf(1.0f / a.T, 3.4e38f);
    const float c = fminf(1.44269504f / a.T, 3.4e38f);  // log2 e / T
    const uint4 *const zv = sl.vectors();
    // The entries' logits, before a gradient may overwrite them; the loss (rank
    // 0) needs those of the whole row.
    const bool whole = FWD && rank == 0;
    T z_entries[kTeacherEntries] = {};
    const bool keeps = tea.mine() && (BWD || whole);
    if (keeps) tea.read_logits(sl.z, whole ? 0 : sl.e0, whole ? a.V : sl.e1, z_entries);
    float m, s;
    if (FWD) {
        m = -INFINITY, s = 0.0f;  // of this thread, then of the CTA, then of the row
        auto raise = [&](float mx) {  // the thread's maximum, and its sum with it
            if (s != 0.0f) s *= Exponent{finite_max(mx), c}(finite_max(m));
            m = mx;
        };
        for (int i = sl.lo + tid; i < sl.hi; i += U * NT) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * NT < sl.hi) raw[u] = BWD ? __ldcg(zv + i + u * NT) : __ldcs(zv + i + u * NT);
            typename Vec16<T>::Max top;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * NT < sl.hi) top.add(raw[u]);
            raise(fmaxf(m, top.top()));
            Sums<T> part;
            const Exponent e{finite_max(m), c};
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * NT < sl.hi) part.add(e, raw[u]);
            s += part.total();
        }
        if (sl.has_edge()) {
            const uint4 raw = sl.load_edge();
            typename Vec16<T>::Max top;
            top.add(raw);
            raise(fmaxf(m, top.top()));
            Sums<T> part;
            part.add(Exponent{finite_max(m), c}, raw);
            s += part.total();
        }
        raise(warp_max(m));
        s = warp_sum(s);
        if (lane == 0) sm.part[warp] = make_float2(m, s);
        if (keeps) tea.keep_logits(z_entries);
        __syncthreads();
        if (warp == 0) send_partial(sm, slices, rank, c);
        if (keeps) tea.softmax(sm, inv_T);  // while the partials travel
        join_partials(a, sm, slices, c, &m, &s);
    } else {
        m = a.stats_in[2 * row];
        s = a.stats_in[2 * row + 1];
        if (keeps) tea.keep_logits(z_entries);
        __syncthreads();  // (grad may be logits: the entries' logits are read before it is written)
    }
    if (BWD) {
        const Exponent e{finite_max(m), c};
        const float cg = a.T * a.grad_loss[row], inv = s == 0.0f ? 0.0f : 1.0f / s, coef = cg * inv;
        for (int i = sl.lo + tid; i < sl.hi; i += U * NT) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * NT < sl.hi) raw[u] = __ldcs(zv + i + u * NT);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * NT < sl.hi) {
                    float v[Slice<T>::kVec];
                    gradient_of<T>(e, coef, raw[u], v);
                    out.store(i + u * NT, v);
                }
        }
        if (sl.has_edge()) {
            float v[Slice<T>::kVec];
            gradient_of<T>(e, coef, sl.load_edge(), v);
            out.store_values(sl.edge(), v);
        }
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

static int log2_of(int slices) {
    int l = 0;
    while ((1 << l) < slices) ++l;
    return l;
}

struct DistillLaunch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    DistillLaunch(int threads, int slices, bool cluster, size_t smem, cudaStream_t s) {
        cfg.blockDim = dim3(static_cast<unsigned>(threads));
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = static_cast<unsigned>(slices);
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = cluster ? 2 : 1;
    }
};

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
    DistillLaunch l(kDistillThreads, slices, FWD, smem, s);
    l.cfg.gridDim = dim3(static_cast<unsigned>(n * slices));
    return cudaLaunchKernelEx(&l.cfg, kernel, p, log2_of(slices));
}

// Bytes of a slice that one CTA takes, at most.  Gradient alone (128256 x 2048):
// 155 us in slices of 128 KB, 163 of 256; each CTA reads the teacher's entries.
constexpr int64_t kSliceBytes = 128 * 1024;
// Loss and gradient, while a cluster can have more CTAs (fp32 128256 x 1024: 174 us in
// slices of 64 KB, 186 of 128; bf16 151936 x 4096: 450 in slices of 76 KB, 556 of 38).
constexpr int64_t kSliceStep = 80 * 1024;

template <bool FWD, bool BWD>
static cudaError_t launch_distill(const DistillParams &p, vie_dtype dtype, int64_t n, cudaStream_t s) {
    const int64_t bytes = static_cast<int64_t>(p.V) * dtype_size(dtype);
    int slices = 1;
    if (!FWD) {  // no partials to join
        while (bytes / slices > kSliceBytes && n * slices < (1 << 30)) slices *= 2;
    } else {
        if (BWD)
            while (slices < kSlices && bytes / slices > kSliceStep) slices *= 2;
        // enough CTAs for the chip, of 32 KB of the row or more
        while (slices < (n <= kFewRows ? kMaxSlices : kSlices) && n * slices < 1024 && bytes / slices > 32768) slices *= 2;
    }
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
