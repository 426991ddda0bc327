// vie_row_softmax.cuh - what the kernels on full logits share whose gradient is a
// softmax: a row's statistics (m = max z and s = sum of exp((z - m) / T)) by the
// slices of a cluster, and the gradient of each slice.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "vie_block.cuh"
#include "vie_device.cuh"

namespace vie {

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
__device__ __forceinline__ float exponent_factor(float T) { return fminf(1.44269504f / T, 3.4e38f); }  // log2 e / T
// The maximum that exponents are taken from: 0 where no logit is above -inf.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;

struct RowSmem {
    float2 gathered[kMaxSlices];  // per slice of the row: max z and the sum of exp((z - max z) / T)
    uint64_t gather_bar;
    float2 part[kRowWarps];       // the same per warp of a slice
    int abort;

    __device__ __forceinline__ void init() {
        abort = 0;
        mbar_init(&gather_bar, 1);
        fence_mbar_init();
    }
};

// Where a slice's gradient goes: by vectors if its rows lie to 16-byte
// addresses as the logits' do, else value by value.
template <typename T>
struct GradSlice {
    static constexpr int kVec = Vec16<T>::kVec;
    T *g;
    int e0, V;
    bool by_vector;

    __device__ __forceinline__ GradSlice(T *row, const Slice<T> &sl)
        : g(row), e0(sl.e0), V(sl.V),
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
    for (int i = sl.lo + threadIdx.x; i < sl.hi; i += kRowThreads) out.store(i, zero);
    if (sl.has_edge()) out.store_values(sl.edge(), zero);
}

template <typename T>
__device__ __forceinline__ void gradient_of(const Exponent &e, float coef, const uint4 &raw, float *v) {
    Vec16<T>::unpack(raw, v);
#pragma unroll
    for (int x = 0; x < Slice<T>::kVec; ++x) v[x] = coef * e(v[x]);
}
// coef exp((z - m) / T) in the slice's values of the gradient.
template <typename T, int U>
__device__ __forceinline__ void store_softmax(const Slice<T> &sl, const GradSlice<T> &out, const Exponent &e,
                                              float coef) {
    constexpr int NT = kRowThreads;
    const uint4 *const zv = sl.vectors();
    for (int i = sl.lo + threadIdx.x; i < sl.hi; i += U * NT) {
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

// The maximum and sum of this thread's vectors of the slice, U of them in flight,
// left in sm.part per warp (read after the next barrier of the CTA).
// KEEP: the slice is read again soon.
template <typename T, int U, bool KEEP>
__device__ __forceinline__ void slice_statistics(const Slice<T> &sl, float c, RowSmem &sm) {
    constexpr int NT = kRowThreads;
    const uint4 *const zv = sl.vectors();
    float m = -INFINITY, s = 0.0f;  // of this thread, then of the warp
    auto raise = [&](float mx) {    // the thread's maximum, and its sum with it
        if (s != 0.0f) s *= Exponent{finite_max(mx), c}(finite_max(m));
        m = mx;
    };
    for (int i = sl.lo + threadIdx.x; i < sl.hi; i += U * NT) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * NT < sl.hi) raw[u] = KEEP ? __ldcg(zv + i + u * NT) : __ldcs(zv + i + u * NT);
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
    if ((threadIdx.x & 31) == 0) sm.part[threadIdx.x >> 5] = make_float2(m, s);
}

// The maximum and sum of this CTA's slice, joined from its warps' (sm.part, written
// before the last barrier), in any warp.
__device__ __forceinline__ void join_warps(const RowSmem &sm, float c, float *m, float *s) {
    const int lane = threadIdx.x & 31;
    const float2 part = lane < kRowWarps ? sm.part[lane] : make_float2(-INFINITY, 0.0f);
    *m = warp_max(part.x);
    *s = warp_sum(part.y != 0.0f ? part.y * Exponent{finite_max(*m), c}(finite_max(part.x)) : 0.0f);
}
// One warp: those to all CTAs of the row.
__device__ __forceinline__ void send_partial(RowSmem &sm, int slices, int rank, float c) {
    const int lane = threadIdx.x & 31;
    float m, s;
    join_warps(sm, c, &m, &s);
    if (lane == 0) mbar_arrive_expect_tx(&sm.gather_bar, 8u * slices);
    if (lane < slices)
        cluster_send(cluster_addr(&sm.gathered[rank], lane), make_float2(m, s),
                     cluster_addr(&sm.gather_bar, lane));
    __syncwarp();
}
// The row's, from those of all its slices, in the same order in every warp.
__device__ __forceinline__ void join_partials(uint32_t *flag, RowSmem &sm, int slices, float c, float *m, float *s) {
    if (!mbar_wait(&sm.gather_bar, 0, &sm.abort) && threadIdx.x == 0) atomicOr(flag, kErrWaitTimeout);
    const int lane = threadIdx.x & 31;
    const float2 part = lane < slices ? sm.gathered[lane] : make_float2(-INFINITY, 0.0f);
    *m = warp_max(part.x);
    *s = warp_sum(part.y != 0.0f ? part.y * Exponent{finite_max(*m), c}(finite_max(part.x)) : 0.0f);
}

// A launch of kRowThreads-thread CTAs that may start before the previous kernel
// on the stream has ended, the CTAs of a row as a cluster if they exchange.
struct RowLaunch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    RowLaunch(int64_t ctas, int cluster, size_t smem, cudaStream_t s) {
        cfg.gridDim = dim3(static_cast<unsigned>(ctas));
        cfg.blockDim = dim3(kRowThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 0 ? 2 : 1;
    }
    RowLaunch(const RowLaunch &) = delete;  // cfg points into it
};

inline int log2_of(int slices) {
    int l = 0;
    while ((1 << l) < slices) ++l;
    return l;
}

}  // namespace vie
