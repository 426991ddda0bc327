// vie_block.cuh - building blocks of the kernels on matrices of either storage
// type: values and 16-byte vectors of them, sums and maxima over a CTA, the
// exponential, and cluster primitives in inline PTX.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace vie {

__device__ __forceinline__ float load_value(const float *p) { return *p; }
__device__ __forceinline__ float load_value(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_value(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// The maximum / sum of v over the NT threads of the CTA, in all of them, in an
// order that depends on NT alone.  `scratch`: shared memory of this call
// alone; every thread of the CTA calls.
template <int NT>
__device__ __forceinline__ float block_max(float v, float (&scratch)[NT / 32]) {
    const int lane = threadIdx.x & 31;
    v = warp_max(v);
    if (lane == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[lane & (NT / 32 - 1)];
#pragma unroll
    for (int o = NT / 64; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
__device__ __forceinline__ float4 shfl_xor_add(float4 v, int o) {
    v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
    v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    v.z += __shfl_xor_sync(0xFFFFFFFFu, v.z, o);
    v.w += __shfl_xor_sync(0xFFFFFFFFu, v.w, o);
    return v;
}
template <int NT>
__device__ __forceinline__ float4 block_sum(float4 v, float4 (&scratch)[NT / 32]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v = shfl_xor_add(v, o);
    if (lane == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[lane & (NT / 32 - 1)];
#pragma unroll
    for (int o = NT / 64; o >= 1; o >>= 1) v = shfl_xor_add(v, o);
    return v;
}

// 16 bytes of a matrix row: kVec values.
template <typename T>
struct Vec16;
template <>
struct Vec16<float> {
    static constexpr int kVec = 4;
    struct Max {  // running maxima, one per position, of vectors; NaN aside
        float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        __device__ __forceinline__ void add(const uint4 &r) {
            v[0] = fmaxf(v[0], __uint_as_float(r.x)), v[1] = fmaxf(v[1], __uint_as_float(r.y));
            v[2] = fmaxf(v[2], __uint_as_float(r.z)), v[3] = fmaxf(v[3], __uint_as_float(r.w));
        }
        __device__ __forceinline__ float top() const { return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])); }
    };
    static __device__ __forceinline__ void unpack(const uint4 &r, float *v) {
        v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y);
        v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 pack(const float *v) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <>
struct Vec16<__nv_bfloat16> {
    static constexpr int kVec = 8;
    struct Max {  // running maxima, one per position, of vectors; NaN aside
        __nv_bfloat162 v[4];
        __device__ __forceinline__ Max() {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __float2bfloat162_rn(-INFINITY);
        }
        __device__ __forceinline__ void add(const uint4 &r) {
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __hmax2(v[i], *reinterpret_cast<const __nv_bfloat162 *>(&w[i]));
        }
        __device__ __forceinline__ float top() const {
            const __nv_bfloat162 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
            return fmaxf(__low2float(m), __high2float(m));
        }
    };
    static __device__ __forceinline__ void unpack(const uint4 &r, float *v) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float *v) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// The part of a row that a CTA deals with: a row is cut into 16-byte vectors at
// 16-byte addresses, and its 2^log2_slices CTAs take consecutive runs of them.
// Vector i of the slice holds values
// e0 + i kVec .. + kVec - 1 of the row; vectors lo .. hi - 1 of nv lie inside
// it.  At most two do not: `edge` is one of them in thread 0 or 1.
template <typename T>
struct Slice {
    static constexpr int kVec = Vec16<T>::kVec;
    const T *z;
    int e0, e1, nv, lo, hi, V;

    __device__ __forceinline__ Slice(const T *row, int V_, int log2_slices, int rank) : z(row), V(V_) {
        const int first = -static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
        const int vectors = (V - first + kVec - 1) / kVec;
        const int per = (vectors + (1 << log2_slices) - 1) >> log2_slices;
        const int v0 = min(rank * per, vectors);
        nv = min(per, vectors - v0);
        e0 = first + v0 * kVec;
        e1 = e0 + nv * kVec;
        lo = e0 < 0 ? 1 : 0;
        hi = e1 > V ? nv - 1 : nv;
    }
    __device__ __forceinline__ const uint4 *vectors() const { return reinterpret_cast<const uint4 *>(z + e0); }
    __device__ __forceinline__ int edge() const { return threadIdx.x == 0 ? 0 : nv - 1; }
    __device__ __forceinline__ bool has_edge() const {
        return threadIdx.x < min(nv, 2) && (edge() < lo || edge() >= hi);
    }
    __device__ __forceinline__ uint4 load_edge() const {  // values outside the row: -inf
        const int e = e0 + edge() * kVec;
        float v[kVec];
#pragma unroll
        for (int x = 0; x < kVec; ++x) v[x] = e + x >= 0 && e + x < V ? load_value(z + e + x) : -INFINITY;
        return Vec16<T>::pack(v);
    }
};

// 2^x of the special function unit (2 ulp), denormal results flushed to 0.
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Thread-block clusters: the barrier in its two halves (no ordering of its own
// in the first), and addresses in the other CTAs' shared memory.
__device__ __forceinline__ void cluster_arrive_relaxed() {
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_addr(const void *p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(a)
                 : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    return a;
}
// The same variable of another CTA of the cluster, as a generic pointer.
template <typename T>
__device__ __forceinline__ T *cluster_peer(T *p, uint32_t rank) {
    uint64_t a;
    asm("mapa.u64 %0, %1, %2;" : "=l"(a) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
    return reinterpret_cast<T *>(a);
}
// Two values into another CTA's shared memory, which count 8 bytes on that CTA's
// mbarrier when they are there: no fence, no barrier of all threads.
__device__ __forceinline__ void cluster_send(uint32_t addr, float2 v, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(addr),
                 "f"(v.x), "f"(v.y), "r"(bar)
                 : "memory");
}

}  // namespace vie
