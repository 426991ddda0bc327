// vie_sample_logits.cu - tokens drawn from full logits with temperature,
// top-k, top-p and min-p of each row, from given uniform numbers (paper,
// Section 2: top-k sampling; Section 3: top-p and min-p as processors of the
// full-vocabulary logit tensor).
//
// Tokens rank by (logit descending, index ascending).  Weights are whole
// numbers, w = floor(2^40 exp((z - max z) (1 / T))), so sums of them are exact
// in any order and a draw does not depend on how the work is split.  All
// filters keep prefixes of the ranked tokens, so they are known by their
// masses, and the kept mass is the smallest of them:
//   S  = mass of the best top_k tokens
//   P  = C_i for the first i with C_i >= top_p S   (C: running mass)
//   Q  = mass of the tokens with w >= min_p 2^40
//   M  = max(2^40, min(S, P, Q))        (the best token alone weighs 2^40)
// and the draw is the first token with C_i > floor(u M): the shortest prefix
// of a given mass, found by narrowing the logits' ranking key digit by digit.
// top_p and u count in steps of 2^-24 (top_p rounded up, u down).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"

namespace vie {

struct SampleLogitsParams {
    const void *logits;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
    int64_t ld;
    int V;
};

constexpr int kSampleThreads = 512;
constexpr uint64_t kOne = 1ull << 40;  // the best token's weight

// floor(mass * count / 2^24), and whether that left a rest; mass < 2^62.
__device__ __forceinline__ uint64_t share_of(uint64_t mass, uint32_t count, bool *rest) {
    const uint64_t low = (mass & 0xFFFFFFu) * count;
    *rest = (low & 0xFFFFFFu) != 0;
    return (mass >> 24) * count + (low >> 24);
}

struct Weigh {
    float best, inv;
    bool warm;
    __device__ __forceinline__ uint64_t operator()(float z) const {
        if (!(z > -INFINITY)) return 0;  // masked out, or NaN
        if (z == best) return kOne;
        if (!warm) return 0;
        return static_cast<uint64_t>(expf((z - best) * inv) * 1099511627776.0f);
    }
};

struct SampleSmem {
    float scratch[kSampleThreads / 32];
    uint64_t mass[256];
    uint32_t count[256];
    uint64_t sum;
    uint64_t above;  // of the ranks before the chosen bin
    uint32_t bin, found;
    int32_t token;
};

__device__ __forceinline__ uint64_t block_sum_u64(SampleSmem &sm, uint64_t v) {
    __syncthreads();
    if (threadIdx.x == 0) sm.sum = 0;
    __syncthreads();
    atomicAdd(reinterpret_cast<unsigned long long *>(&sm.sum), static_cast<unsigned long long>(v));
    __syncthreads();
    return sm.sum;
}

// The shortest prefix of the ranked tokens with mass (BY_COUNT: with a number
// of tokens) >= target, of which the row has that much: the last token's key,
// how many of the tokens with this key it takes, and the mass before them.
template <typename T, bool BY_COUNT>
__device__ void shortest_prefix(SampleSmem &sm, const T *z, int V, const Weigh &weigh, uint64_t target, uint32_t *key,
                                uint64_t *ties, uint64_t *mass_before) {
    uint32_t prefix = 0;
    uint64_t before = 0, mass = 0;  // what the ranks before `prefix` amount to
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int b = threadIdx.x; b < 256; b += kSampleThreads) sm.mass[b] = 0, sm.count[b] = 0;
        __syncthreads();
        for (int v = threadIdx.x; v < V; v += kSampleThreads) {
            const float x = load_value(z + v);
            const uint64_t w = weigh(x);
            if (w == 0) continue;
            const uint32_t o = order_f32(x);
            if (shift < 24 && (o >> (shift + 8)) != prefix) continue;
            const uint32_t b = (o >> shift) & 255u;
            atomicAdd(&sm.count[b], 1u);
            atomicAdd(reinterpret_cast<unsigned long long *>(&sm.mass[b]), static_cast<unsigned long long>(w));
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint64_t c = before;
            int b = 255;
            for (; b > 0; --b) {
                const uint64_t add = BY_COUNT ? sm.count[b] : sm.mass[b];
                if (c + add >= target) break;
                c += add;
                mass += sm.mass[b];
            }
            sm.bin = static_cast<uint32_t>(b);
            sm.above = c;
            sm.sum = mass;
        }
        __syncthreads();
        prefix = (prefix << 8) | sm.bin;
        before = sm.above;
        mass = sm.sum;
    }
    *key = prefix;
    *mass_before = mass;
    const uint64_t w = weigh(unorder_f32(prefix));
    *ties = BY_COUNT ? target - before : (target - before + w - 1) / w;
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_logits_kernel(const SampleLogitsParams a) {
    __shared__ SampleSmem sm;
    const int64_t row = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits) + row * a.ld;
    const int V = a.V;
    float best = -INFINITY;
    for (int v = threadIdx.x; v < V; v += kSampleThreads) best = fmaxf(best, load_value(z + v));
    best = block_max<kSampleThreads>(best, sm.scratch);
    if (best == -INFINITY) {  // nothing to draw from
        if (threadIdx.x == 0) a.token[row] = -1, a.prob[row] = 0.0f;
        return;
    }
    const float temp = a.temperature != nullptr ? a.temperature[row] : 1.0f;
    Weigh weigh{best, 1.0f / temp, temp > 0.0f};
    const float top_p = a.top_p != nullptr ? a.top_p[row] : 1.0f, min_p = a.min_p != nullptr ? a.min_p[row] : 0.0f;
    const int top_k = !weigh.warm ? 1 : (a.top_k != nullptr ? a.top_k[row] : 0);

    uint64_t S = 0, Q = 0, positive = 0;
    const uint64_t least_w = min_p > 0.0f ? static_cast<uint64_t>(ceilf(fminf(min_p, 2.0f) * 1099511627776.0f)) : 0;
    for (int v = threadIdx.x; v < V; v += kSampleThreads) {
        const uint64_t w = weigh(load_value(z + v));
        S += w;
        positive += w != 0;
        Q += w >= least_w ? w : 0;
    }
    S = block_sum_u64(sm, S);
    Q = block_sum_u64(sm, Q);
    positive = block_sum_u64(sm, positive);
    uint32_t key;
    uint64_t ties, before;
    if (top_k > 0 && static_cast<uint64_t>(top_k) < positive) {
        shortest_prefix<T, true>(sm, z, V, weigh, static_cast<uint64_t>(top_k), &key, &ties, &before);
        S = before + ties * weigh(unorder_f32(key));
    }
    uint64_t M = S < Q ? S : Q;
    if (top_p < 1.0f) {
        bool rest;
        const uint32_t p24 = top_p > 0.0f ? static_cast<uint32_t>(ceilf(top_p * 16777216.0f)) : 0;
        uint64_t least = share_of(S, p24, &rest);
        least += rest;
        if (least == 0) least = 1;
        shortest_prefix<T, false>(sm, z, V, weigh, least, &key, &ties, &before);
        const uint64_t P = before + ties * weigh(unorder_f32(key));
        if (P < M) M = P;
    }
    if (M < kOne) M = kOne;
    const float u = a.u[row];
    const uint32_t u24 = u > 0.0f ? static_cast<uint32_t>(fminf(u * 16777216.0f, 16777215.0f)) : 0;
    bool rest;
    const uint64_t target = share_of(M, u24, &rest) + 1;
    shortest_prefix<T, false>(sm, z, V, weigh, target, &key, &ties, &before);
    // the ties-th token with this key, by index: runs of tokens in order
    if (threadIdx.x == 0) sm.found = 0;
    __syncthreads();
    for (int v0 = 0; v0 < V; v0 += kSampleThreads) {
        const int v = v0 + threadIdx.x;
        const bool hit = v < V && order_f32(load_value(z + v)) == key;
        const uint32_t in_warp = __ballot_sync(0xFFFFFFFFu, hit);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sm.count[threadIdx.x >> 5] = __popc(in_warp);
        __syncthreads();
        uint64_t at = sm.found;
        for (unsigned w = 0; w < threadIdx.x >> 5; ++w) at += sm.count[w];
        at += __popc(in_warp & ((1u << (threadIdx.x & 31)) - 1u));
        if (hit && at + 1 == ties) {
            a.token[row] = v;
            a.prob[row] = static_cast<float>(weigh(unorder_f32(key))) / static_cast<float>(M);
        }
        __syncthreads();
        if (threadIdx.x == 0)
            for (int w = 0; w < kSampleThreads / 32; ++w) sm.found += sm.count[w];
    }
}

}  // namespace vie

using namespace vie;

extern "C" vie_status vie_sample_logits(const void *logits, vie_dtype dtype, int64_t batch, int64_t V, int64_t ld,
                                        const float *u, const float *temperature, const int32_t *top_k,
                                        const float *top_p, const float *min_p, int32_t *out_token, float *out_prob,
                                        vie_stream stream) {
    const char *fn = "vie_sample_logits";
    if (batch < 0 || batch > VIE_MANY_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: batch=%lld outside [0, %d]", fn, static_cast<long long>(batch),
                    VIE_MANY_MAX);
    if (V < 1 || V > VIE_SAMPLE_V_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: V=%lld outside [1, %d]", fn, static_cast<long long>(V), VIE_SAMPLE_V_MAX);
    const vie_status st = check_matrix(fn, "logits", logits, dtype, batch, V, ld);
    if (st != VIE_OK) return st;
    if (batch > 0 && (u == nullptr || out_token == nullptr || out_prob == nullptr))
        return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(u, 4) || !aligned_to(temperature, 4) || !aligned_to(top_k, 4) || !aligned_to(top_p, 4) ||
        !aligned_to(min_p, 4) || !aligned_to(out_token, 4) || !aligned_to(out_prob, 4))
        return fail(VIE_ERR_INVALID_ARG, "%s: buffers must be 4-byte aligned", fn);
    if (batch == 0) return VIE_OK;
    SampleLogitsParams p = {};
    p.logits = logits, p.u = u, p.temperature = temperature, p.top_p = top_p, p.min_p = min_p, p.top_k = top_k;
    p.token = out_token, p.prob = out_prob, p.ld = ld, p.V = static_cast<int>(V);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == VIE_DTYPE_BF16)
        sample_logits_kernel<__nv_bfloat16><<<static_cast<unsigned>(batch), kSampleThreads, 0, s>>>(p);
    else
        sample_logits_kernel<float><<<static_cast<unsigned>(batch), kSampleThreads, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}
