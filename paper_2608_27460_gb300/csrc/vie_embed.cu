// vie_embed.cu - rows of an embedding table, scaled, and the table's gradient.
// Models with tied embeddings read the same matrix that the output head
// projects on (paper, Section 3: W_out, one row per token).
//
//   lookup    out[i, :] = scale * table[token_i, :]
//   gradient  G[v, :] (+)= scale * sum over i with token_i = v of g[i, :]
//
// Products and sums are fp32, each result is rounded once.  The gradient's
// sums run in the order of the positions i: the tokens are sorted (stably),
// and each run of equal tokens is summed by itself, so results do not change
// from call to call.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"

namespace vie {

// ---- lookup -----------------------------------------------------------------

constexpr int kEmbedThreads = 256;

struct EmbedParams {
    const void *table;
    const int32_t *tokens;
    void *out;
    int64_t ld, ld_out, n;
    int64_t V;
    int d;
    float scale;
    uint32_t *flag;
};

template <typename TI, typename TO>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedParams a) {
    for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
        const int32_t tok = a.tokens[i];
        TO *out = static_cast<TO *>(a.out) + i * a.ld_out;
        const bool in = tok >= 0 && tok < a.V;
        if (tok >= a.V && threadIdx.x == 0) atomicOr(a.flag, kErrTokenIndex);
        const TI *row = static_cast<const TI *>(a.table) + (in ? tok : 0) * a.ld;
        if constexpr (std::is_same<TI, TO>::value) {
            if (a.scale == 1.0f && in) {  // a copy: every bit is kept
                for (int c = threadIdx.x; c < a.d; c += kEmbedThreads) out[c] = row[c];
                continue;
            }
        }
        for (int c = threadIdx.x; c < a.d; c += kEmbedThreads)
            store_value(out + c, in ? a.scale * load_value(row + c) : 0.0f);
    }
}

// ---- stable sort of the tokens ----------------------------------------------
// Least significant digit first, 8 bits at a time.  A block takes kSortTile
// consecutive pairs, its warps consecutive runs of it; a pair's place among
// its block's pairs of the same digit follows from the warps' digit counts
// and, inside a run, from the lanes before it with the same digit.

constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32, kSortRounds = 8;
constexpr int kSortTile = kSortThreads * kSortRounds;

struct SortPass {
    const int32_t *tokens;  // first pass: the caller's tokens, else NULL
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    uint32_t *counts;  // [256][blocks]
    uint32_t n, blocks, V, shift;
    uint32_t *flag;
};

// Tokens outside [0, V) sort behind all others, as V.
__device__ __forceinline__ uint32_t sort_key(const SortPass &a, uint32_t i) {
    if (a.tokens == nullptr) return a.key_in[i];
    const int32_t tok = a.tokens[i];
    return tok >= 0 && static_cast<uint32_t>(tok) < a.V ? static_cast<uint32_t>(tok) : a.V;
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortPass a) {
    __shared__ uint32_t count[256];
    count[threadIdx.x] = 0;
    __syncthreads();
    for (int r = 0; r < kSortRounds; ++r) {
        const uint32_t i = blockIdx.x * kSortTile + r * kSortThreads + threadIdx.x;
        if (i >= a.n) continue;
        if (a.tokens != nullptr && a.tokens[i] >= 0 && static_cast<uint32_t>(a.tokens[i]) >= a.V)
            atomicOr(a.flag, kErrTokenIndex);
        atomicAdd(&count[(sort_key(a, i) >> a.shift) & 255u], 1u);
    }
    __syncthreads();
    a.counts[static_cast<size_t>(threadIdx.x) * a.blocks + blockIdx.x] = count[threadIdx.x];
}

// Exclusive prefix sums over counts[0 .. total), in place; one CTA.
__global__ void __launch_bounds__(1024) sort_scan_kernel(uint32_t *counts, uint32_t total) {
    __shared__ uint32_t part[32];
    uint32_t base = 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t i0 = 0; i0 < total; i0 += 1024) {
        const uint32_t i = i0 + threadIdx.x;
        const uint32_t v = i < total ? counts[i] : 0;
        uint32_t incl = v;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) part[warp] = incl;
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int w = 0; w < 32; ++w) {
            before += w < warp ? part[w] : 0;
            all += part[w];
        }
        if (i < total) counts[i] = base + before + incl - v;
        base += all;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(const SortPass a) {
    __shared__ uint32_t at[kSortWarps][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kSortWarps * 256; i += kSortThreads) (&at[0][0])[i] = 0;
    __syncthreads();
    const uint32_t run = blockIdx.x * kSortTile + warp * (kSortTile / kSortWarps);
    for (int r = 0; r < kSortRounds; ++r) {
        const uint32_t i = run + r * 32 + lane;
        if (i < a.n) atomicAdd(&at[warp][(sort_key(a, i) >> a.shift) & 255u], 1u);
    }
    __syncthreads();
    {
        uint32_t next = a.counts[static_cast<size_t>(threadIdx.x) * a.blocks + blockIdx.x];
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t c = at[w][threadIdx.x];
            at[w][threadIdx.x] = next;
            next += c;
        }
    }
    __syncthreads();
    for (int r = 0; r < kSortRounds; ++r) {
        const uint32_t i = run + r * 32 + lane;
        const bool in = i < a.n;
        const uint32_t key = in ? sort_key(a, i) : 0;
        const uint32_t digit = in ? (key >> a.shift) & 255u : 256u;
        const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
        const uint32_t before = __popc(same & ((1u << lane) - 1u));
        uint32_t to = 0;
        if (in) to = at[warp][digit] + before;
        __syncwarp();
        if (in && before == 0) at[warp][digit] += __popc(same);
        __syncwarp();
        if (in) {
            a.key_out[to] = key;
            a.pos_out[to] = a.tokens != nullptr ? i : a.pos_in[i];
        }
    }
}

// ---- sums over the runs of equal tokens -------------------------------------

struct GradParams {
    const uint32_t *key, *pos;  // sorted
    const void *grad;
    void *out;
    int64_t ld_grad, ld;
    uint32_t n, V;
    int d, accumulate;
    float scale;
};

// One CTA per sorted position; the first of a run sums it.
template <typename TI, typename TO>
__global__ void __launch_bounds__(kEmbedThreads) embed_grad_kernel(const GradParams a) {
    const uint32_t i = blockIdx.x, key = a.key[i];
    if (key >= a.V || (i > 0 && a.key[i - 1] == key)) return;
    TO *out = static_cast<TO *>(a.out) + static_cast<int64_t>(key) * a.ld;
    for (int c = threadIdx.x; c < a.d; c += kEmbedThreads) {
        float sum = 0.0f;
        for (uint32_t j = i; j < a.n && a.key[j] == key; ++j)
            sum += load_value(static_cast<const TI *>(a.grad) + a.pos[j] * a.ld_grad + c);
        sum *= a.scale;
        if (a.accumulate) sum += load_value(out + c);
        store_value(out + c, sum);
    }
}

struct GradWorkspace {
    uint32_t blocks;
    int64_t key, pos, counts, bytes;  // offsets: two arrays of n each for keys and positions
};

static GradWorkspace grad_workspace(int64_t n) {
    GradWorkspace w;
    const int64_t arr = (4 * n + 255) / 256 * 256;
    w.blocks = static_cast<uint32_t>((n + kSortTile - 1) / kSortTile);
    w.key = 0;
    w.pos = 2 * arr;
    w.counts = 4 * arr;
    w.bytes = w.counts + int64_t(w.blocks) * 1024;
    return w;
}

template <typename TI, typename TO>
static void start_grad(const GradParams &p, cudaStream_t s) {
    embed_grad_kernel<TI, TO><<<p.n, kEmbedThreads, 0, s>>>(p);
}
template <typename TI, typename TO>
static void start_embed(const EmbedParams &p, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(p.n < 65536 ? p.n : 65536);
    embed_kernel<TI, TO><<<grid, kEmbedThreads, 0, s>>>(p);
}

// f<TI, TO>(p, s) for the two storage types.
#define VIE_BY_TYPES(f, in, out, p, s)                                      \
    do {                                                                    \
        if ((in) == VIE_DTYPE_BF16 && (out) == VIE_DTYPE_BF16)              \
            f<__nv_bfloat16, __nv_bfloat16>(p, s);                          \
        else if ((in) == VIE_DTYPE_BF16)                                    \
            f<__nv_bfloat16, float>(p, s);                                  \
        else if ((out) == VIE_DTYPE_BF16)                                   \
            f<float, __nv_bfloat16>(p, s);                                  \
        else                                                                \
            f<float, float>(p, s);                                          \
    } while (0)

static vie_status check_embed(const char *fn, const int32_t *tokens, int64_t n, int64_t V, int32_t d) {
    if (n < 0 || n > VIE_MANY_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_MANY_MAX);
    if (V < 1 || V > INT32_MAX - 1)
        return fail(VIE_ERR_INVALID_ARG, "%s: V=%lld outside [1, 2^31-2]", fn, static_cast<long long>(V));
    if (d < 1 || d > VIE_D_MAX) return fail(VIE_ERR_INVALID_ARG, "%s: d=%d outside [1, %d]", fn, d, VIE_D_MAX);
    if (n > 0 && tokens == nullptr) return fail(VIE_ERR_INVALID_ARG, "%s: tokens is NULL", fn);
    if (!aligned_to(tokens, 4)) return fail(VIE_ERR_INVALID_ARG, "%s: tokens must be 4-byte aligned", fn);
    return VIE_OK;
}

}  // namespace vie

using namespace vie;

extern "C" {

vie_status vie_embed(const void *table, vie_dtype dtype, int64_t V, int32_t d, int64_t ld, const int32_t *tokens,
                     int64_t n, float scale, void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream) {
    const char *fn = "vie_embed";
    vie_status st = check_embed(fn, tokens, n, V, d);
    if (st == VIE_OK) st = check_matrix(fn, "table", table, dtype, V, d, ld);
    if (st == VIE_OK) st = check_matrix(fn, "out", out, out_dtype, n, d, ld_out);
    if (st != VIE_OK || n == 0) return st;
    EmbedParams p = {};
    p.table = table, p.tokens = tokens, p.out = out, p.ld = ld, p.ld_out = ld_out, p.n = n, p.V = V, p.d = d;
    p.scale = scale;
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    VIE_BY_TYPES(start_embed, dtype, out_dtype, p, static_cast<cudaStream_t>(stream));
    e = cudaGetLastError();
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_embed_grad_workspace(int64_t n, int64_t V, int32_t d, int64_t *bytes) {
    const char *fn = "vie_embed_grad_workspace";
    alignas(4) static const int32_t some = 0;
    const vie_status st = check_embed(fn, &some, n, V, d);
    if (st != VIE_OK) return st;
    if (bytes == nullptr) return fail(VIE_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    *bytes = grad_workspace(n).bytes;
    return VIE_OK;
}

vie_status vie_embed_grad(const int32_t *tokens, int64_t n, const void *grad, vie_dtype dtype, int64_t ld_grad,
                          float scale, int64_t V, int32_t d, void *out, vie_dtype out_dtype, int64_t ld,
                          int32_t accumulate, void *workspace, int64_t workspace_bytes, vie_stream stream) {
    const char *fn = "vie_embed_grad";
    vie_status st = check_embed(fn, tokens, n, V, d);
    if (st == VIE_OK) st = check_matrix(fn, "grad", grad, dtype, n, d, ld_grad);
    if (st == VIE_OK) st = check_matrix(fn, "out", out, out_dtype, V, d, ld);
    if (st != VIE_OK) return st;
    const GradWorkspace w = grad_workspace(n);
    if (n > 0 && (workspace == nullptr || workspace_bytes < w.bytes || !aligned_to(workspace, 16)))
        return fail(VIE_ERR_INVALID_ARG, "%s: workspace must be %lld bytes, 16-byte aligned (it has %lld)", fn,
                    static_cast<long long>(w.bytes), static_cast<long long>(workspace == nullptr ? 0 : workspace_bytes));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (!accumulate) {
        const size_t row = static_cast<size_t>(d) * dtype_size(out_dtype);
        const size_t pitch = static_cast<size_t>(ld) * dtype_size(out_dtype);
        e = pitch == row ? cudaMemsetAsync(out, 0, row * V, s) : cudaMemset2DAsync(out, pitch, 0, row, V, s);
        if (e != cudaSuccess) return fail_cuda(e, fn);
    }
    if (n == 0) return VIE_OK;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    uint32_t *key[2], *pos[2];
    for (int i = 0; i < 2; ++i) {
        key[i] = reinterpret_cast<uint32_t *>(ws + w.key) + i * (w.pos / 8);
        pos[i] = reinterpret_cast<uint32_t *>(ws + w.pos) + i * (w.pos / 8);
    }
    SortPass a = {};
    a.counts = reinterpret_cast<uint32_t *>(ws + w.counts);
    a.n = static_cast<uint32_t>(n), a.blocks = w.blocks, a.V = static_cast<uint32_t>(V);
    e = device_flag_word(&a.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    int to = 0;
    for (a.shift = 0; a.shift < 32 && (V >> a.shift) != 0; a.shift += 8, to ^= 1) {
        a.tokens = a.shift == 0 ? tokens : nullptr;
        a.key_in = key[to ^ 1], a.pos_in = pos[to ^ 1], a.key_out = key[to], a.pos_out = pos[to];
        sort_count_kernel<<<w.blocks, kSortThreads, 0, s>>>(a);
        sort_scan_kernel<<<1, 1024, 0, s>>>(a.counts, 256 * w.blocks);
        sort_scatter_kernel<<<w.blocks, kSortThreads, 0, s>>>(a);
    }
    GradParams p = {};
    p.key = key[to ^ 1], p.pos = pos[to ^ 1], p.grad = grad, p.out = out, p.ld_grad = ld_grad, p.ld = ld;
    p.n = a.n, p.V = a.V, p.d = d, p.accumulate = accumulate != 0, p.scale = scale;
    VIE_BY_TYPES(start_grad, dtype, out_dtype, p, s);
    e = cudaGetLastError();
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

}  // extern "C"
