// vie_embed.cu - rows of an embedding table, scaled, and the table's gradient.
// Models with tied embeddings read the same matrix that the output head
// projects on (paper, Section 3: W_out, one row per token).
//
//   lookup    out[i, :] = scale * table[token_i, :]
//   gradient  G[v, :] (+)= scale * sum over i with token_i = v of g[i, :]
//
// Bound by the bytes of the rows.  Measured: lookup of 16384 rows of 1024 bf16
// 8.9 us (a copy of the distinct rows' and the output's bytes would take 7.0), of 32
// rows 1.5; gradient table of 262144 x 640 fp32 from 8192 rows 101 us (100 to
// write it), 16384 rows of 1024 bf16 added to fp32 34 us (12.9; 8 of it to sort
// the tokens, and three launches).
//
// Products and sums are fp32, each result is rounded once.  The gradient's
// sums run in the order of the positions i: the tokens are sorted (stably),
// and each run of equal tokens is summed by itself, so results do not change
// from call to call.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"

namespace vie {

constexpr int kEmbedThreads = 256;
constexpr int kEmbedWarps = kEmbedThreads / 32;
constexpr int kEmbedBlocks = 4;  // blocks of columns that a lookup's warp has in flight

// kW values of a row per lane, as loaded.  kVector: one vector of kW at a 16-byte
// (or 8-byte) address; otherwise 32 apart, value by value: rows of any width,
// pitch and alignment.  Loads do not branch: a lane beyond the row reads the
// row's first values.
template <typename T, int kW, bool kVector>
struct LaneRow {
    using Word = typename std::conditional<!kVector, T, typename std::conditional<sizeof(T) * kW == 8, uint2, uint4>::type>::type;
    static constexpr int kWords = kVector ? 1 : kW;
    static_assert(sizeof(Word) * kWords == sizeof(T) * kW, "all values of a lane");
    Word r[kWords];

    __device__ __forceinline__ static int column(int lane) { return kVector ? lane * kW : lane; }
    // row: the row's start; c: this lane's first column
    __device__ __forceinline__ void load(const T *row, int c, int d) {
#pragma unroll
        for (int x = 0; x < kWords; ++x) {
            const int at = c + 32 * x;
            r[x] = *reinterpret_cast<const Word *>(row + (at < d ? at : 0));
        }
    }
    __device__ __forceinline__ void store(T *row, int c, int d) const {
#pragma unroll
        for (int x = 0; x < kWords; ++x)
            if (c + 32 * x < d) *reinterpret_cast<Word *>(row + c + 32 * x) = r[x];
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int x = 0; x < kWords; ++x) r[x] = Word{};
    }
    __device__ __forceinline__ void values(float *v) const {
#pragma unroll
        for (int x = 0; x < kWords; ++x) split(r[x], v + x * (kW / kWords));
    }
    __device__ __forceinline__ void set(const float *v) {
#pragma unroll
        for (int x = 0; x < kWords; ++x) join(v + x * (kW / kWords), r[x]);
    }

  private:
    static __device__ __forceinline__ uint32_t pack2(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    static __device__ __forceinline__ void split(float x, float *v) { *v = x; }
    static __device__ __forceinline__ void split(__nv_bfloat16 x, float *v) { *v = __bfloat162float(x); }
    static __device__ __forceinline__ void split(const uint2 &x, float *v) {  // four bf16
        v[0] = bf16_lo(x.x), v[1] = bf16_hi(x.x), v[2] = bf16_lo(x.y), v[3] = bf16_hi(x.y);
    }
    static __device__ __forceinline__ void split(const uint4 &x, float *v) { Vec16<T>::unpack(x, v); }
    static __device__ __forceinline__ void join(const float *v, float &x) { x = *v; }
    static __device__ __forceinline__ void join(const float *v, __nv_bfloat16 &x) { x = __float2bfloat16_rn(*v); }
    static __device__ __forceinline__ void join(const float *v, uint2 &x) { x = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])); }
    static __device__ __forceinline__ void join(const float *v, uint4 &x) { x = Vec16<T>::pack(v); }
};

// ---- lookup -----------------------------------------------------------------
// A warp per row and block of columns; bound by the bytes of the rows.

struct EmbedParams {
    const void *table;
    const int32_t *tokens;
    void *out;
    int64_t ld, ld_out, n, V;
    int d;
    float scale;
    uint32_t *flag;
};

template <typename TI, typename TO, int kW, bool kVector>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedParams a) {
    constexpr int kBlock = 32 * kW, kBlocks = kEmbedBlocks;  // a warp's columns at a time, and how many it has in flight
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one
    const int lane = threadIdx.x & 31;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kEmbedWarps + (threadIdx.x >> 5);
    if (i >= a.n) return;
    const int32_t tok = a.tokens[i];
    const bool in = tok >= 0 && tok < a.V;
    if (tok >= a.V && lane == 0 && blockIdx.y == 0) atomicOr(a.flag, kErrTokenIndex);
    const TI *row = static_cast<const TI *>(a.table) + (in ? tok : 0) * a.ld;
    TO *out = static_cast<TO *>(a.out) + i * a.ld_out;
    const int c0 = blockIdx.y * kBlocks * kBlock + LaneRow<TI, kW, kVector>::column(lane);
    LaneRow<TI, kW, kVector> r[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) r[b].load(row, c0 + b * kBlock, a.d);
    if constexpr (std::is_same<TI, TO>::value) {
        if (a.scale == 1.0f) {  // a copy: every bit is kept
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                if (!in) r[b].clear();
                r[b].store(out, c0 + b * kBlock, a.d);
            }
            return;
        }
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        float v[kW];
        r[b].values(v);
#pragma unroll
        for (int w = 0; w < kW; ++w) v[w] = in ? a.scale * v[w] : 0.0f;
        LaneRow<TO, kW, kVector> o;
        o.set(v);
        o.store(out, c0 + b * kBlock, a.d);
    }
}

// ---- tokens in order: entries (token, position) sorted by a key of the token,
// then by position.  Entries of tokens outside [0, V) come last, as token V.

using Entry = uint64_t;
__device__ __forceinline__ Entry make_entry(uint32_t tok, uint32_t pos) { return static_cast<uint64_t>(tok) << 32 | pos; }
__device__ __forceinline__ uint32_t entry_token(Entry e) { return static_cast<uint32_t>(e >> 32); }
__device__ __forceinline__ uint32_t entry_pos(Entry e) { return static_cast<uint32_t>(e); }

// The places of a warp's 32 entries, by digit: *at is where the warp's next
// entry of a lane's digit goes.  Lanes without an entry: NULL, and a digit that
// no other has.
__device__ __forceinline__ uint32_t claim_place(uint32_t *at, uint32_t digit) {
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
    const uint32_t before = __popc(same & ((1u << (threadIdx.x & 31)) - 1u));
    uint32_t place = 0;
    if (at != nullptr) place = *at + before;
    __syncwarp();
    if (at != nullptr && before == 0) *at += __popc(same);
    __syncwarp();
    return place;
}

// Up to kGroupMax tokens: one kernel whose CTAs share nothing.  CTA b takes the
// tokens with tok % 128 = b: it reads all tokens (they come from L2), keeps its
// own in order, counts those of the CTAs before it, which gives the place of
// its output, and sorts its own by tok / 128, 6 bits at a time.  Frequent
// tokens often have neighbouring numbers, so this spreads them; a CTA with
// more entries than fit its shared memory sorts in the output arrays.
// More CTAs, if asked for, clear the gradient table meanwhile.
constexpr int kBuckets = 128, kBucketBits = 7, kDigitBits = 6, kDigits = 1 << kDigitBits;
constexpr int kGroupThreads = 1024, kGroupWarps = kGroupThreads / 32;  // (a lane per warp's count)
static_assert(kGroupWarps == 32, "a warp's lanes hold the warps' counts");
constexpr int kGroupCap = 2048;  // entries per list in shared memory
constexpr int64_t kGroupMax = 131072;

// Counter of a digit in a warp; a warp's counters lie in different banks.
__device__ __forceinline__ int counter(int digit, int warp) { return digit * kGroupWarps + ((warp + digit) & (kGroupWarps - 1)); }

// The counters as exclusive prefix sums, by digit, then by warp.  part: a word per warp.
__device__ __forceinline__ void scan_counters(uint32_t *at, uint32_t *part) {
    constexpr int kPer = kGroupWarps * kDigits / kGroupThreads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t c[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int l = threadIdx.x * kPer + i;
        c[i] = at[counter(l / kGroupWarps, l % kGroupWarps)];
        sum += c[i];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) part[warp] = incl;
    __syncthreads();
    const uint32_t p = part[lane];
    uint32_t run = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? p : 0) + incl - sum;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int l = threadIdx.x * kPer + i;
        at[counter(l / kGroupWarps, l % kGroupWarps)] = run;
        run += c[i];
    }
    __syncthreads();
}

struct GroupParams {
    const int32_t *tokens;
    Entry *sorted, *other;
    uint32_t *flag;
    uint32_t n, V;
    int passes;
    void *fill;          // rows to clear, or NULL
    int64_t fill_pitch;  // bytes
    int64_t fill_row;    // bytes per row, a multiple of 2
};

__device__ __forceinline__ void clear_bytes(unsigned char *p, int64_t bytes, int64_t at, int64_t step) {
    // p and bytes are multiples of 2; the 16-byte middle by vectors
    const int64_t head = min(static_cast<int64_t>(-reinterpret_cast<uintptr_t>(p) & 15u), bytes);
    const int64_t vectors = (bytes - head) / 16;
    for (int64_t i = at; i < vectors; i += step) reinterpret_cast<uint4 *>(p + head)[i] = make_uint4(0, 0, 0, 0);
    const int64_t rest = (bytes - vectors * 16) / 2;  // 2-byte values outside it
    for (int64_t i = at; i < rest; i += step) {
        const int64_t o = 2 * i < head ? 2 * i : 2 * i + vectors * 16;
        *reinterpret_cast<uint16_t *>(p + o) = 0;
    }
}

// Rows of a table, cut into pieces that CTA `part` of `parts` clears.
__device__ __forceinline__ void clear_rows(const GroupParams &a, int64_t part, int64_t parts) {
    unsigned char *p = static_cast<unsigned char *>(a.fill);
    if (a.fill_pitch == a.fill_row) {
        const int64_t bytes = a.fill_row * a.V, per = ((bytes + parts - 1) / parts + 15) / 16 * 16;
        const int64_t lo = min(part * per, bytes), hi = min(lo + per, bytes);
        clear_bytes(p + lo, hi - lo, threadIdx.x, blockDim.x);
    } else {
        const int64_t per = (a.V + parts - 1) / parts, hi = min((part + 1) * per, static_cast<int64_t>(a.V));
        for (int64_t r = part * per + (threadIdx.x >> 5); r < hi; r += blockDim.x >> 5)
            clear_bytes(p + r * a.fill_pitch, a.fill_row, threadIdx.x & 31, 32);
    }
}

__global__ void __launch_bounds__(kGroupThreads, 2) group_tokens_kernel(const GroupParams a) {
    __shared__ Entry list[2][kGroupCap];
    __shared__ uint32_t at[kGroupWarps * kDigits];  // [digit][warp], then where each warp's next entry goes
    __shared__ uint32_t part[kGroupWarps], below;
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one
    if (blockIdx.x >= kBuckets) {
        clear_rows(a, blockIdx.x - kBuckets, gridDim.x - kBuckets);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bucket = blockIdx.x;
    // each warp: a run of tokens, 128 (4 per lane) at a time
    const uint32_t run = ((a.n + kGroupWarps - 1) / kGroupWarps + 127) / 128 * 128;
    const uint32_t lo = warp * run, hi = min(lo + run, a.n);
    const bool aligned = (reinterpret_cast<uintptr_t>(a.tokens) & 15u) == 0;
    auto load4 = [&](uint32_t i, uint32_t *t) {  // tokens i .. i + 3; those outside [0, V): none
        int4 x = make_int4(-1, -1, -1, -1);
        if (aligned && i + 4 <= hi) {
            x = *reinterpret_cast<const int4 *>(a.tokens + i);
        } else {
            if (i < hi) x.x = a.tokens[i];
            if (i + 1 < hi) x.y = a.tokens[i + 1];
            if (i + 2 < hi) x.z = a.tokens[i + 2];
            if (i + 3 < hi) x.w = a.tokens[i + 3];
        }
        t[0] = static_cast<uint32_t>(x.x), t[1] = static_cast<uint32_t>(x.y);
        t[2] = static_cast<uint32_t>(x.z), t[3] = static_cast<uint32_t>(x.w);
    };
    uint32_t mine = 0, before = 0;
    bool beyond = false;
#pragma unroll 4
    for (uint32_t i = lo + 4 * lane; i < hi; i += 128) {
        uint32_t t[4];
        load4(i, t);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const bool in = t[x] < a.V;
            beyond |= !in && t[x] < 0x80000000u;
            mine += in && (t[x] & (kBuckets - 1)) == bucket;
            before += in && (t[x] & (kBuckets - 1)) < bucket;
        }
    }
    if (beyond && bucket == 0) atomicOr(a.flag, kErrTokenIndex);
    mine = __reduce_add_sync(0xFFFFFFFFu, mine);
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    if (tid == 0) below = 0;
    __syncthreads();
    if (lane == 0) {
        part[warp] = mine;
        atomicAdd(&below, before);
    }
    __syncthreads();
    const uint32_t in_warp = part[lane];
    const uint32_t count = __reduce_add_sync(0xFFFFFFFFu, in_warp);
    uint32_t next = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? in_warp : 0);
    Entry *const out = a.sorted + below;
    if (bucket == kBuckets - 1)
        for (uint32_t i = below + count + tid; i < a.n; i += kGroupThreads) a.sorted[i] = make_entry(a.V, 0);
    // the lists that the passes go between; the last one to write is `out`, or is copied there
    const bool small = count <= kGroupCap;
    Entry *from = small ? list[0] : ((a.passes & 1) ? a.other + below : out);
    Entry *to = small ? list[1] : ((a.passes & 1) ? out : a.other + below);
    for (uint32_t i0 = lo; i0 < hi; i0 += 128) {  // the same for all lanes
        const uint32_t i = i0 + 4 * lane;
        uint32_t t[4], m[4], mask[4];
        load4(i, t);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            m[x] = t[x] < a.V && (t[x] & (kBuckets - 1)) == bucket;
            mask[x] = __ballot_sync(0xFFFFFFFFu, m[x]);
        }
        uint32_t o = next;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            o += __popc(mask[x] & ((1u << lane) - 1u));
            next += __popc(mask[x]);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (m[x]) from[o++] = make_entry(t[x], i + x);
    }
    __syncthreads();
    const uint32_t chunk = ((count + kGroupWarps - 1) / kGroupWarps + 31) / 32 * 32;  // per warp
    const uint32_t c0 = min(warp * chunk, count), c1 = min(c0 + chunk, count);
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = kBucketBits + pass * kDigitBits;
        auto digit_of = [&](Entry e) { return (entry_token(e) >> shift) & (kDigits - 1); };
        for (int i = tid; i < kGroupWarps * kDigits; i += kGroupThreads) at[i] = 0;
        __syncthreads();
        for (uint32_t i = c0 + lane; i < c1; i += 32) atomicAdd(&at[counter(digit_of(from[i]), warp)], 1u);
        __syncthreads();
        scan_counters(at, part);
        for (uint32_t i0 = c0; i0 < c1; i0 += 32) {
            const uint32_t i = i0 + lane;
            const bool in = i < c1;
            const Entry e = in ? from[i] : 0;
            const uint32_t place = claim_place(in ? &at[counter(digit_of(e), warp)] : nullptr, in ? digit_of(e) : kDigits);
            if (in) to[place] = e;
        }
        __syncthreads();
        Entry *const swap = from;
        from = to;
        to = swap;
    }
    if (small)
        for (uint32_t i = tid; i < count; i += kGroupThreads) out[i] = from[i];
}

// More tokens: a sort over the whole array, least significant digit first, 8
// bits at a time, in three launches per pass.
constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32, kSortRounds = 8;
constexpr int kSortTile = kSortThreads * kSortRounds;

struct SortPass {
    const int32_t *tokens;  // first pass: the caller's tokens, else NULL
    const Entry *from;
    Entry *to;
    uint32_t *counts;  // [256][blocks]
    uint32_t n, blocks, V, shift;
    uint32_t *flag;
};

__device__ __forceinline__ Entry sort_entry(const SortPass &a, uint32_t i) {
    if (a.tokens == nullptr) return a.from[i];
    const uint32_t tok = static_cast<uint32_t>(a.tokens[i]);
    return make_entry(tok < a.V ? tok : a.V, i);
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
        atomicAdd(&count[(entry_token(sort_entry(a, i)) >> a.shift) & 255u], 1u);
    }
    __syncthreads();
    a.counts[static_cast<size_t>(threadIdx.x) * a.blocks + blockIdx.x] = count[threadIdx.x];
}

// Exclusive prefix sums over counts[0 .. total), in place; one CTA, eight
// counters per thread at a time (total is a multiple of 8, counts 16-byte aligned).
__global__ void __launch_bounds__(1024) sort_scan_kernel(uint32_t *counts, uint32_t total) {
    __shared__ uint32_t part[32];
    uint32_t base = 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t i0 = 0; i0 < total; i0 += 8 * 1024) {
        const uint32_t i = i0 + 8 * threadIdx.x;
        uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (i < total) {
            x[0] = reinterpret_cast<const uint4 *>(counts + i)[0];
            x[1] = reinterpret_cast<const uint4 *>(counts + i)[1];
        }
        const uint32_t v[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
        uint32_t sum = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[k];
        uint32_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) part[warp] = incl;
        __syncthreads();
        const uint32_t p = part[lane];
        uint32_t run = base + __reduce_add_sync(0xFFFFFFFFu, lane < warp ? p : 0) + incl - sum;
        base += __reduce_add_sync(0xFFFFFFFFu, p);
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k] = run;
            run += v[k];
        }
        if (i < total) {
            reinterpret_cast<uint4 *>(counts + i)[0] = make_uint4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<uint4 *>(counts + i)[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
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
        if (i < a.n) atomicAdd(&at[warp][(entry_token(sort_entry(a, i)) >> a.shift) & 255u], 1u);
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
        const Entry e = in ? sort_entry(a, i) : 0;
        const uint32_t digit = (entry_token(e) >> a.shift) & 255u;
        const uint32_t to = claim_place(in ? &at[warp][digit] : nullptr, in ? digit : 256u);
        if (in) a.to[to] = e;
    }
}

// ---- sums over the runs of equal tokens -------------------------------------
// A warp takes `chunk` sorted entries and a block of columns and adds the rows
// up in order, eight of them in flight, and with them the rows of the table
// that they are added to.  A run of a token that goes on beyond the chunk at
// either end leaves the chunk's part of its sum in the workspace (0: of a run
// that began before the chunk, 1: of one that begins in it), and
// join_runs_kernel adds the parts up in order.

struct GradParams {
    const Entry *sorted;
    const void *grad;
    void *out;
    float *parts;  // [chunks][2][d]
    int64_t ld_grad, ld;
    uint32_t n, V, chunk;
    int d, accumulate;
    float scale;
};

// Additions to an fp32 table are made in L2: a row has one of them per call, so
// their order does not matter, and the warp need not wait for the row (16384
// tokens x 1024: 43 us with the rows read, 35 without).  They flush results
// below 2^-126 to 0.  A bf16 table's rows are read, to round the sum once.
template <typename T>
constexpr bool kAddsInL2 = std::is_same<T, float>::value;

// scale * sum (+ what was there, if that was read) into a row of the table.
template <typename T, int kW, bool kVector>
__device__ __forceinline__ void put_row(const GradParams &a, T *row, int c, const float *sum,
                                        const LaneRow<T, kW, kVector> &there) {
    float v[kW];
    if constexpr (kAddsInL2<T>) {
        if (a.accumulate) {
            if constexpr (kVector) {
                static_assert(kW == 4, "a vector of fp32");
                if (c < a.d)
                    atomicAdd(reinterpret_cast<float4 *>(row + c), make_float4(a.scale * sum[0], a.scale * sum[1],
                                                                              a.scale * sum[2], a.scale * sum[3]));
            } else {
#pragma unroll
                for (int w = 0; w < kW; ++w)
                    if (c + 32 * w < a.d) atomicAdd(row + c + 32 * w, a.scale * sum[w]);
            }
            return;
        }
    } else {
        if (a.accumulate) there.values(v);
    }
#pragma unroll
    for (int w = 0; w < kW; ++w) v[w] = !kAddsInL2<T> && a.accumulate ? fmaf(a.scale, sum[w], v[w]) : a.scale * sum[w];
    LaneRow<T, kW, kVector> o;
    o.set(v);
    o.store(row, c, a.d);
}

// A lane's columns of a row of fp32 parts.
template <int kW, bool kVector>
struct PartRow {
    __device__ __forceinline__ static int column(int c, int w) { return kVector ? c + w : c + 32 * w; }
};

template <typename TI, typename TO, int kW, bool kVector>
__global__ void __launch_bounds__(kEmbedThreads, 2) sum_runs_kernel(const GradParams a) {
    constexpr int kRows = 8;
    griddep_launch_dependents();
    griddep_wait();
    const int lane = threadIdx.x & 31;
    const uint32_t chunk = blockIdx.x * kEmbedWarps + (threadIdx.x >> 5);
    const uint32_t lo = chunk * a.chunk;
    if (lo >= a.n) return;
    const uint32_t hi = min(lo + a.chunk, a.n);
    const int c = blockIdx.y * 32 * kW + LaneRow<TI, kW, kVector>::column(lane);
    float acc[kW];
    auto restart = [&] {
#pragma unroll
        for (int w = 0; w < kW; ++w) acc[w] = 0.0f;
    };
    auto leave_part = [&](int which) {
        float *part = a.parts + (static_cast<int64_t>(chunk) * 2 + which) * a.d;
#pragma unroll
        for (int w = 0; w < kW; ++w)
            if (PartRow<kW, kVector>::column(c, w) < a.d) part[PartRow<kW, kVector>::column(c, w)] = acc[w];
    };
    restart();
    bool from_before = lo > 0 && entry_token(a.sorted[lo - 1]) == entry_token(a.sorted[lo]);
    bool open = false;
    for (uint32_t i0 = lo; i0 < hi; i0 += 32) {
        const uint32_t i = i0 + lane;
        const Entry e = i < hi ? a.sorted[i] : make_entry(a.V, 0);
        const bool valid = entry_token(e) < a.V;  // the empty slots come last
        const uint32_t next = i + 1 < a.n ? entry_token(a.sorted[i + 1]) : a.V;
        const uint32_t ends = __ballot_sync(0xFFFFFFFFu, valid && entry_token(e) != next);
        const int count = __popc(__ballot_sync(0xFFFFFFFFu, valid));
        for (int r0 = 0; r0 < count; r0 += kRows) {
            LaneRow<TI, kW, kVector> row[kRows];
            LaneRow<TO, kW, kVector> there[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) {  // (beyond `count`: row 0, not used)
                const uint32_t pos = __shfl_sync(0xFFFFFFFFu, entry_pos(e), r0 + u);
                row[u].load(static_cast<const TI *>(a.grad) + pos * a.ld_grad, c, a.d);
            }
            if (!kAddsInL2<TO> && a.accumulate) {
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const int64_t tok = __shfl_sync(0xFFFFFFFFu, entry_token(e), r0 + u);
                    if (ends >> (r0 + u) & 1u) there[u].load(static_cast<const TO *>(a.out) + tok * a.ld, c, a.d);
                }
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                if (r0 + u >= count) break;
                float v[kW];
                row[u].values(v);
#pragma unroll
                for (int w = 0; w < kW; ++w) acc[w] += v[w];
                open = true;
                if (ends >> (r0 + u) & 1u) {
                    const int64_t tok = __shfl_sync(0xFFFFFFFFu, entry_token(e), r0 + u);
                    if (from_before) leave_part(0);
                    else put_row<TO, kW, kVector>(a, static_cast<TO *>(a.out) + tok * a.ld, c, acc, there[u]);
                    from_before = open = false;
                    restart();
                }
            }
        }
        if (count < 32) break;
    }
    if (open) leave_part(from_before ? 0 : 1);
}

// A warp per chunk and block of columns: if a run begins in the chunk and goes on
// beyond it, the sum of its parts.  Runs of many parts (a very frequent token)
// are shared by the warps of the CTA, each of which adds up consecutive parts.
template <typename TO, int kW, bool kVector>
__global__ void __launch_bounds__(kEmbedThreads) join_runs_kernel(const GradParams a) {
    constexpr int kParts = 8;  // in flight
    constexpr uint32_t kOwn = 16;  // parts that a warp adds up alone
    __shared__ uint32_t run_token[kEmbedWarps], run_parts[kEmbedWarps];
    __shared__ float share[kEmbedWarps][32 * kW];
    griddep_launch_dependents();
    griddep_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.y * 32 * kW + LaneRow<TO, kW, kVector>::column(lane);
    const uint32_t chunk0 = blockIdx.x * kEmbedWarps, chunk = chunk0 + warp;
    // parts lo .. hi - 1 of the run that begins in chunk `begin` (part 0 in slot 1, the others in slots 0)
    auto add_parts = [&](uint32_t begin, uint32_t lo, uint32_t hi, float *acc) {
#pragma unroll
        for (int w = 0; w < kW; ++w) acc[w] = 0.0f;
        for (uint32_t j = lo; j < hi; j += kParts) {
            float v[kParts][kW];
#pragma unroll
            for (int u = 0; u < kParts; ++u) {
                const uint32_t x = min(j + u, hi - 1);
                const float *part = a.parts + (2 * (static_cast<int64_t>(begin) + x) + (x == 0)) * a.d;
#pragma unroll
                for (int w = 0; w < kW; ++w) {
                    const int col = PartRow<kW, kVector>::column(c, w);
                    v[u][w] = part[col < a.d ? col : 0];
                }
            }
#pragma unroll
            for (int u = 0; u < kParts; ++u)
                if (j + u < hi) {
#pragma unroll
                    for (int w = 0; w < kW; ++w) acc[w] += v[u][w];
                }
        }
    };
    auto put = [&](uint32_t tok, const float *acc) {
        TO *const row = static_cast<TO *>(a.out) + static_cast<int64_t>(tok) * a.ld;
        LaneRow<TO, kW, kVector> there;
        if (!kAddsInL2<TO> && a.accumulate) there.load(row, c, a.d);
        put_row<TO, kW, kVector>(a, row, c, acc, there);
    };
    // the run that begins in this warp's chunk and goes on, and its parts
    const uint64_t lo = static_cast<uint64_t>(chunk) * a.chunk, hi = lo + a.chunk;
    uint32_t tok = a.V, parts = 0;
    if (hi < a.n) {
        const uint32_t last = entry_token(a.sorted[hi - 1]), after = entry_token(a.sorted[hi]);
        const uint32_t first = entry_token(a.sorted[lo]), before = lo > 0 ? entry_token(a.sorted[lo - 1]) : a.V;
        if (last < a.V && after == last && !(first == last && before == last)) tok = last;
    }
    if (tok < a.V) {
        parts = 1;
        auto begins = [&](uint64_t ch) {  // whether chunk ch begins with the run's token
            const uint64_t at = ch * a.chunk;
            return at < a.n && entry_token(a.sorted[at < a.n ? at : 0]) == tok;
        };
        while (true) {  // 32 chunks at a time, 1024 where all of those belong to it
            const uint64_t next = static_cast<uint64_t>(chunk) + parts;
            const uint32_t near = __ballot_sync(0xFFFFFFFFu, begins(next + lane));
            if (near != 0xFFFFFFFFu) {
                parts += __ffs(~near) - 1;
                break;
            }
            const uint32_t far = __ballot_sync(0xFFFFFFFFu, begins(next + 32 * lane + 31));
            parts += far == 0xFFFFFFFFu ? 1024 : 32 * (__ffs(~far) - 1);
        }
        if (parts <= kOwn) {
            float acc[kW];
            add_parts(chunk, 0, parts, acc);
            put(tok, acc);
        }
    }
    if (lane == 0) run_token[warp] = tok, run_parts[warp] = parts;
    if (!__syncthreads_or(parts > kOwn)) return;
    for (int r = 0; r < kEmbedWarps; ++r) {
        const uint32_t m = run_parts[r];
        if (m <= kOwn) continue;
        const uint32_t per = (m + kEmbedWarps - 1) / kEmbedWarps;
        float acc[kW];
        add_parts(chunk0 + r, min(warp * per, m), min((warp + 1) * per, m), acc);
#pragma unroll
        for (int w = 0; w < kW; ++w) share[warp][w * 32 + lane] = acc[w];
        __syncthreads();
        if (warp == r) {
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                acc[w] = 0.0f;
                for (int x = 0; x < kEmbedWarps; ++x) acc[w] += share[x][w * 32 + lane];
            }
            put(run_token[r], acc);
        }
        __syncthreads();
    }
}

constexpr int64_t kChunkMin = 8;

// Workspace: the entries twice, the counts of the large sort, the parts of runs.
struct GradWorkspace {
    uint32_t blocks, chunk, chunks;
    int64_t entries, counts, parts, bytes;  // offsets (entries: of the second array)
};

static GradWorkspace grad_workspace(int64_t n, int32_t d) {
    auto round_up = [](int64_t v) { return (v + 255) / 256 * 256; };
    GradWorkspace w;
    w.blocks = n > kGroupMax ? static_cast<uint32_t>((n + kSortTile - 1) / kSortTile) : 0;
    // Short chunks: many rows in flight from few tokens (2048 x 1024: 11.6 us in
    // chunks of 8, 13.6 of 16).  Longer ones leave fewer parts (65536 x 1024: 89 us
    // in chunks of 64, 92 of 16), as long as there are warps enough.
    const int64_t most = std::max<int64_t>(1024, 8192 / ((d + 127) / 128));
    w.chunk = kChunkMin;
    while (n / w.chunk > most) w.chunk *= 2;
    w.chunks = static_cast<uint32_t>((n + w.chunk - 1) / w.chunk);
    w.entries = round_up(8 * n);
    w.counts = 2 * w.entries;
    w.parts = w.counts + round_up(int64_t(w.blocks) * 1024);
    // never more for fewer tokens: a program keeps one for its longest batch
    w.bytes = w.parts + std::min<int64_t>((n + kChunkMin - 1) / kChunkMin, most + 1) * 8 * d;
    return w;
}

// Launches a kernel that may start while the one before it ends.
template <typename F, typename... A>
static cudaError_t chain(F kernel, dim3 grid, int threads, cudaStream_t s, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename TI, typename TO, int kW, bool kVector>
static cudaError_t start_sums(const GradParams &p, uint32_t chunks, cudaStream_t s) {
    const dim3 grid((chunks + kEmbedWarps - 1) / kEmbedWarps, static_cast<unsigned>((p.d + 32 * kW - 1) / (32 * kW)));
    cudaError_t e = chain(sum_runs_kernel<TI, TO, kW, kVector>, grid, kEmbedThreads, s, p);
    if (e == cudaSuccess && chunks > 1) e = chain(join_runs_kernel<TO, kW, kVector>, grid, kEmbedThreads, s, p);
    return e;
}
template <typename TI, typename TO, int kW, bool kVector>
static cudaError_t start_embed(const EmbedParams &p, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>((p.n + kEmbedWarps - 1) / kEmbedWarps),
                    static_cast<unsigned>((p.d + kEmbedBlocks * 32 * kW - 1) / (kEmbedBlocks * 32 * kW)));
    return chain(embed_kernel<TI, TO, kW, kVector>, grid, kEmbedThreads, s, p);
}

// How rows of two matrices are read and written: 8 values per lane (a 16-byte
// vector) if both are bf16 and rows are wide enough for a warp, 4 otherwise (60000 rows of
// 1024, bf16 to fp32: 43 us; 62 with 8, whose two fp32 vectors per lane lie 32
// bytes apart); value by value where addresses do not allow either.
enum class Access { kWide, kNarrow, kValues };
static Access access_of(const void *a, vie_dtype ta, int64_t lda, const void *b, vie_dtype tb, int64_t ldb, int d) {
    auto fits = [&](const void *p, vie_dtype t, int64_t ld, int w) {
        const int bytes = w * dtype_size(t);
        return aligned_to(p, static_cast<uintptr_t>(bytes)) && ld * dtype_size(t) % bytes == 0 && d % w == 0;
    };
    if (ta == VIE_DTYPE_BF16 && tb == VIE_DTYPE_BF16 && d > 128 && fits(a, ta, lda, 8) && fits(b, tb, ldb, 8))
        return Access::kWide;
    return fits(a, ta, lda, 4) && fits(b, tb, ldb, 4) ? Access::kNarrow : Access::kValues;
}

// f<TI, TO, kW, kVector>(...) for two storage types and how rows are accessed.
#define VIE_BY_ACCESS(f, TI, TO, access, ...) \
    ((access) == Access::kNarrow ? f<TI, TO, 4, true>(__VA_ARGS__) : f<TI, TO, 4, false>(__VA_ARGS__))
#define VIE_BY_TYPES(f, in, out, access, ...)                                                       \
    ((access) == Access::kWide  ? f<__nv_bfloat16, __nv_bfloat16, 8, true>(__VA_ARGS__)             \
     : (in) == VIE_DTYPE_BF16                                                                       \
         ? ((out) == VIE_DTYPE_BF16 ? VIE_BY_ACCESS(f, __nv_bfloat16, __nv_bfloat16, access, __VA_ARGS__) \
                                    : VIE_BY_ACCESS(f, __nv_bfloat16, float, access, __VA_ARGS__))  \
         : ((out) == VIE_DTYPE_BF16 ? VIE_BY_ACCESS(f, float, __nv_bfloat16, access, __VA_ARGS__)   \
                                    : VIE_BY_ACCESS(f, float, float, access, __VA_ARGS__)))

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
    const Access access = access_of(table, dtype, ld, out, out_dtype, ld_out, d);
    e = VIE_BY_TYPES(start_embed, dtype, out_dtype, access, p, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_embed_grad_workspace(int64_t n, int64_t V, int32_t d, int64_t *bytes) {
    const char *fn = "vie_embed_grad_workspace";
    alignas(4) static const int32_t some = 0;
    const vie_status st = check_embed(fn, &some, n, V, d);
    if (st != VIE_OK) return st;
    if (bytes == nullptr) return fail(VIE_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    *bytes = grad_workspace(n, d).bytes;
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
    const GradWorkspace w = grad_workspace(n, d);
    if (n > 0 && (workspace == nullptr || workspace_bytes < w.bytes || !aligned_to(workspace, 16)))
        return fail(VIE_ERR_INVALID_ARG, "%s: workspace must be %lld bytes, 16-byte aligned (it has %lld)", fn,
                    static_cast<long long>(w.bytes), static_cast<long long>(workspace == nullptr ? 0 : workspace_bytes));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t row = int64_t(d) * dtype_size(out_dtype), pitch = ld * dtype_size(out_dtype);
    const bool grouped = n <= kGroupMax;
    cudaError_t e = cudaSuccess;
    if (!accumulate && (n == 0 || !grouped)) {
        e = pitch == row ? cudaMemsetAsync(out, 0, static_cast<size_t>(row * V), s)
                         : cudaMemset2DAsync(out, static_cast<size_t>(pitch), 0, static_cast<size_t>(row),
                                             static_cast<size_t>(V), s);
        if (e != cudaSuccess) return fail_cuda(e, fn);
    }
    if (n == 0) return VIE_OK;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    Entry *entries[2] = {reinterpret_cast<Entry *>(ws), reinterpret_cast<Entry *>(ws + w.entries)};
    uint32_t *flag = nullptr;
    e = device_flag_word(&flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    int sorted = 0;
    if (grouped) {
        GroupParams g = {};
        g.tokens = tokens, g.sorted = entries[0], g.other = entries[1], g.flag = flag;
        g.n = static_cast<uint32_t>(n), g.V = static_cast<uint32_t>(V);
        while (((V - 1) >> kBucketBits) >> (g.passes * kDigitBits)) ++g.passes;
        unsigned clearing = 0;
        if (!accumulate) {
            g.fill = out, g.fill_pitch = pitch, g.fill_row = row;
            clearing = static_cast<unsigned>(std::min<int64_t>(4096, (row * V + (1 << 17) - 1) >> 17));  // 128 KB each
        }
        e = chain(group_tokens_kernel, dim3(kBuckets + clearing), kGroupThreads, s, g);
    } else {
        SortPass a = {};
        a.counts = reinterpret_cast<uint32_t *>(ws + w.counts);
        a.n = static_cast<uint32_t>(n), a.blocks = w.blocks, a.V = static_cast<uint32_t>(V), a.flag = flag;
        for (a.shift = 0; a.shift < 32 && (V >> a.shift) != 0; a.shift += 8) {
            a.tokens = a.shift == 0 ? tokens : nullptr;
            a.from = entries[sorted], a.to = entries[sorted ^ 1];
            sorted ^= 1;
            sort_count_kernel<<<w.blocks, kSortThreads, 0, s>>>(a);
            sort_scan_kernel<<<1, 1024, 0, s>>>(a.counts, 256 * w.blocks);
            sort_scatter_kernel<<<w.blocks, kSortThreads, 0, s>>>(a);
        }
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return fail_cuda(e, fn);
    GradParams p = {};
    p.sorted = entries[sorted], p.grad = grad, p.out = out, p.parts = reinterpret_cast<float *>(ws + w.parts);
    p.ld_grad = ld_grad, p.ld = ld, p.n = static_cast<uint32_t>(n), p.V = static_cast<uint32_t>(V), p.chunk = w.chunk;
    p.d = d, p.accumulate = accumulate != 0, p.scale = scale;
    const Access access = access_of(grad, dtype, ld_grad, out, out_dtype, ld, d);
    e = VIE_BY_TYPES(start_sums, dtype, out_dtype, access, p, w.chunks, s);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

}  // extern "C"
