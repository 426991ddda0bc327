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
// and the draw is the first token with C_i > floor(u M): twice the shortest
// prefix of a given mass, nothing is ranked as a whole.
// top_p and u count in steps of 2^-24 (top_p rounded up, u down).
//
// A cluster of CTAs takes a row; each reads its slice once from memory and a few
// times more from L2:
//   1. the maximum.  With a top_k, the threads' own maxima give a logit that at
//      least top_k tokens reach: those that do go to the first CTA, which
//      does the rest.
//   2. the masses S and Q, and about those of the tokens down to four depths
//      (max z - z) / T;
//   3. a histogram of masses over 1024 steps of depth, of the tokens in the least of
//      these ranges that holds the prefix; the bin in which it ends follows;
//   4. the tokens of that bin go to the first CTA, which finds the prefix's last
//      one exactly, by finer histograms and comparisons (sorting them all took 10 us
//      more for bins of a thousand).
// A bin of more tokens than fit is cut further by the logits' ranking keys.
//
// Reading a row once would take 10 us for 64 fp32 rows of 262144; measured there, on
// normal logits of spread 2.5: 39 us if all rows have a top_k of 50 (T 0.8), 70 with
// a min_p of 0.05, 77 without a filter, 93 at top_p 0.9 (T 0.8; 107 at T 1.2, 152 at
// 2.5, where the prefix is more than half of all tokens), 66 for a mixture: the
// exponentials of all values, 28 instructions each, then the histogram.  bf16 rows
// take about as long (32, 64, 74, 89; 117 at T 1.2).  One row of 151936: 10.6 us with
// that top_k, 17 to 26 with the others (bf16 to 30), a chain of seven exchanges
// between its CTAs of about a microsecond each.
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
    int64_t ld, batch;
    int V;
    bool by_work;  // rows of more work first
};

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;
constexpr int kBins = 1024;       // two per thread
constexpr int kBinsPerUnit = 36;  // bins per unit of (max z - z) / T: weights are 0 from 27.8 units on
constexpr int kCap = 4096;        // tokens that the first CTA ranks
constexpr int kFew = 256;         // tokens that are compared with each other
static_assert(kFew <= kSampleThreads, "a thread per token");
constexpr int kMaxSplit = 16;     // CTAs per row, at most
constexpr uint64_t kOne = 1ull << 40;  // the best token's weight
static_assert(kBins == 2 * kSampleThreads, "two bins per thread");

// floor(mass * count / 2^24), and whether that left a rest; mass < 2^62.
__device__ __forceinline__ uint64_t share_of(uint64_t mass, uint32_t count, bool *rest) {
    const uint64_t low = (mass & 0xFFFFFFu) * count;
    *rest = (low & 0xFFFFFFu) != 0;
    return (mass >> 24) * count + (low >> 24);
}

struct Weigh {
    float best, inv;
    bool warm;
    // -(z - max z) / T >= 0: nothing to draw from (-inf, NaN) is +inf
    __device__ __forceinline__ float depth(float z) const {
        if (!(z > -INFINITY)) return INFINITY;
        if (z == best) return 0.0f;
        const float d = -((z - best) * inv);
        return warm && d >= 0.0f ? d : INFINITY;
    }
    // floor(2^40 exp(-depth)), from the bits of the fp32 exponential
    static __device__ __forceinline__ uint64_t of_depth(float depth) {
        const uint32_t e = __float_as_uint(expf(-depth));
        const int shift = static_cast<int>(e >> 23) - (127 + 23 - 40);
        const uint64_t mantissa = (e & 0x7FFFFFu) | 0x800000u;
        return shift >= 0 ? mantissa << shift : (shift > -24 ? mantissa >> -shift : 0);
    }
    __device__ __forceinline__ uint64_t operator()(float z) const { return of_depth(depth(z)); }
    // Larger logits never have larger bins; kBins and more: weight 0.
    static __device__ __forceinline__ int bin_of(float depth) {
        return static_cast<int>(fminf(depth * kBinsPerUnit, static_cast<float>(kBins)));
    }
};

// floor(2^40 e) = 2^20 high + low for 0 <= e <= 1: two additions that cut off what
// is below 2^-20 and 2^-40.
__device__ __forceinline__ void split_weight(float e, uint32_t *high, uint32_t *low) {
    const float t = __fadd_rz(e, 8.0f), t2 = __fadd_rz(e - (t - 8.0f), 7.62939453125e-06f);  // 2^-17
    *high = __float_as_uint(t) - 0x41000000u;
    *low = __float_as_uint(t2) - 0x37000000u;
}

struct SampleSmem {
    uint64_t cand[kCap];         // of the first CTA: tokens to rank, as ranking keys
    uint64_t few[kFew], few_mass[kFew];
    uint64_t before[kBins];      // of the first CTA: what the bins before this one amount to
    uint32_t hist[3][kBins];     // counts in [0], or masses in parts: their low 14 bits, the next 14, the rest
    uint64_t slots[2][kMaxSplit][4];
    uint64_t warp_sums[kSampleWarps];
    float scratch[kSampleWarps];
    float edge[4], bin_edge[4];  // least logits of the depths; of two bins, and of those before each
    float4 depth_sums[kSampleWarps];
    uint64_t told[2][3];         // of the first CTA: what it has found, for all
    uint64_t found[2], total;    // of the first CTA: what its threads have found, and all bins' amount
    uint32_t cand_count, few_count, place;
};

// What a CTA does by itself.
struct SampleBlock {
    SampleSmem &sm;
    Weigh weigh;

    __device__ __forceinline__ SampleBlock(SampleSmem &sm_, const Weigh &weigh_) : sm(sm_), weigh(weigh_) {}

    __device__ __forceinline__ uint64_t weight_of(uint64_t key) const { return key == 0 ? 0 : weigh(key_value(key)); }
    __device__ __forceinline__ uint64_t block_sum(uint64_t v) const {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) v += shfl_xor_u64(v, o);
        __syncthreads();
        if (lane == 0) sm.warp_sums[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < kSampleWarps ? sm.warp_sums[lane] : 0;
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) v += shfl_xor_u64(v, o);
        return v;
    }
    // Sum of the threads before this one; *total: of all.
    __device__ __forceinline__ uint64_t block_before(uint64_t v, uint64_t *total) const {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        uint64_t incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t x = shfl_up_u64(incl, o);
            if (lane >= o) incl += x;
        }
        __syncthreads();
        if (lane == 31) sm.warp_sums[warp] = incl;
        __syncthreads();
        uint64_t run = incl - v, all = 0;
#pragma unroll
        for (int w = 0; w < kSampleWarps; ++w) {
            run += w < warp ? sm.warp_sums[w] : 0;
            all += sm.warp_sums[w];
        }
        *total = all;
        return run;
    }
    __device__ __forceinline__ uint64_t block_max_u64(uint64_t v) const {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) v = max(v, shfl_xor_u64(v, o));
        __syncthreads();
        if (lane == 0) sm.warp_sums[threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < kSampleWarps ? sm.warp_sums[lane] : 0;
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) v = max(v, shfl_xor_u64(v, o));
        return v;
    }
    __device__ __forceinline__ void forget() const {  // what is looked for is always there; never an index of chance
        __syncthreads();
        if (threadIdx.x == 0) sm.found[0] = sm.found[1] = 0, sm.few_count = 0;
        __syncthreads();
    }
    __device__ __forceinline__ void clear_hist() const {
        for (int b = threadIdx.x; b < kBins; b += kSampleThreads) sm.hist[0][b] = sm.hist[1][b] = sm.hist[2][b] = 0;
        __syncthreads();
    }
    // A slice has at most 2^18 values, and w is at most 2^40: the sums of the
    // parts stay below 2^32 (2^18 (2^14 - 1), and 2^18 2^12).
    __device__ __forceinline__ void count_mass(int bin, uint64_t w) const {
        const uint32_t a = static_cast<uint32_t>(w) & 0x3FFFu, b = static_cast<uint32_t>(w >> 14) & 0x3FFFu;
        const uint32_t c = static_cast<uint32_t>(w >> 28);
        if (a) atomicAdd(&sm.hist[0][bin], a);
        if (b) atomicAdd(&sm.hist[1][bin], b);
        if (c) atomicAdd(&sm.hist[2][bin], c);
    }
    // The same for the weight of an exponential (fewer instructions).
    __device__ __forceinline__ void count_weight(int bin, float e) const {
        uint32_t high, low;
        split_weight(e, &high, &low);
        const uint32_t b = (low >> 14 | high << 6) & 0x3FFFu, c = high >> 8;
        atomicAdd(&sm.hist[0][bin], low & 0x3FFFu);
        if (b) atomicAdd(&sm.hist[1][bin], b);
        if (c) atomicAdd(&sm.hist[2][bin], c);
    }
};

// First CTA: of its n candidates those with keys low .. high, best first: the
// key of the first one at which the running mass (or number), from `before`
// on, reaches target, and that mass, in all threads; they have that much.
// Nothing is sorted: histograms over the keys leave a few candidates, which are
// compared with each other.  (Keys differ, so this ends.)
__device__ __forceinline__ uint64_t first_to_reach(SampleSmem &sm, Weigh weigh, bool by_count, int n, uint64_t low, uint64_t high,
                                                uint64_t before, uint64_t target, uint64_t *mass) {
    const SampleBlock block(sm, weigh);
    const int tid = threadIdx.x;
    auto in = [&](uint64_t key) { return key >= low && key <= high; };
    auto mass_of = [&](uint64_t key) { return by_count ? static_cast<uint64_t>(1) : block.weight_of(key); };
    const uint64_t *few = sm.cand;
    int left = n;
    while (left > kFew) {
        const int bits = 64 - __clzll(static_cast<long long>(high - low)), shift = bits > 10 ? bits - 10 : 0;
        block.forget();
        block.clear_hist();
        for (int i = tid; i < n; i += kSampleThreads) {
            const uint64_t key = sm.cand[i];
            if (!in(key)) continue;
            const int b = static_cast<int>((high - key) >> shift);
            if (by_count) atomicAdd(&sm.hist[0][b], 1u);
            else block.count_mass(b, mass_of(key));
        }
        __syncthreads();
        uint64_t v[2], total;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int b = 2 * tid + x;
            v[x] = sm.hist[0][b] + (static_cast<uint64_t>(sm.hist[1][b]) << 14) + (static_cast<uint64_t>(sm.hist[2][b]) << 28);
        }
        uint64_t run = before + block.block_before(v[0] + v[1], &total);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (run < target && target <= run + v[x]) sm.found[0] = 2 * tid + x, sm.found[1] = run;
            run += v[x];
        }
        __syncthreads();
        before = sm.found[1];
        high -= sm.found[0] << shift;
        const uint64_t width = (static_cast<uint64_t>(1) << shift) - 1;
        if (high - low > width) low = high - width;
        for (int i = tid; i < n; i += kSampleThreads) {
            const uint64_t key = sm.cand[i];
            if (!in(key)) continue;
            const uint32_t at = atomicAdd(&sm.few_count, 1u);
            if (at < kFew) sm.few[at] = key;
        }
        __syncthreads();
        left = static_cast<int>(sm.few_count);
        few = sm.few;
    }
    block.forget();
    uint64_t own = 0, mine = 0;
    if (tid < left) {
        own = few[tid];
        mine = in(own) ? mass_of(own) : 0;
        sm.few_mass[tid] = mine;
    }
    __syncthreads();
    if (tid < left) {
        uint64_t after = before;
#pragma unroll 8
        for (int x = 0; x < left; ++x) after += few[x] >= own ? sm.few_mass[x] : 0;
        if (after - mine < target && target <= after) sm.found[0] = tid, sm.found[1] = after;
    }
    __syncthreads();
    *mass = sm.found[1];
    return few[sm.found[0]];
}

// What all CTAs of a row know and do together.
template <typename T>
struct SampleRow : SampleBlock {
    const Slice<T> sl;
    int slices, rank;
    int turn, tale;  // of the exchanges, and of what the first CTA tells
    bool crowded;    // the last prefix has taken the histograms
    uint64_t key_low, key_high;

    __device__ __forceinline__ SampleRow(SampleSmem &sm_, const T *row, int V, int log2_slices, int rank_)
        : SampleBlock(sm_, Weigh{0.0f, 0.0f, false}), sl(row, V, log2_slices, rank_), slices(1 << log2_slices), rank(rank_), turn(0), tale(0), crowded(false), key_low(0), key_high(0) {}

    __device__ __forceinline__ void sync() const {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    // f(z, index) for the slice's values, in no order.
    template <typename F>
    __device__ __forceinline__ void each(const F &f) const {
        constexpr int kVec = Slice<T>::kVec, U = 2;
        const uint4 *const zv = sl.vectors();
        auto of_vector = [&](const uint4 &raw, int i) {
            float v[kVec];
            Vec16<T>::unpack(raw, v);
#pragma unroll
            for (int x = 0; x < kVec; ++x) f(v[x], sl.e0 + i * kVec + x);
        };
        for (int i = sl.lo + threadIdx.x; i < sl.hi; i += U * kSampleThreads) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kSampleThreads < sl.hi) raw[u] = zv[i + u * kSampleThreads];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kSampleThreads < sl.hi) of_vector(raw[u], i + u * kSampleThreads);
        }
        if (sl.has_edge()) of_vector(sl.load_edge(), sl.edge());  // (values outside the row: -inf)
    }
    // The same for the values of `least` and more, and below `limit` (NaN: no
    // limit), if any: a vector without one of `least` is passed over at once.
    template <typename F>
    __device__ __forceinline__ void each_above(float least, float limit, const F &f) const {
        constexpr int kVec = Slice<T>::kVec, U = 4;
        const uint4 *const zv = sl.vectors();
        auto of_vector = [&](const uint4 &raw, int i) {
            typename Vec16<T>::Max top;
            top.add(raw);
            if (!(top.top() >= least)) return;
            float v[kVec];
            Vec16<T>::unpack(raw, v);
#pragma unroll
            for (int x = 0; x < kVec; ++x)
                if (v[x] >= least && !(v[x] >= limit)) f(v[x], sl.e0 + i * kVec + x);
        };
        for (int i = sl.lo + threadIdx.x; i < sl.hi; i += U * kSampleThreads) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kSampleThreads < sl.hi) raw[u] = zv[i + u * kSampleThreads];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kSampleThreads < sl.hi) of_vector(raw[u], i + u * kSampleThreads);
        }
        if (sl.has_edge()) of_vector(sl.load_edge(), sl.edge());
    }
    // f(z) for the values of `least` and more, 32 at a time: those that a warp
    // finds wait in a queue until they fill it.  The candidates' memory is used.
    template <typename F>
    __device__ __forceinline__ void each_above_in_turn(float least, const F &f) const {
        constexpr int kVec = Slice<T>::kVec, U = 4;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        float *const queue = reinterpret_cast<float *>(sm.cand) + warp * (2 * kCap / kSampleWarps);  // 512 values
        static_assert(2 * kCap / kSampleWarps >= 32 * 8 + 32, "a vector of every lane, and what waits");
        int waiting = 0;  // the same in all lanes
        auto work = [&] {
            __syncwarp();
            while (waiting >= 32) {
                waiting -= 32;
                f(queue[waiting + lane]);
            }
            __syncwarp();
        };
        auto of_vector = [&](const uint4 &raw) {
            float v[kVec];
            Vec16<T>::unpack(raw, v);
#pragma unroll
            for (int x = 0; x < kVec; ++x) {
                const uint32_t in = __ballot_sync(0xFFFFFFFFu, v[x] >= least);
                if (v[x] >= least) queue[waiting + __popc(in & ((1u << lane) - 1u))] = v[x];
                waiting += __popc(in);
            }
            work();
        };
        constexpr uint32_t kNone = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;  // -inf
        const uint4 none = make_uint4(kNone, kNone, kNone, kNone);
        const uint4 *const zv = sl.vectors();
        for (int i0 = sl.lo + 32 * warp; i0 < sl.hi; i0 += U * kSampleThreads) {  // the same in all lanes
            const int i = i0 + lane;
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = i + u * kSampleThreads < sl.hi ? zv[i + u * kSampleThreads] : none;
#pragma unroll
            for (int u = 0; u < U; ++u) of_vector(raw[u]);
        }
        if (warp == 0) of_vector(sl.has_edge() ? sl.load_edge() : none);
        __syncwarp();
        if (lane < waiting) f(queue[lane]);
    }
    // The least logit in bins 0 .. bin; a whole warp calls.
    __device__ __forceinline__ float least_of_bins(int bin) const {
        const uint32_t lane = threadIdx.x & 31;
        auto within = [&](uint32_t key) { return Weigh::bin_of(weigh.depth(unorder_f32(key))) <= bin; };
        uint32_t lo = order_f32(-INFINITY) + 1, hi = order_f32(weigh.best);  // (the best is in bin 0)
        {  // it is near where the real numbers have it
            const float guess = weigh.best - static_cast<float>(bin + 1) / (kBinsPerUnit * weigh.inv);
            const uint32_t key = order_f32(guess);
            if (key > lo + 512 && key + 511 < hi && __ballot_sync(0xFFFFFFFFu, within(lane & 1 ? key + 511 : key - 512)) == 0xAAAAAAAAu)
                lo = key - 511, hi = key + 511;
        }
        while (lo < hi) {  // ends: hi - lo falls to a 32nd at each turn
            const uint32_t step = (hi - lo) / 32 + 1, key = lo + min(lane * step, hi - lo);
            const uint32_t in = __ballot_sync(0xFFFFFFFFu, within(key));
            if (in == 0) {  // (the lanes end before hi)
                lo += 31 * step + 1;
                continue;
            }
            const uint32_t at = __ffs(in) - 1;
            hi = min(hi, lo + at * step);
            if (at > 0) lo += (at - 1) * step + 1;
        }
        return unorder_f32(hi);
    }
    // Up to four numbers of each CTA (any thread's: all have them) to all CTAs.
    __device__ __forceinline__ void exchange(uint64_t a, uint64_t b = 0, uint64_t c = 0, uint64_t d = 0) {
        turn ^= 1;
        if (threadIdx.x < slices) {
            uint64_t *const to = cluster_peer(&sm.slots[turn][rank][0], threadIdx.x);
            to[0] = a, to[1] = b, to[2] = c, to[3] = d;
        }
        sync();
    }
    __device__ __forceinline__ uint64_t sum_all(int which) const {
        uint64_t s = 0;
        for (int r = 0; r < slices; ++r) s += sm.slots[turn][r][which];
        return s;
    }
    __device__ __forceinline__ uint64_t max_all(int which) const {
        uint64_t s = 0;
        for (int r = 0; r < slices; ++r) s = max(s, sm.slots[turn][r][which]);
        return s;
    }
    // ---- histograms
    // sm.before of the first CTA, from the histograms of all CTAs (complete, after
    // a sync): each CTA adds up its share of the bins, the first one the
    // running values.  All CTAs call; the candidates' memory is used.
    __device__ __forceinline__ void join_hists(bool by_count) const {
        const int share = kBins / slices, groups = max(1, kSampleThreads / share);  // groups of threads share the CTAs
        uint64_t *const stage = sm.cand;
        for (int t = threadIdx.x; t < share * groups; t += kSampleThreads) {
            const int b = rank * share + t % share;
            uint64_t v = 0;
            for (int r = t / share; r < slices; r += groups) {
                uint32_t x[3] = {};
#pragma unroll
                for (int part = 0; part < 3; ++part)
                    if (!(by_count && part > 0)) x[part] = *cluster_peer(&sm.hist[part][b], r);
#pragma unroll
                for (int part = 0; part < 3; ++part) v += static_cast<uint64_t>(x[part]) << (14 * part);
            }
            stage[t] = v;
        }
        __syncthreads();
        for (int t = threadIdx.x; t < share; t += kSampleThreads) {
            uint64_t v = 0;
            for (int g = 0; g < groups; ++g) v += stage[g * share + t];
            *cluster_peer(&sm.before[rank * share + t], 0) = v;
        }
        sync();
        if (rank != 0) return;
        const int b = 2 * threadIdx.x;
        const uint64_t v0 = sm.before[b], v1 = sm.before[b + 1];
        uint64_t total;
        const uint64_t run = block_before(v0 + v1, &total);
        sm.before[b] = run;
        sm.before[b + 1] = run + v0;
        if (threadIdx.x == 0) sm.total = total;
        __syncthreads();
    }
    // First CTA: the bin in which the prefix of `target` ends, and what is
    // before it, in sm.found; no candidates yet.  The bins have that much.
    __device__ __forceinline__ void find_bin(uint64_t target) const {
        forget();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int b = 2 * threadIdx.x + x;
            const uint64_t end = b + 1 < kBins ? sm.before[b + 1] : sm.total;
            if (sm.before[b] < target && target <= end) sm.found[0] = b, sm.found[1] = sm.before[b];
        }
        if (threadIdx.x == 0) sm.cand_count = 0;
        __syncthreads();
    }
    // What the first CTA's threads have (a, b, c there), in all CTAs: two
    // buffers, so that a CTA may still read the last while the next is written.
    __device__ __forceinline__ void tell(uint64_t *a, uint64_t *b, uint64_t *c) {
        tale ^= 1;
        if (rank == 0 && threadIdx.x == 0) sm.told[tale][0] = *a, sm.told[tale][1] = *b, sm.told[tale][2] = *c;
        sync();
        const uint64_t *const told = cluster_peer(&sm.told[tale][0], 0);
        *a = told[0];
        *b = told[1];
        *c = told[2];
    }
    __device__ __forceinline__ void find_bin_for_all(uint64_t target, uint64_t *bin, uint64_t *before) {
        uint64_t none = 0;
        if (rank == 0) {
            find_bin(target);
            *bin = sm.found[0], *before = sm.found[1];
        }
        tell(bin, before, &none);
    }

    // ---- tokens to rank
    // The logits of a bin: `least` and more, and below `limit` (NaN: no limit).
    struct Range {
        float least, limit;
        __device__ __forceinline__ bool has(float z) const { return z >= least && !(z >= limit); }
        // their ranking keys' ends
        __device__ __forceinline__ uint64_t low() const { return static_cast<uint64_t>(order_f32(least)) << 32; }
        __device__ __forceinline__ uint64_t high() const {
            return isnan(limit) ? ~0ull : (static_cast<uint64_t>(order_f32(limit)) << 32) - 1;
        }
    };
    // The slice's values in one of two ranges go to the first CTA, unless they are
    // too many.
    __device__ __forceinline__ void gather(const Range &r0, const Range &r1) const {
        uint32_t *const count = cluster_peer(&sm.cand_count, 0);
        uint64_t *const cand = cluster_peer(&sm.cand[0], 0);
        each_above(fminf(r0.least, r1.least), __int_as_float(0x7FC00000), [&](float z, int index) {
            if (!r0.has(z) && !r1.has(z)) return;
            const uint32_t at = atomicAdd(count, 1u);
            if (at < kCap) cand[at] = make_key(z, static_cast<uint32_t>(index));
        });
    }
    __device__ __forceinline__ void gather(const Range &range) const { gather(range, range); }
    // How many they are, after a sync.  No thread has a read of the first CTA's
    // memory in flight afterwards.
    __device__ __forceinline__ uint32_t gathered() const {
        if (threadIdx.x == 0) sm.place = *cluster_peer(&sm.cand_count, 0);
        __syncthreads();
        return sm.place;
    }
    // Those of two bins, in all threads of the CTA.
    __device__ __forceinline__ void ranges_of(int bin0, int bin1, Range *r0, Range *r1) const {
        __syncthreads();
        const int warp = threadIdx.x >> 5;
        if (warp < 4) {
            const int b = (warp < 2 ? bin0 : bin1) - (warp & 1);
            const float edge = b >= 0 ? least_of_bins(b) : __int_as_float(0x7FC00000);
            if ((threadIdx.x & 31) == 0) sm.bin_edge[warp] = edge;
        }
        __syncthreads();
        *r0 = Range{sm.bin_edge[0], sm.bin_edge[1]};
        *r1 = Range{sm.bin_edge[2], sm.bin_edge[3]};
    }
    __device__ __forceinline__ uint64_t first_of(bool by_count, int n, uint64_t low, uint64_t high, uint64_t before,
                                                 uint64_t target, uint64_t *mass) const {
        return first_to_reach(sm, weigh, by_count, n, low, high, before, target, mass);
    }

    // ---- a prefix in all of the row
    struct Prefix {
        uint32_t key;   // of its last token (the upper half of a ranking key)
        uint64_t ties;  // how many of the tokens with this key it takes (by count, or where `index` is below 0)
        uint64_t mass;  // its mass (not by count)
        int index;      // the last token's, if it is known, else -1
    };
    // The tokens among which the shortest prefix with `target` tokens or mass
    // ends go to the first CTA, which has joined the histograms of it: how many
    // they are, what is before them (and, if they are one key too many to rank,
    // that key); their keys lie in key_low .. key_high.
    __device__ __forceinline__ uint32_t collect(bool by_count, uint64_t target, uint64_t *before, uint32_t *only_key) {
        uint64_t bin = 0;
        crowded = false;
        find_bin_for_all(target, &bin, before);
        Range range, same;
        ranges_of(static_cast<int>(bin), static_cast<int>(bin), &range, &same);
        gather(range);
        key_low = range.low(), key_high = range.high();
        sync();
        uint32_t n = gathered();
        if (n <= kCap) return n;
        // a crowded bin: cut by keys, low .. high are left
        crowded = true;
        uint64_t most = 0, least = 0;
        each_above(range.least, range.limit, [&](float z, int) {
            const uint32_t key = order_f32(z);
            most = max(most, static_cast<uint64_t>(key));
            least = max(least, static_cast<uint64_t>(~key));
        });
        most = block_max_u64(most), least = block_max_u64(least);
        exchange(most, least);
        uint32_t high = static_cast<uint32_t>(max_all(0)), low = ~static_cast<uint32_t>(max_all(1));
        while (n > kCap && low != high) {  // ends: every turn takes 10 bits off high - low
            const int bits = 32 - __clz(high - low), shift = bits > 10 ? bits - 10 : 0;
            clear_hist();
            each([&](float z, int) {
                const uint32_t key = order_f32(z);
                if (!(z > -INFINITY) || key < low || key > high) return;
                const int b = (high - key) >> shift;
                if (by_count) atomicAdd(&sm.hist[0][b], 1u);
                else count_mass(b, weigh(z));
            });
            sync();
            join_hists(by_count);
            uint64_t b = 0, more = 0;
            find_bin_for_all(target - *before, &b, &more);
            *before += more;
            high -= static_cast<uint32_t>(b) << shift;
            const uint32_t width = (1u << shift) - 1u;
            if (high - low > width) low = high - width;
            gather(Range{unorder_f32(low), unorder_f32(high + 1)});  // (above +inf: NaN)
            key_low = static_cast<uint64_t>(low) << 32, key_high = static_cast<uint64_t>(high) << 32 | 0xFFFFFFFFu;
            sync();
            n = gathered();
        }
        *only_key = high;
        return n;
    }
    // Of a key too many to rank: how many of its tokens the prefix takes.
    __device__ __forceinline__ Prefix of_ties(bool by_count, uint64_t target, uint64_t before, uint32_t key) const {
        const uint64_t w = weigh(unorder_f32(key));
        const uint64_t ties = by_count ? target - before : (target - before + w - 1) / w;
        return Prefix{key, ties, before + ties * w, -1};
    }
    // The shortest prefix with `target` tokens or mass, in all CTAs.
    __device__ __forceinline__ Prefix shortest_prefix(bool by_count, uint64_t target) {
        uint64_t before = 0, last = 0, mass = 0, ties = 0;
        uint32_t only_key = 0;
        const uint32_t n = collect(by_count, target, &before, &only_key);
        if (n > kCap) return of_ties(by_count, target, before, only_key);
        if (rank == 0) {
            last = first_of(by_count, static_cast<int>(n), key_low, key_high, before, target, &mass);
            uint64_t same = 0;  // candidates with its logit, down to it
            for (uint32_t i = threadIdx.x; i < n; i += kSampleThreads)
                same += (sm.cand[i] >> 32) == (last >> 32) && sm.cand[i] >= last;
            ties = block_sum(same);
        }
        tell(&last, &mass, &ties);
        return Prefix{static_cast<uint32_t>(last >> 32), ties, mass, key_index(last)};
    }
    // The index of the ties-th token (from 1) with this key, written by the CTA that has it.
    __device__ __forceinline__ void write_tie(uint32_t key, uint64_t ties, int32_t *token) {
        uint64_t own = 0;
        each([&](float z, int) { own += z > -INFINITY && order_f32(z) == key; });
        own = block_sum(own);
        exchange(own);
        uint64_t earlier = 0;
        for (int r = 0; r < rank; ++r) earlier += sm.slots[turn][r][0];
        if (ties <= earlier || ties > earlier + own) return;
        // runs of kSampleThreads values in order
        uint64_t found = earlier;
        const int lo = max(sl.e0, 0), hi = min(sl.e1, sl.V);
        for (int v0 = lo; v0 < hi; v0 += kSampleThreads) {
            const int v = v0 + threadIdx.x;
            const float z = v < hi ? load_value(sl.z + v) : -INFINITY;
            const bool hit = z > -INFINITY && order_f32(z) == key;
            uint64_t total;
            const uint64_t at = found + block_before(hit, &total);
            if (hit && at + 1 == ties) *token = v;
            found += total;
        }
    }
};

// The row of a cluster where not all run at once: within blocks of kSampleThreads
// rows those without a top_k, several times the work, come first (64 rows of 262144, a
// third of them without: 70 us, 81 in the batch's order).
__device__ __forceinline__ int64_t row_by_work(const SampleLogitsParams &a, SampleSmem &sm, int64_t turn) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t base = turn / kSampleThreads * kSampleThreads;
    const bool is_row = base + tid < a.batch;
    bool long_row = false;
    if (is_row) {
        const int k = a.top_k[base + tid];
        long_row = !(k > 0 && k < a.V) && (a.temperature == nullptr || a.temperature[base + tid] > 0.0f);
    }
    const uint32_t mask = __ballot_sync(0xFFFFFFFFu, long_row);
    if (lane == 0) sm.slots[0][warp][0] = static_cast<uint64_t>(__popc(mask));
    __syncthreads();
    int before = __popc(mask & ((1u << lane) - 1u)), all = 0;  // long rows
    for (int w = 0; w < kSampleWarps; ++w) {
        const int in_warp = static_cast<int>(sm.slots[0][w][0]);
        all += in_warp;
        before += w < warp ? in_warp : 0;
    }
    if (is_row && (long_row ? before : all + tid - before) == turn - base) sm.place = tid;
    __syncthreads();
    return base + sm.place;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_logits_kernel(const SampleLogitsParams a, int log2_slices) {
    extern __shared__ __align__(16) unsigned char sample_smem[];
    SampleSmem &sm = *reinterpret_cast<SampleSmem *>(sample_smem);
    const int rank = blockIdx.x & ((1 << log2_slices) - 1), tid = threadIdx.x;
    const int64_t turn = blockIdx.x >> log2_slices;
    cluster_arrive_relaxed();  // all CTAs of the cluster run, before their memory is written
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one
    const int64_t row = a.by_work ? row_by_work(a, sm, turn) : turn;
    SampleRow<T> r(sm, static_cast<const T *>(a.logits) + row * a.ld, a.V, log2_slices, rank);
    const float temp = a.temperature != nullptr ? a.temperature[row] : 1.0f;
    const float top_p = a.top_p != nullptr ? a.top_p[row] : 1.0f, min_p = a.min_p != nullptr ? a.min_p[row] : 0.0f;
    const float u = a.u[row];
    const bool warm = temp > 0.0f;
    const int top_k = !warm ? 1 : (a.top_k != nullptr ? a.top_k[row] : 0);
    r.clear_hist();

    float own = -INFINITY;
    r.each([&](float z, int) { own = fmaxf(own, z); });
    float best = block_max<kSampleThreads>(own, sm.scratch);
    cluster_wait();
    r.exchange(order_f32(best));
    best = unorder_f32(static_cast<uint32_t>(r.max_all(0)));
    if (best == -INFINITY) {  // nothing to draw from
        if (rank == 0 && tid == 0) a.token[row] = -1, a.prob[row] = 0.0f;
        return;
    }
    r.weigh = Weigh{best, 1.0f / temp, warm};
    const Weigh weigh = r.weigh;

    const uint64_t least_w = min_p > 0.0f ? static_cast<uint64_t>(ceilf(fminf(min_p, 2.0f) * 1099511627776.0f)) : 0;
    const uint32_t p24 = top_p > 0.0f ? static_cast<uint32_t>(ceilf(fminf(top_p, 1.0f) * 16777216.0f)) : 0;
    const bool cuts_p = top_p < 1.0f;
    const uint32_t u24 = u > 0.0f ? static_cast<uint32_t>(fminf(u * 16777216.0f, 16777215.0f)) : 0;
    bool rest;
    auto least_of = [&](uint64_t S) {  // ceil(top_p S), at least 1
        const uint64_t least = share_of(S, p24, &rest);
        return max(least + rest, static_cast<uint64_t>(1));
    };

    // The first CTA has all tokens from some depth up, n of them and top_k at
    // least: the row's token.
    auto finish_top_k = [&](int n, float least) {
        const uint64_t high = static_cast<uint64_t>(order_f32(best)) << 32 | 0xFFFFFFFFu;
        uint64_t low = static_cast<uint64_t>(order_f32(least)) << 32, mass;
        if (n > top_k) low = r.first_of(true, n, low, high, 0, static_cast<uint64_t>(top_k), &mass);
        uint64_t s = 0, q = 0;
        for (int i = tid; i < n; i += kSampleThreads) {
            const uint64_t key = sm.cand[i], w = key >= low ? r.weight_of(key) : 0;
            s += w;
            q += w >= least_w ? w : 0;
        }
        const uint64_t S = r.block_sum(s), Q = r.block_sum(q);
        uint64_t M = min(S, Q);
        if (cuts_p && least_of(S) < M) {
            r.first_of(false, n, low, high, 0, least_of(S), &mass);
            M = min(M, mass);
        }
        M = max(M, kOne);
        const uint64_t key = r.first_of(false, n, low, high, 0, share_of(M, u24, &rest) + 1, &mass);
        if (tid == 0) {
            a.token[row] = key_index(key);
            a.prob[row] = static_cast<float>(r.weight_of(key)) / static_cast<float>(M);
        }
    };
    using Range = typename SampleRow<T>::Range;
    const float kNoLimit = __int_as_float(0x7FC00000);
    uint64_t S = 0, Q = 0;
    bool whole = true;  // all tokens of a weight are in
    if (top_k > 0 && top_k < a.V) {
        // bins of the threads' maxima: where top_k of them are reached, at least top_k tokens are
        if (top_k <= kSampleThreads << log2_slices) {
            const int bin = Weigh::bin_of(weigh.depth(own));
            if (bin < kBins) atomicAdd(&sm.hist[0][bin], 1u);
            r.sync();
            uint64_t last = kBins, none = 0, enough = 0;
            r.join_hists(true);
            if (rank == 0) {
                if (sm.total >= static_cast<uint64_t>(top_k)) {
                    r.find_bin(static_cast<uint64_t>(top_k));
                    last = sm.found[0];
                }
            }
            r.tell(&last, &none, &enough);
            if (last < kBins) {
                const float least = r.least_of_bins(static_cast<int>(last));
                r.gather(Range{least, kNoLimit});
                r.sync();
                const uint32_t n = r.gathered();
                cluster_arrive_relaxed();  // the first CTA stays until all have read how many there are
                if (n <= kCap) {
                    if (rank == 0) finish_top_k(static_cast<int>(n), least);
                    cluster_wait();
                    return;
                }
                cluster_wait();
            }
            r.clear_hist();  // (after a sync that follows its reading)
        }
        uint64_t positive = 0;
        r.each([&](float z, int) {
            const int bin = Weigh::bin_of(weigh.depth(z));
            if (bin < kBins) {
                atomicAdd(&sm.hist[0][bin], 1u);
                ++positive;
            }
        });
        positive = r.block_sum(positive);
        r.exchange(positive);
        positive = r.sum_all(0);
        r.join_hists(true);
        if (static_cast<uint64_t>(top_k) < positive) {
            whole = false;
            uint64_t bin = 0, before = 0;
            r.find_bin_for_all(static_cast<uint64_t>(top_k), &bin, &before);
            const uint64_t *const firsts = cluster_peer(&sm.before[0], 0);
            const uint64_t end = bin + 1 < kBins ? firsts[bin + 1] : positive;
            if (end <= kCap) {
                // all tokens down to that bin: the first CTA does the rest
                const float least = r.least_of_bins(static_cast<int>(bin));
                r.gather(Range{least, kNoLimit});
                r.sync();
                if (rank == 0) finish_top_k(static_cast<int>(end), least);
                return;
            }
            // too many to rank: their last one's key, and the mass down to it
            r.sync();  // (the bins before it are read)
            const auto cut = r.shortest_prefix(true, static_cast<uint64_t>(top_k));
            uint64_t s = 0;
            r.each([&](float z, int) {
                if (z > -INFINITY && order_f32(z) > cut.key) s += weigh(z);
            });
            s = r.block_sum(s);
            r.exchange(s);
            S = r.sum_all(0) + cut.ties * weigh(unorder_f32(cut.key));
        }
        r.sync();  // (the histograms are read)
        r.clear_hist();
    }

    // masses: of all tokens, of those that min_p keeps, and in fp32 down to some
    // depths: the histogram need not go deeper than the first that holds the
    // prefix.  (Prefixes of 0.8 to 0.98 of the mass end at 4 to 11 below the best
    // token for normal logits of a spread of 1 to 4 T, 20011 to 262144 of them,
    // and the depths divide that range: of 151936 at a spread of 2.5, rows at
    // top_p 0.8 end at 7.1 on average, 0.9: 8.0, 0.95: 9.1, 0.98: 10.1, one in six
    // of these beyond the last depth.  64 rows of 262144 at a spread of 4: 76 us at
    // top_p 0.8, 81 at 0.95, 110 at 0.98, two rows in three of it beyond.)
    constexpr int kDepths[4] = {5 * kBinsPerUnit, 7 * kBinsPerUnit, 17 * kBinsPerUnit / 2, 21 * kBinsPerUnit / 2};  // bins
    const bool usual = warm && best < INFINITY && weigh.inv < INFINITY;
    float to_depth[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // in units of the best token's weight
    {
        if (tid < 128) {
            const int i = tid >> 5;
            const float least = r.least_of_bins((i == 0 ? kDepths[0] : i == 1 ? kDepths[1] : i == 2 ? kDepths[2] : kDepths[3]) - 1);
            if ((tid & 31) == 0) sm.edge[i] = least;
        }
        __syncthreads();
        const float edge[4] = {sm.edge[0], sm.edge[1], sm.edge[2], sm.edge[3]};
        uint64_t s = 0, q = 0;
        if (usual) {
            // w in two halves of 20 bits: a thread's at most 520 values leave their sums below 2^32
            const float least_e = static_cast<float>(least_w) * 9.094947017729282e-13f;  // 2^-40
            uint32_t hi[2] = {}, lo[2] = {};
            const auto add = [&](float z, bool for_min_p) {
                const float e = fmaxf(expf((z - best) * weigh.inv), 0.0f);  // (NaN: 0)
                uint32_t h, l;
                split_weight(e, &h, &l);
                hi[0] += h, lo[0] += l;
                if (for_min_p && e >= least_e) hi[1] += h, lo[1] += l;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (z >= edge[i]) to_depth[i] += e;
            };
            if (least_w > 0) r.each([&](float z, int) { add(z, true); });
            else r.each([&](float z, int) { add(z, false); });
            s = (static_cast<uint64_t>(hi[0]) << 20) + lo[0];
            q = least_w > 0 ? (static_cast<uint64_t>(hi[1]) << 20) + lo[1] : s;
        } else {
            r.each([&](float z, int) {
                const uint64_t w = weigh(z);
                s += w;
                q += w >= least_w ? w : 0;
                const float e = static_cast<float>(w) * 9.094947017729282e-13f;  // 2^-40
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (z >= edge[i]) to_depth[i] += e;
            });
        }
        s = r.block_sum(s), q = r.block_sum(q);
        const float4 d = block_sum<kSampleThreads>(make_float4(to_depth[0], to_depth[1], to_depth[2], to_depth[3]), sm.depth_sums);
        auto pair = [](float a, float b) { return static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a); };
        r.exchange(s, q, pair(d.x, d.y), pair(d.z, d.w));
        if (whole) S = r.sum_all(0);
        Q = r.sum_all(1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            to_depth[i] = 0.0f;
            for (int x = 0; x < r.slices; ++x)
                to_depth[i] += __uint_as_float(static_cast<uint32_t>(sm.slots[r.turn][x][2 + i / 2] >> (32 * (i & 1))));
        }
    }
    // The histogram down to a depth that holds `most`.  The sums above are off by
    // 600 roundings at most, so a ten-thousandth is taken off them.
    auto join_masses = [&](uint64_t most) {
        const float share = static_cast<float>(most) * 9.094947017729282e-13f * 1.0001f;
        int depth = 4;
#pragma unroll
        for (int i = 3; i >= 0; --i)
            if (share <= to_depth[i]) depth = i;
        const float least = depth == 4 ? r.least_of_bins(kBins - 1) : sm.edge[depth];
        r.each_above_in_turn(least, [&](float z) {
            const float d = weigh.depth(z);
            r.count_weight(Weigh::bin_of(d), expf(-d));
        });
        r.sync();
        r.join_hists(false);
    };
    uint64_t M = min(S, Q);
    bool joined = false;
    if (cuts_p && least_of(S) < M) {
        join_masses(least_of(S));
        // P's bin bounds M, and with it the draw: where both bounds draw from
        // one bin, the tokens of the two bins are all that is needed
        uint64_t bins = 0, before_p = 0, before_t = 0;
        if (rank == 0) {
            r.find_bin(least_of(S));
            const uint64_t bin_p = sm.found[0], end_p = bin_p + 1 < kBins ? sm.before[bin_p + 1] : sm.total;
            before_p = sm.found[1];
            r.find_bin(share_of(max(min(M, end_p), kOne), u24, &rest) + 1);
            const uint64_t bin_t = sm.found[0];
            before_t = sm.found[1];
            r.find_bin(share_of(max(min(M, before_p + 1), kOne), u24, &rest) + 1);
            bins = bin_p | bin_t << 16 | static_cast<uint64_t>(sm.found[0] == bin_t) << 32;
        }
        r.tell(&bins, &before_p, &before_t);
        if (bins >> 32) {
            const int bin_p = static_cast<int>(bins & 0xFFFF), bin_t = static_cast<int>(bins >> 16 & 0xFFFF);
            Range of_p, of_t;
            r.ranges_of(bin_p, bin_t, &of_p, &of_t);
            r.gather(of_p, of_t);
            r.sync();
            const uint32_t n = r.gathered();
            cluster_arrive_relaxed();  // the first CTA stays until all have read how many there are
            if (n <= kCap) {
                if (rank == 0) {
                    const int all = static_cast<int>(n);
                    uint64_t mass;
                    r.first_of(false, all, of_p.low(), of_p.high(), before_p, least_of(S), &mass);
                    M = max(min(M, mass), kOne);
                    const uint64_t key = r.first_of(false, all, of_t.low(), of_t.high(), before_t, share_of(M, u24, &rest) + 1, &mass);
                    if (tid == 0) {
                        a.token[row] = key_index(key);
                        a.prob[row] = static_cast<float>(r.weight_of(key)) / static_cast<float>(M);
                    }
                }
                cluster_wait();
                return;
            }
            cluster_wait();
        }
        M = min(M, r.shortest_prefix(false, least_of(S)).mass);
        if (r.crowded) {
            r.sync();  // (the histograms are read)
            r.clear_hist();
        }
        joined = !r.crowded;
    }
    M = max(M, kOne);
    const uint64_t target = share_of(M, u24, &rest) + 1;
    if (!joined) join_masses(target);
    uint64_t before = 0, mass;
    uint32_t key = 0;
    const uint32_t n = r.collect(false, target, &before, &key);
    cluster_arrive_relaxed();  // the first CTA stays until all have read how many there are
    if (n > kCap) {
        cluster_wait();
        r.write_tie(key, r.of_ties(false, target, before, key).ties, a.token + row);
    } else {
        if (rank != 0) {  // the first CTA has all that it needs
            cluster_wait();
            return;
        }
        const uint64_t last = r.first_of(false, static_cast<int>(n), r.key_low, r.key_high, before, target, &mass);
        key = static_cast<uint32_t>(last >> 32);
        if (tid == 0) a.token[row] = key_index(last);
        cluster_wait();
    }
    if (rank == 0 && tid == 0) a.prob[row] = static_cast<float>(weigh(unorder_f32(key))) / static_cast<float>(M);
}

// CTAs of a launch, about: twice what runs at once (two per SM), since rows differ
// in their work (64 rows of 262144 with settings of their own: 55 us, 78 with 304
// CTAs; where all rows are alike 32 to 107, 21 to 91 with 304).
constexpr int64_t kCtas = 608;
// Bytes of a row per CTA, at most: what runs at once is read again from L2 then
// (1000 rows of 151936 fp32: 325 us in two slices, 335 in one; without a top_k 444 and 507; four: 400 and more).
constexpr int64_t kSliceBytes = 384 << 10;

template <typename T>
static cudaError_t start_sample(SampleLogitsParams p, cudaStream_t s) {
    const int64_t batch = p.batch;
    // CTAs per row: enough for the chip, of 8192 values or more, or so that slices
    // stay in L2; 2^18 values each at most
    int log2_slices = 0;
    while (((p.V - 1) >> log2_slices) >= (1 << 18)) ++log2_slices;
    while (log2_slices < (batch <= 8 ? 4 : 3) && (batch << (log2_slices + 1)) <= kCtas && (p.V >> log2_slices) >= 16384) ++log2_slices;
    while (log2_slices < 3 && (p.V * static_cast<int64_t>(sizeof(T))) >> log2_slices > kSliceBytes) ++log2_slices;
    p.by_work = p.top_k != nullptr && (batch << log2_slices) > kCtas / 2;
    auto kernel = sample_logits_kernel<T>;
    static PerDevice prepared;
    const cudaError_t e = prepared.once([&] {
        const cudaError_t x = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SampleSmem));
        return x != cudaSuccess ? x : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(batch << log2_slices));
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = sizeof(SampleSmem);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << log2_slices;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p, log2_slices);
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
    p.token = out_token, p.prob = out_prob, p.ld = ld, p.batch = batch, p.V = static_cast<int>(V);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == VIE_DTYPE_BF16 ? start_sample<__nv_bfloat16>(p, s) : start_sample<float>(p, s);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}
