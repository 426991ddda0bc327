// vie_e2m1_logits.cu - full logits of a 4-bit head on the tensor cores.
//
//   out[i, v] = s_i t_v sum_b sigma_ib tau_vb sum_(j in b) x_ij w_vj
//
// with codes x, w (e2m1), block scales sigma, tau (e4m3, 16 columns each) and row
// scales s, t (powers of two): block-scaled MMAs of 128 vocabulary rows by up to
// 256 rows of x and 64 columns, scales and accumulators in TMEM.
//
// A persistent CTA per SM takes tiles of 128 vocabulary rows by BN rows of x.  Two
// producer threads fill a ring of stages of 256 or 512 columns: codes by TMA boxes
// of 128 bytes a row (columns and rows beyond the matrix read as 0), scales by bulk
// copies of their 512-byte tiles, which lie in memory as TMEM wants them.  Four
// warps take a stage's scales to the stage's own columns of TMEM, each to its
// quarter of the lanes (all four hold the same); an issuing thread runs the MMAs.
// That a stage is full again says that its MMAs are over, so its columns are free.
// Epilogue warps scale the accumulators and write them.
//
// (tcgen05.cp, which takes scales to TMEM without registers, runs in order with
// the MMAs, some 100 cycles a copy of 512 bytes: 51 us for one row of x on 262144 x
// 1152.)
//
// Measured, on the device alone, inputs of other calls in between (the floor: bytes
// at the copy rate, 6.79 TB/s):
//   262144 x 1152, 1 row of x, fp32    29.0 us (25.2)     bytes: 171 MB of the head's
//   262144 x 1152, 32 rows, fp32       32.0 us (30.0)     bytes; writes of 512 a row and tile
//   100003 x 1000, 129 rows, fp32      20.9 us (15.9)     782 tiles on 152 SMs: 22 of them have a sixth
//   128256 x 2048, 256 rows, bf16      41.9 us (31.5)
//   128256 x 2048, 2048 rows, bf16      259 us (99.5; 4.2 PFLOP/s), fp32 305 us (177)
// Many rows: the tensor pipe is 43 % busy.  A stage of 256 columns moves about 126 KB
// through shared memory (54 in by TMA, 48 read by the MMAs, 24 by the scale warps,
// four of which read the same): 980 cycles at 128 bytes each, were they all to share one
// path, beside some 190 of the epilogue's accesses, of the 1200 that the stage takes; and
// the accumulator's 128 columns per warp are drained between tiles.  Multicasting x to
// pairs of CTAs (254 us, 256 without) and MMAs of pairs of CTAs (268 us; 232 instead of 189 at
// 151936 x 1024) gained nothing.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"
#include "vie_e2m1.cuh"
#include "vie_e2m1_logits.h"
#include "vie_launch.h"
#include "vie_tcgen05.cuh"

namespace vie {

constexpr int kE2m1Kb = 256;                // columns of a K-block: 128 bytes of codes a row, a box
constexpr int kE2m1KbTiles = kE2m1Kb / 64;  // its scale tiles, and MMAs
constexpr int64_t kMarkedBytes = 4 << 20;   // of x's codes: one thirtieth of L2

template <int BN>
struct E2m1Shape {
    static constexpr int kXTiles = BN > 128 ? 2 : 1;              // tiles of 128 rows of x
    // K-blocks per stage: what a stage costs besides its bytes (waits, arrivals) is paid for
    // more of them where shared memory holds enough such stages.
    static constexpr int kBlocks = BN > 64 ? 1 : 2;
    static constexpr int kSteps = kBlocks * kE2m1KbTiles;         // scale tiles and MMAs of a stage
    static constexpr int kBoxW = kE2m1TileRows * 128, kBoxX = BN * 128;
    static constexpr int kStageW = kBlocks * kBoxW, kStageX = kBlocks * kBoxX;
    static constexpr int kSet = kSteps * kE2m1TileBytes;          // a stage's scales of 128 rows
    static constexpr int kStageBytes = kStageW + kStageX + (1 + kXTiles) * kSet;
    static constexpr int kBuffers = BN > 128 ? 1 : 2;             // accumulators
    static constexpr int kScaleCols = 4 * kSteps * (1 + kXTiles);  // TMEM columns of a stage's scales
    static constexpr int kScaleBase = (kBuffers * BN + 31) / 32 * 32;
    static constexpr int kByMemory = (232448 - 1024 - 2048) / kStageBytes, kByTmem = (512 - kScaleBase) / kScaleCols;
    static constexpr int kStages = kByMemory < kByTmem ? kByMemory : kByTmem;
    static constexpr int kEpilogueWarps = BN >= 128 ? 8 : 4;
    static constexpr int kWarpCols = BN * 4 / kEpilogueWarps;     // columns that an epilogue warp writes
    static constexpr int kScaleWarp = 4 + kEpilogueWarps;         // the first of four
    static constexpr int kThreads = 32 * (kScaleWarp + 4);
    static constexpr int kSmem = 1024 + kStages * kStageBytes;  // 1024: the ring starts at a multiple of it
    static_assert(kStages >= 2 && kStages <= 16, "ring");
};

// Whether s t, the powers of two of a row of x and of a vocabulary row, is infinite or 0
// where their result, sum s t, may be neither: a sum is 0 or between 2^-20 (codes 1/2,
// scales 2^-9) and 2^37 (2^14 products of 2688^2), so below 2^-187 all results are 0 (those
// of two rows of zeros, whose powers are 2^-126, among them).
__device__ __forceinline__ bool is_far(float s, float t) {
    const float both = s * t;
    return both == INFINITY || (both == 0.0f && s * 0x1p40f * t != 0.0f);
}
// Some rows' powers s: the least above 2^-126, the largest, and 2^-126 if it is among them
// (rows of zeros, as padding has them, are apart) or 1.  is_far has no s for a t from `from`
// to below `to`.
struct PowerRange {
    float from, to, least, largest, lowest;
    __device__ __forceinline__ void set(float least_, float largest_, float lowest_) {
        least = least_, largest = largest_, lowest = lowest_;
        from = fmaxf(0x1p-149f / least, lowest < 1.0f ? 0x1p-23f : 0.0f);
        to = largest > 2.0f ? 0x1p127f / (0.5f * largest) : INFINITY;
    }
    __device__ __forceinline__ bool may_be_far(float t) const {
        return !(t >= from && t < to) && (least * t == 0.0f || largest * t == INFINITY || is_far(lowest, t));
    }
};
// sum s t then.  t = first last, and of sum * first * s * last one product is inexact, at
// most, which is the result's own: s and t are between 2^-126 and 2^117.  For t from
// 2^-100 to 2^90, sum t is a number.  Where t is larger, sum first is one, times s it is
// above 2^-82, and infinite only where the result is; where t is smaller, sum first is above
// 2^-106, times s below 2^94, and below 2^-126 only where the result is below 2^-166,
// which is 0.
__device__ __forceinline__ float far_product(float sum, float s, float t) {
    const float last = t < 0x1p-100f ? 0x1p-40f : t > 0x1p90f ? 0x1p27f : 1.0f;
    const float first = t < 0x1p-100f ? t * 0x1p40f : t > 0x1p90f ? t * 0x1p-27f : t;
    return sum * first * s * last;
}

template <int BN>
struct E2m1Smem {
    uint64_t full[16], scaled[16], empty[16], acc_full[2], acc_empty[2], final_bar;
    uint32_t tmem_base;
    int abort, any_far;
    float x_scale[E2m1Shape<BN>::kEpilogueWarps][E2m1Shape<BN>::kWarpCols];  // (no barrier between warps: one may give up)
    PowerRange x_range[E2m1Shape<BN>::kEpilogueWarps];  // of those
};

// Ends a wait that ran out: the flag for the host, `abort` for the other roles.
__device__ __forceinline__ void give_up(uint32_t *flag, int *abort) {
    atomicOr(flag, kErrWaitTimeout);
    *static_cast<volatile int *>(abort) = 1;
}

// Where an epilogue lane writes its vocabulary row v: columns c and c + 1 of a
// tile (rows of the output, ld apart) at a time, in ascending order; all lanes of
// the warp call.  WORDS (bf16): lanes trade, an even lane writes its own and its
// neighbour's value of column c in one word, the odd one those of column c + 1.  It
// needs even V and ld and rows that start at such words, and is a parameter of the
// kernel because a branch per store costs more than the stores (151936 x 1024 for
// 2048 rows: 357 us; 213 value by value, 193 by words).
template <typename T, bool WORDS>
struct ColumnStore {
    T *o;
    int64_t ld;
    int rows;  // of this lane, columns counted from its first
    __device__ __forceinline__ ColumnStore(T *out, int64_t ld_, int64_t v, int64_t V, int rows_) : ld(ld_) {
        const int odd = WORDS ? static_cast<int>(v & 1) : 0;  // (a tile's first row is even: the lane is odd as well)
        o = out + odd * ld + (v - odd);
        rows = v < V ? rows_ - odd : 0;
    }
    __device__ __forceinline__ void pair(int c, uint32_t both) {  // of bf16
        if constexpr (WORDS) {
            const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, both, 1);
            const uint32_t w = (threadIdx.x & 1) == 0 ? __byte_perm(both, other, 0x5410) : __byte_perm(other, both, 0x7632);
            if (c < rows) *reinterpret_cast<uint32_t *>(o) = w;
            o += 2 * ld;
        } else {
            put(c, static_cast<uint16_t>(both));
            put(c + 1, static_cast<uint16_t>(both >> 16));
        }
    }
    __device__ __forceinline__ void pair(int c, float a, float b) {
        if constexpr (sizeof(T) == 2) {
            pair(c, pack_bf16(a, b));
        } else {
            put(c, a);
            put(c + 1, b);
        }
    }

  private:
    template <typename V>
    __device__ __forceinline__ void put(int c, V value) {
        static_assert(sizeof(V) == sizeof(T), "one value");
        if (c < rows) *reinterpret_cast<V *>(o) = value;
        o += ld;
    }
};

// Those results of a tile (vocabulary rows from v0 on, rows of x from i0 on), over what the
// epilogue has written there; all threads of the CTA call, after its tiles.  Such rows are
// hardly ever met, so this is the simplest way: a pair of rows per thread, from the codes.
// (In the epilogue, any code besides sum (s t) costs all calls 2 to 16 %: its warps hand an
// accumulator back while the MMAs wait for it.)  2.6 ms where all rows of 262144 x 1152
// for 32 rows are such.
template <typename T>
__device__ __noinline__ void far_results(const E2m1Product &p, int64_t v0, int64_t i0, int rows) {
    griddep_wait();
    const int blocks = (p.d + 15) / 16, tiles = e2m1_tiles(p.d);
    const int64_t pitch = e2m1_pitch(p.d);
    for (int k = threadIdx.x; k < kE2m1TileRows * rows; k += blockDim.x) {
        const int64_t v = v0 + k % kE2m1TileRows, i = i0 + k / kE2m1TileRows;
        if (v >= p.V || i >= p.n) continue;
        const float s = p.x_row_scales[i], t = p.w_row_scales[v];
        if (!is_far(s, t)) continue;
        const uint2 *const x = reinterpret_cast<const uint2 *>(p.x_codes + i * pitch);
        const uint2 *const w = reinterpret_cast<const uint2 *>(p.w_codes + v * pitch);
        float sum = 0.0f;
        for (int b = 0; b < blocks; ++b) {
            const uint2 cx = x[b], cw = w[b];
            float xv[16], wv[16], part = 0.0f;
            from_e2m1(cx.x, xv), from_e2m1(cx.y, xv + 8);
            from_e2m1(cw.x, wv), from_e2m1(cw.y, wv + 8);
#pragma unroll
            for (int j = 0; j < 16; ++j) part = fmaf(xv[j], wv[j], part);
            const float sigma = from_e4m3(p.x_scales[e2m1_scale_at(i, b, tiles)]);
            const float tau = from_e4m3(p.w_scales[e2m1_scale_at(v, b, tiles)]);
            sum = fmaf(part, sigma * tau, sum);
        }
        store_value(static_cast<T *>(p.out) + i * p.ld + v, far_product(sum, s, t));
    }
}

template <int BN, typename T, bool WORDS>
__global__ void __launch_bounds__(E2m1Shape<BN>::kThreads, 1)
    e2m1_logits_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                       const __grid_constant__ CUtensorMap map_x_last, const __grid_constant__ E2m1Product p, int v_tiles,
                       int x_tiles, int last_rows) {
    using Sh = E2m1Shape<BN>;
    constexpr int S = Sh::kStages;
    extern __shared__ unsigned char e2m1_smem[];
    __shared__ E2m1Smem<BN> sm;
    unsigned char *const ring =
        reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(e2m1_smem) + 1023) & ~uintptr_t(1023));
    unsigned char *const ring_x = ring + S * Sh::kStageW;
    unsigned char *const ring_s = ring_x + S * Sh::kStageX;  // per stage: scales of W, then of x
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tiles64 = e2m1_tiles(p.d), n_stages = (tiles64 + Sh::kSteps - 1) / Sh::kSteps;  // of a tile
    const int64_t total = static_cast<int64_t>(v_tiles) * x_tiles;
    volatile int *const abort = &sm.abort;
    volatile int never = 0;

    if (tid == 0) {
        tma_prefetch_map(&map_w);
        tma_prefetch_map(&map_x);
        tma_prefetch_map(&map_x_last);
        for (int s = 0; s < S; ++s) {
            mbar_init(&sm.full[s], 2);
            mbar_init(&sm.scaled[s], 4);
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.acc_full[b], 1);
            mbar_init(&sm.acc_empty[b], Sh::kEpilogueWarps);
        }
        mbar_init(&sm.final_bar, 1);
        sm.abort = sm.any_far = 0;
        fence_mbar_init();
    }
    if (warp == 2) {
        tmem_alloc(&sm.tmem_base, 512);
        tmem_relinquish();
        tc_fence_before_sync();
    }
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sm.tmem_base;
    griddep_launch_dependents();
    // The inputs may come from the kernels before this one.
    if (warp != 0 || !p.w_ready) griddep_wait();

    // Tiles: x fastest, so that the CTAs that share rows of W run together.
    if (warp == 0 || warp == 3) {
        // ---------------- producers: W (warp 0), x (warp 3) ----------------
        // One thread alone would be what a stage waits for: a few hundred cycles for
        // its wait, its expected bytes and four or five copies.
        if (lane == 0) {
            const bool of_w = warp == 0;
            // W that is read again for the next tile of x stays in L2 without a mark.  Marked as
            // the last to be evicted, 128256 x 2048 for 2048 rows takes 257 us instead of 260, but
            // such lines outlive the kernel: sums of 100 MB, read again and again, take 25.6 us
            // after it for good, and 17.4 without.  x may have the mark up to what L2 does not miss
            // (2.4 MB: 17.4; 9 MB 21.5).
            const uint64_t policy = of_w ? x_tiles == 1 ? l2_evict_first_policy() : l2_normal_policy()
                                    : p.n * e2m1_pitch(p.d) <= kMarkedBytes ? l2_evict_last_policy() : l2_normal_policy();
            unsigned char *const codes = of_w ? ring : ring_x;
            const int stage_codes = of_w ? Sh::kStageW : Sh::kStageX;
            const int sets = of_w ? 1 : Sh::kXTiles;
            const int64_t last_x_tile = (p.n - 1) / kE2m1TileRows;
            int s = 0, issued = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int64_t t = blockIdx.x; ok && t < total; t += gridDim.x) {
                const int64_t vt = t / x_tiles;
                const int xt = static_cast<int>(t - vt * x_tiles);
                const int y = of_w ? static_cast<int>(vt * kE2m1TileRows) : xt * BN;
                // The last tile of x has a box of its own: rows that are not there cost a TMA
                // load time as well (100003 x 1000 for 129 rows of x: 21.2 us, 23.8 with them).
                // What lies in shared memory behind them gives columns that are not stored.
                const bool last = xt == x_tiles - 1;
                const CUtensorMap *const map = of_w ? &map_w : last ? &map_x_last : &map_x;
                const int box = of_w ? Sh::kBoxW : Sh::kBoxX, box_bytes = !of_w && last ? last_rows * 128 : box;
                const uint8_t *from[2];
                if (of_w) {
                    from[0] = from[1] = p.w_scales + vt * tiles64 * kE2m1TileBytes;
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {  // a tile beyond the last is not stored: any scales do for it
                        const int64_t rt = min(static_cast<int64_t>(xt) * BN / kE2m1TileRows + i, last_x_tile);
                        from[i] = p.x_scales + rt * tiles64 * kE2m1TileBytes;
                    }
                }
                for (int k = 0; k < n_stages; ++k) {
                    if (issued >= S && !mbar_wait(&sm.empty[s], ph ^ 1u, abort)) {
                        ok = false;
                        break;
                    }
                    const int steps = min(Sh::kSteps, tiles64 - k * Sh::kSteps);
                    const int boxes = (steps + kE2m1KbTiles - 1) / kE2m1KbTiles;
                    const uint32_t bytes = static_cast<uint32_t>(steps * kE2m1TileBytes);
                    mbar_arrive_expect_tx(&sm.full[s], boxes * box_bytes + sets * bytes);
#pragma unroll
                    for (int i = 0; i < Sh::kBlocks; ++i)
                        if (i < boxes)
                            tma_load_2d(codes + s * stage_codes + i * box, map, (k * Sh::kBlocks + i) * 128, y, &sm.full[s],
                                        policy);
                    unsigned char *const sc = ring_s + (s * (1 + Sh::kXTiles) + (of_w ? 0 : 1)) * Sh::kSet;
                    bulk_g2s(sc, from[0] + k * Sh::kSet, bytes, &sm.full[s], policy);
                    if (sets > 1) bulk_g2s(sc + Sh::kSet, from[1] + k * Sh::kSet, bytes, &sm.full[s], policy);
                    ++issued;
                    if (++s == S) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
            }
            if (!ok) {
                give_up(p.flag, &sm.abort);
                for (int i = max(0, issued - S); i < issued; ++i)  // copies in flight land before the CTA ends
                    mbar_wait(&sm.full[i % S], (i / S) & 1, &never);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_e2m1_f32(kE2m1TileRows, BN);  // (narrower last tiles cost all of them 2 %)
            int s = 0, ti = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int64_t t = blockIdx.x; ok && t < total; t += gridDim.x, ++ti) {
                const int b = ti % Sh::kBuffers, ub = ti / Sh::kBuffers;
                if (ub > 0 && !mbar_wait(&sm.acc_empty[b], (ub - 1) & 1, abort)) {
                    ok = false;
                    break;
                }
                const uint32_t acc = tmem + static_cast<uint32_t>(b * BN);
                for (int k = 0; k < n_stages; ++k) {
                    if (!mbar_wait(&sm.full[s], ph, abort) || !mbar_wait(&sm.scaled[s], ph, abort)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                    const int steps = tiles64 - k * Sh::kSteps;  // of this stage and those behind it
                    const uint32_t sfa = tmem + Sh::kScaleBase + s * Sh::kScaleCols;
                    const uint32_t sfb = sfa + 4 * Sh::kSteps;
                    const uint64_t ad = umma_desc_k_sw128(ring + s * Sh::kStageW);
                    const uint64_t bd = umma_desc_k_sw128(ring_x + s * Sh::kStageX);
#pragma unroll
                    for (int j = 0; j < Sh::kSteps; ++j) {
                        constexpr int kInBox = kE2m1KbTiles;  // steps of 32 bytes in a box of 128
                        const uint64_t at_w = j / kInBox * (Sh::kBoxW >> 4) + j % kInBox * 2;
                        const uint64_t at_x = j / kInBox * (Sh::kBoxX >> 4) + j % kInBox * 2;
                        if (j < steps)
                            umma_e2m1(acc, ad + at_w, bd + at_x, idesc, sfa + 4 * j, sfb + 4 * Sh::kXTiles * j,
                                      (k | j) != 0 ? 1u : 0u);
                    }
                    umma_commit(&sm.empty[s]);
                    if (++s == S) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                if (ok) umma_commit(&sm.acc_full[b]);
            }
            if (!ok) give_up(p.flag, &sm.abort);
            umma_commit(&sm.final_bar);  // every MMA has finished before TMEM is freed
            mbar_wait(&sm.final_bar, 0, &never);
        }
        __syncwarp();
    } else if (warp >= Sh::kScaleWarp) {
        // ---------------- scales: shared memory -> TMEM ----------------
        const uint32_t cols = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16) + Sh::kScaleBase;
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int64_t t = blockIdx.x; ok && t < total; t += gridDim.x) {
            for (int k = 0; k < n_stages; ++k) {
                if (!mbar_wait(&sm.full[s], ph, abort)) {
                    if (lane == 0) give_up(p.flag, &sm.abort);
                    ok = false;
                    break;
                }
                // The MMAs that read these columns are over (their commit freed the stage that
                // `full` says is filled again): the stores to them come behind that.
                tc_fence_after_sync();
                // (what lies behind the matrix's last scales is not used by an MMA)
                const uint4 *const sc = reinterpret_cast<const uint4 *>(ring_s + s * (1 + Sh::kXTiles) * Sh::kSet) + lane;
                constexpr int kTile = kE2m1TileBytes / 16, kSet = Sh::kSet / 16;
                const uint32_t at = cols + s * Sh::kScaleCols;
                uint32_t r[16];
                auto gather = [&](int j, const uint4 &w) { r[j] = w.x, r[j + 1] = w.y, r[j + 2] = w.z, r[j + 3] = w.w; };
#pragma unroll
                for (int h = 0; h < Sh::kBlocks; ++h) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) gather(4 * j, sc[(4 * h + j) * kTile]);
                    tmem_st_32x32b_x16(at + 16 * h, r);
                }
#pragma unroll
                for (int h = 0; h < Sh::kBlocks * Sh::kXTiles; ++h) {  // x: step 0 of each tile of rows, step 1, ...
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int step = (4 * h + j) / Sh::kXTiles, i = (4 * h + j) % Sh::kXTiles;
                        gather(4 * j, sc[(1 + i) * kSet + step * kTile]);
                    }
                    tmem_st_32x32b_x16(at + 16 * (Sh::kBlocks + h), r);
                }
                tmem_wait_st();
                tc_fence_before_sync();
                if (lane == 0) mbar_arrive(&sm.scaled[s]);
                if (++s == S) {
                    s = 0;
                    ph ^= 1u;
                }
            }
        }
    } else if (warp >= 4) {
        // ---------------- epilogue ----------------
        constexpr int kCols = Sh::kWarpCols, kChunk = kCols < 32 ? kCols : 32;
        const int quarter = warp & 3, c0 = (warp - 4) / 4 * kCols;
        float *const x_scale = sm.x_scale[warp - 4];
        int ti = 0, last_xt = -1;
        for (int64_t t = blockIdx.x; t < total; t += gridDim.x, ++ti) {
            const int b = ti % Sh::kBuffers, ub = ti / Sh::kBuffers;
            const int64_t vt = t / x_tiles;
            const int xt = static_cast<int>(t % x_tiles);
            const int64_t i0 = static_cast<int64_t>(xt) * BN, v = vt * kE2m1TileRows + 32 * quarter + lane;
            if (xt != last_xt) {
                __syncwarp();  // the scales of the last tile have been read
                float least = INFINITY, largest = 0.0f, lowest = 1.0f;
                for (int c = lane; c < kCols; c += 32) {
                    const bool real = i0 + c0 + c < p.n;
                    const float s = real ? p.x_row_scales[i0 + c0 + c] : 0.0f;
                    x_scale[c] = s;
                    if (real && s > 0x1p-126f) least = fminf(least, s), largest = fmaxf(largest, s);
                    else if (real && s <= 0x1p-126f) lowest = s;
                }
                least = -warp_max(-least), largest = warp_max(largest), lowest = -warp_max(-lowest);
                if (lane == 0) sm.x_range[warp - 4].set(least, largest, lowest);
                __syncwarp();
                last_xt = xt;
            }
            const float tv = v < p.V ? p.w_row_scales[v] : 0.0f;
            const int rows = static_cast<int>(min(static_cast<int64_t>(kCols), p.n - i0 - c0));
            ColumnStore<T, WORDS> put(static_cast<T *>(p.out) + (i0 + c0) * p.ld, p.ld, v, p.V, rows);
            if (!mbar_wait(&sm.acc_full[b], ub & 1, abort)) {
                if (lane == 0) give_up(p.flag, &sm.abort);
                break;
            }
            tc_fence_after_sync();
            const uint32_t acc = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + b * BN + c0;
            // The accumulator is handed back as soon as its last columns are in registers:
            // 64 of fp32, or 128 rounded to bf16.
            auto scaled = [&](uint32_t sum, int c) { return __uint_as_float(sum) * (x_scale[c] * tv); };
            auto hand_back = [&] {
                tc_fence_before_sync();
                if (lane == 0) mbar_arrive(&sm.acc_empty[b]);
                if (v < p.V && sm.x_range[warp - 4].may_be_far(tv))
                    for (int c = 0; c < kCols; ++c)  // (of columns beyond the last, s is 0)
                        if (is_far(x_scale[c], tv)) *static_cast<volatile int *>(&sm.any_far) = 1;
            };
            if constexpr (sizeof(T) == 2 && kCols == 128) {
                uint32_t r[64];
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    uint32_t part[32];
                    tmem_ld_32x32b_x32(acc + c, part);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; j += 2)
                        r[(c + j) / 2] = pack_bf16(scaled(part[j], c + j), scaled(part[j + 1], c + j + 1));
                }
                hand_back();
#pragma unroll
                for (int c = 0; c < kCols; c += 2) put.pair(c, r[c / 2]);
            } else {
                constexpr int kHeld = kCols < 64 ? kCols : 64, kFirst = kCols - kHeld;
#pragma unroll
                for (int c = 0; c < kFirst; c += 32) {
                    uint32_t part[32];
                    tmem_ld_32x32b_x32(acc + c, part);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; j += 2)
                        put.pair(c + j, scaled(part[j], c + j), scaled(part[j + 1], c + j + 1));
                }
                uint32_t r[kHeld];
#pragma unroll
                for (int c = 0; c < kHeld; c += kChunk) {
                    const uint32_t at = acc + kFirst + c;
                    if constexpr (kChunk == 32) tmem_ld_32x32b_x32(at, reinterpret_cast<uint32_t(&)[32]>(r[c]));
                    else tmem_ld_32x32b_x16(at, reinterpret_cast<uint32_t(&)[16]>(r[c]));
                }
                tmem_wait_ld();
                hand_back();
#pragma unroll
                for (int c = 0; c < kHeld; c += 2)
                    put.pair(kFirst + c, scaled(r[c], kFirst + c), scaled(r[c + 1], kFirst + c + 1));
            }
        }
    }
    __syncthreads();
    if (warp == 2) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
    if (sm.any_far && sm.abort == 0)
        for (int64_t t = blockIdx.x; t < total; t += gridDim.x)
            far_results<T>(p, t / x_tiles * kE2m1TileRows, t % x_tiles * BN, BN);
}

template <int BN, typename T, bool WORDS>
static cudaError_t start_e2m1_logits(const E2m1Product &p, cudaStream_t stream) {
    using Sh = E2m1Shape<BN>;
    auto kernel = e2m1_logits_kernel<BN, T, WORDS>;
    static PerDevice prepared;
    cudaError_t e = prepared.once(
        [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem); });
    int sms = 0;
    if (e == cudaSuccess) e = sm_count(&sms);
    if (e != cudaSuccess) return e;
    const uint64_t pitch = static_cast<uint64_t>(e2m1_pitch(p.d));
    const int x_tiles = static_cast<int>((p.n + BN - 1) / BN);
    const int last_rows = static_cast<int>(p.n - static_cast<int64_t>(x_tiles - 1) * BN + 7) / 8 * 8;  // BN at most
    CUtensorMap map_w, map_x, map_x_last;
    if (!make_map_u8(&map_w, const_cast<uint8_t *>(p.w_codes), static_cast<uint64_t>(p.V), pitch, pitch, kE2m1TileRows) ||
        !make_map_u8(&map_x_last, const_cast<uint8_t *>(p.x_codes), static_cast<uint64_t>(p.n), pitch, pitch,
                     static_cast<uint32_t>(last_rows)))
        return cudaErrorInvalidValue;
    map_x = map_x_last;  // (the only one where there is one tile)
    if (x_tiles > 1 && !make_map_u8(&map_x, const_cast<uint8_t *>(p.x_codes), static_cast<uint64_t>(p.n), pitch, pitch, BN))
        return cudaErrorInvalidValue;
    const int v_tiles = static_cast<int>((p.V + kE2m1TileRows - 1) / kE2m1TileRows);
    const int64_t total = static_cast<int64_t>(v_tiles) * x_tiles;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(static_cast<unsigned>(total < sms ? total : sms));
    cfg.blockDim = dim3(Sh::kThreads);
    cfg.dynamicSmemBytes = Sh::kSmem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, map_w, map_x, map_x_last, p, v_tiles, x_tiles, last_rows);
}

// Tiles as wide as the rows of x: every column of an MMA costs time, whether it is
// stored or not.  Above 128 rows tiles of 256 are the faster ones at nearly all sizes
// (128256 x 2048 bf16, us with tiles of 256 / of 128: 129 rows 35 / 46, 256 42 / 47, 512 72 / 86,
// 2048 254 / 327; 100003 x 1000, 200 rows 24.8 / 24.0): they read W once per 256 rows.
template <typename T, bool WORDS>
static cudaError_t start_by_rows(const E2m1Product &p, cudaStream_t stream) {
    if (p.n <= 16) return start_e2m1_logits<16, T, WORDS>(p, stream);
    if (p.n <= 32) return start_e2m1_logits<32, T, WORDS>(p, stream);
    if (p.n <= 64) return start_e2m1_logits<64, T, WORDS>(p, stream);
    if (p.n <= 128) return start_e2m1_logits<128, T, WORDS>(p, stream);
    return start_e2m1_logits<256, T, WORDS>(p, stream);
}

cudaError_t launch_e2m1_logits(const E2m1Product &p, vie_dtype dtype, cudaStream_t stream) {
    if (dtype == VIE_DTYPE_F32) return start_by_rows<float, false>(p, stream);
    const bool words = p.V % 2 == 0 && (p.n == 1 || p.ld % 2 == 0) && aligned_to(p.out, 4);
    return words ? start_by_rows<__nv_bfloat16, true>(p, stream)
                 : start_by_rows<__nv_bfloat16, false>(p, stream);
}

}  // namespace vie
