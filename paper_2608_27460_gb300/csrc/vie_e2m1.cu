// vie_e2m1.cu - a head in microscaled 4-bit floating point: quantisation of rows,
// the values that they stand for, and full logits (vie_e2m1.cuh has the format).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <type_traits>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"
#include "vie_e2m1.cuh"
#include "vie_e2m1_logits.h"

namespace vie {

struct QuantizeParams {
    const void *x;
    uint8_t *codes, *scales;
    float *row_scales;
    void *values;  // or NULL
    int64_t n, ld, ld_values;
    int d;
    int late;  // the next kernel may read what the kernels before this one have written, as soon as it starts
};

constexpr int kQuantizeThreads = 256;
constexpr int kQuantizeWarps = kQuantizeThreads / 32;

// a / b from r = 1 / b to an ulp or two, without over- or underflow in between: one
// correction of q = a r by its remainder (Markstein, "Computation of elementary
// functions on the IBM RISC System/6000 processor", 1990).  With b of few bits the
// remainder is exact and the result off by 2^-45 before its rounding: where a / b is a
// midpoint of codes or scales it is that number, and where it is not (half an ulp
// away or more, a having 24 bits) it is another.
__device__ __forceinline__ float quotient(float a, float b, float r) {
    const float q = a * r;
    return fmaf(fmaf(-q, b, a), r, q);
}
__device__ __forceinline__ float reciprocal_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// words[i] = all[i + first], first < 4 (the same in all lanes), without indexing registers.
template <int N>
__device__ __forceinline__ void take_words(const uint32_t (&all)[N], int first, uint32_t (&words)[N - 3]) {
    uint32_t by2[N - 2];
#pragma unroll
    for (int i = 0; i < N - 2; ++i) by2[i] = (first & 2) != 0 ? all[i + 2] : all[i];
#pragma unroll
    for (int i = 0; i < N - 3; ++i) words[i] = (first & 1) != 0 ? by2[i + 1] : by2[i];
}

// Eight values of a row as they are stored, 0 beyond it.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint32_t w[4];
    // Of a row at a 16-byte address.
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, int left) {
        if (left >= 8) {
            const uint4 a = *reinterpret_cast<const uint4 *>(p);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
            return;
        }
        const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = (2 * i < left ? q[2 * i] : 0u) | (2 * i + 1 < left ? static_cast<uint32_t>(q[2 * i + 1]) << 16 : 0u);
    }
    // Of one `shift` bytes behind such an address: vectors at such addresses that hold a
    // value of the row are read whole.
    __device__ __forceinline__ void load_shifted(const __nv_bfloat16 *p, int left, int shift) {
        const uint4 *const v = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) - shift);
        const uint4 a = v[0], b = shift + 2 * left > 16 ? v[1] : make_uint4(0, 0, 0, 0);
        const uint32_t all[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint32_t words[5];
        take_words(all, shift / 4, words);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(words[i], words[i + 1], 8 * (shift % 4));
        if (left < 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (2 * i >= left) w[i] = 0;
                else if (2 * i + 1 >= left) w[i] &= 0xFFFFu;
            }
        }
    }
    // The largest magnitude, as the bits of an fp32 value (NaN above infinity).
    __device__ __forceinline__ uint32_t top() const {
        const uint32_t m = 0x7FFF7FFFu;
        const uint32_t t = __vmaxu2(__vmaxu2(w[0] & m, w[1] & m), __vmaxu2(w[2] & m, w[3] & m));
        return max(t << 16, t & 0xFFFF0000u);
    }
    __device__ __forceinline__ float value(int i) const { return i % 2 == 0 ? bf16_lo(w[i / 2]) : bf16_hi(w[i / 2]); }
    __device__ __forceinline__ void scale(float by) {  // a power of two that leaves them exact
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(bf16_lo(w[i]) * by, bf16_hi(w[i]) * by);
    }
    // x_i / b as far as it decides codes, from r = 1 / b to an ulp or two.  Of x b^-1 with 8
    // bits of x and 4 of b, what is not a midpoint of codes is 2^-10 or more from all of
    // them: rounded to multiples of 2^-10 (the sum's last place), the others are exact.
    __device__ __forceinline__ void quotients(float, float r, float *v) const {
        constexpr float kShift = 12288.0f;  // 1.5 * 2^13
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(value(i), r, kShift) - kShift;
    }
};
template <>
struct Raw8<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float *p, int left) {
        if (left >= 8) {
            const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i < left ? __float_as_uint(p[i]) : 0u;
    }
    __device__ __forceinline__ void load_shifted(const float *p, int left, int shift) {
        const uint4 *const v = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) - shift);
        const uint4 none = make_uint4(0, 0, 0, 0), a = v[0], b = shift + 4 * left > 16 ? v[1] : none;
        const uint4 c = shift + 4 * left > 32 ? v[2] : none;
        const uint32_t all[12] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, c.y, c.z, c.w};
        uint32_t words[9];
        take_words(all, shift / 4, words);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = words[i];
        if (left < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= left) w[i] = 0;
        }
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, w[i] & 0x7FFFFFFFu);
        return t;
    }
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void scale(float by) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(value(i) * by);
    }
    __device__ __forceinline__ void quotients(float b, float r, float *v) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = quotient(value(i), b, r);
    }
};

template <typename T>
__device__ __forceinline__ void store8(T *p, const float *v, int left) {
    if (left >= 8) {
        reinterpret_cast<uint4 *>(p)[0] = Vec16<T>::pack(v);
        if constexpr (sizeof(T) == 4) reinterpret_cast<uint4 *>(p)[1] = Vec16<T>::pack(v + 4);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) store_value(p + i, v[i]);
}

// The same for a row at any address: lane l of the warp has vector `vec` (lane 0's +
// l) of a row of `width` values, in [0, width / 8] and beyond.  What lies between two
// 16-byte addresses is of two vectors, so a lane gets the end of the one before its
// own from its neighbour; the first and last lanes' halves go value by value.
template <typename T>
__device__ __forceinline__ void store8_shifted(T *row, int vec, const float *v, int width) {
    constexpr int kWords = sizeof(T) == 2 ? 4 : 8;  // of eight values; 16 or 32 bytes
    const int lane = threadIdx.x & 31, left = width - 8 * vec;
    // values of this vector before the first 16-byte address in it (0: it starts there)
    const int head = static_cast<int>(-(reinterpret_cast<uintptr_t>(row) & 15u) & 15u) / static_cast<int>(sizeof(T));
    uint32_t own[kWords], before[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i)
        own[i] = sizeof(T) == 2 ? pack_bf16(v[2 * i % 8], v[(2 * i + 1) % 8]) : __float_as_uint(v[i]);
#pragma unroll
    for (int i = 0; i < kWords; ++i) before[i] = __shfl_up_sync(0xFFFFFFFFu, own[i], 1);
    // this lane's: the kWords words that end where its vector's values before `head` do
    const int end = 8 * vec + head, start = end - 8;  // values of the row
    T *const p = row + start;
    if (lane > 0 && end <= width) {
        uint32_t all[kWords + 4], words[kWords + 1];
#pragma unroll
        for (int i = 0; i < kWords; ++i) all[i] = before[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) all[kWords + i] = own[i];
        const int bytes = head * static_cast<int>(sizeof(T));
        take_words(all, bytes / 4, words);
        uint4 q[kWords / 4];
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i)
            q[i] = make_uint4(__funnelshift_r(words[4 * i], words[4 * i + 1], 8 * (bytes % 4)),
                              __funnelshift_r(words[4 * i + 1], words[4 * i + 2], 8 * (bytes % 4)),
                              __funnelshift_r(words[4 * i + 2], words[4 * i + 3], 8 * (bytes % 4)),
                              __funnelshift_r(words[4 * i + 3], words[4 * i + 4], 8 * (bytes % 4)));
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) reinterpret_cast<uint4 *>(p)[i] = q[i];
    }
    // value by value: this vector's own before `head` where no whole 16 bytes were
    // written there, and its others where the next lane has not written them
    const bool next_whole = lane < 31 && end + 8 <= width;
    const bool whole = lane > 0 && end <= width;
    if (!whole || !next_whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left && (i < head ? !whole : !next_whole)) store_value(row + 8 * vec + i, v[i]);
    }
}

struct None {};  // no values wanted

// Rows to codes and scales: a row in registers, its largest magnitude, its codes.  A
// lane takes eight values at a time, two lanes a block.
//
// ROW_WARPS 1: a warp per row, a CTA for 32 rows of a tile, 8 at a time: the four
// rows of each of its warps are those whose scales lie side by side, so that the
// CTA's scales (gathered in shared memory) are written 128 bytes at a time.
// ROW_WARPS 8: a CTA per row, for the latency of few rows, and for long ones; 0: with
// fewer warps, as many as the launch has (fp32 40000 x 5120 141 us, with 256 threads of
// which three eighths are idle 246; bf16 100000 x 2560 158, 210).
// NV: vectors of eight values that a lane keeps.  SHIFTED: not all rows of x and of
// the values lie at 16-byte addresses.
//
// Bound by bytes where rows lie at 16-byte addresses: 262144 x 1152 bf16 129 us, with
// bf16 values 203 (of a copy's rate 0.88 and 1.0), fp32 197 (1.0), 30000 x 8192 bf16
// with values 175 (0.94), 100395 x 3008 262 (0.78); rows of more than 2048 columns of bf16
// without values by a CTA's chain of loads, barrier and stores (100000 x 2112 153 us, 60000 x
// 4096 143, 40000 x 5120 109: 0.52, 0.65, 0.71), narrow ones by a warp's turns (300000 x 64 55
// us, x 256 58: 0.13, 0.50).  Elsewhere by the instructions that take vectors apart and join
// them: 262144 x 1001 bf16 173 us, with values 339 (0.57 and 0.52; value by value 483), fp32
// 275 (0.64).  32 x 1152 fp32: 1.5 us.
//
// CTAs per SM: what the registers of a row leave.  They are what bounds a warp per row,
// and vectors that it does not have cost as many, so NV goes by one there (262144 x 1152
// bf16: five vectors 127 us, with values 202; eight 145 and 225; fp32 196, 234: before zeros
// had one code, which costs 1 to 3 %).
template <typename T, typename TV, int ROW_WARPS, int NV>
constexpr int quantize_ctas() {
    const bool values = !std::is_same<TV, None>::value;
    if (sizeof(T) == 4) return ROW_WARPS != 1 ? (NV > 4 ? 2 : 3) : NV > 6 ? 2 : NV > 3 ? 3 : 4;
    if (ROW_WARPS != 1) return 4;
    return values ? (NV > 6 ? 3 : NV > 3 ? 4 : 5) : NV > 5 ? 4 : NV > 3 ? 5 : 6;
}

template <typename T, typename TV, int ROW_WARPS, int NV, bool SHIFTED>
__global__ void __launch_bounds__(kQuantizeThreads, quantize_ctas<T, TV, ROW_WARPS, NV>())
    quantize_kernel(const QuantizeParams a) {
    constexpr bool kMany = ROW_WARPS == 1;
    constexpr int kRounds = kMany ? 4 : 1;
    const int row_lanes = ROW_WARPS > 0 ? 32 * ROW_WARPS : static_cast<int>(blockDim.x);
    constexpr bool kValues = !std::is_same<TV, None>::value;
    extern __shared__ __align__(16) uint8_t scale_bytes[];  // kMany: [tiles][row % 8 of 32][row / 32][4]
    __shared__ uint32_t warp_top[kQuantizeWarps];
    const int warp = threadIdx.x >> 5, at = kMany ? threadIdx.x & 31 : threadIdx.x;
    const int tiles = e2m1_tiles(a.d);
    const int64_t pitch = e2m1_pitch(a.d);
    if (!a.late) griddep_launch_dependents();
    griddep_wait();
    if (a.late) griddep_launch_dependents();
    // CTA c of kMany takes rows 8 (c % 4) + 0 .. 7 of each 32 of tile c / 4
    const int64_t first = kMany ? static_cast<int64_t>(blockIdx.x / 4) * kE2m1TileRows + 8 * (blockIdx.x % 4) + warp
                                : static_cast<int64_t>(blockIdx.x);
#pragma unroll 1
    for (int round = 0; round < kRounds; ++round) {
        const int64_t r = first + 32 * round;
        const bool real = r < a.n;
        const T *const row = static_cast<const T *>(a.x) + (real ? r : 0) * a.ld;
        const int width = real ? a.d : 0;  // rows beyond the last have scales of 0 and nothing else
        [[maybe_unused]] const int shift = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15u);
        Raw8<T> raw[NV];
        uint32_t tops[NV], top = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int j = 8 * (k * row_lanes + at);
            raw[k] = {};
            if (j < width) {
                if constexpr (SHIFTED) raw[k].load_shifted(row + j, width - j, shift);
                else raw[k].load(row + j, width - j);
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            tops[k] = raw[k].top();
            top = max(top, tops[k]);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (!kMany) {
            if ((threadIdx.x & 31) == 0) warp_top[warp] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kQuantizeWarps; ++w) top = max(top, 32 * w < row_lanes ? warp_top[w] : 0u);
        }
        const bool finite = top < 0x7F800000u;
        const int E = e2m1_exponent(finite ? top : 0u);
        float scale = power_of_two(E), inv = power_of_two(-E), unit = scale;  // of quotients, of values
        if (at == 0 && real) a.row_scales[r] = finite ? scale : NAN;
        if (!finite || E < -100) {  // (sigma scale would be subnormal, its reciprocal infinite)
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                raw[k].scale(finite ? inv : 0.0f);
                if (!finite) raw[k] = {};
                tops[k] = raw[k].top();
            }
            if (!finite) unit = NAN;
            scale = inv = 1.0f;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (k * row_lanes >= 8 * tiles) break;  // (the same for all lanes: they exchange)
            const int vec = k * row_lanes + at, left = width - 8 * vec;
            const uint32_t block_top = max(tops[k], __shfl_xor_sync(0xFFFFFFFFu, tops[k], 1));
            const uint32_t sigma8 = to_e4m3(quotient(__uint_as_float(block_top) * inv, 6.0f, 1.0f / 6.0f));
            const float sigma = from_e4m3(sigma8);
            float v[8];
            raw[k].quotients(sigma * scale, sigma8 != 0 ? reciprocal_approx(sigma) * inv : 0.0f, v);
            const uint32_t codes = to_e2m1(v);
            if (vec % 2 == 0 && vec < 8 * tiles) {
                if (kMany) scale_bytes[(vec / 8) * 128 + warp * 16 + round * 4 + vec / 2 % 4] = static_cast<uint8_t>(sigma8);
                else a.scales[e2m1_scale_at(r, vec / 2, tiles)] = static_cast<uint8_t>(sigma8);
            }
            if (real && vec * 4 < pitch) *reinterpret_cast<uint32_t *>(a.codes + r * pitch + vec * 4) = codes;
            if constexpr (kValues) {
                from_e2m1(codes, v);
                const float u = sigma * unit;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= u;
                TV *const out = static_cast<TV *>(a.values) + r * a.ld_values;
                if constexpr (SHIFTED) store8_shifted(out, vec, v, width);
                else if (left > 0) store8(out + 8 * vec, v, left);
            }
        }
    }
    if (kMany) {
        __syncthreads();
        uint4 *const out = reinterpret_cast<uint4 *>(a.scales + e2m1_scale_at(first - warp, 0, tiles));
        for (int i = threadIdx.x; i < 8 * tiles; i += kQuantizeThreads)
            out[(i / 8) * (kE2m1TileBytes / 16) + i % 8] = reinterpret_cast<const uint4 *>(scale_bytes)[i];
    }
}

struct E2m1Matrix {
    const uint8_t *codes, *scales;
    const float *row_scales;
    int64_t n;
};

// What the codes stand for, a warp per row, eight values per lane, kUnpack such vectors
// read before the first is written.  A CTA's rows are two neighbours in each quarter of
// a tile of scales: the 32 bytes that are fetched for one of them are all of its.
//
// Bound by bytes: 262144 x 1152 to bf16 119 us, to fp32 203 (of a copy's rate 0.96 and
// 1.0; with one vector read at a time, rows of a CTA next to each other and a lane's fp32
// values written as one vector 173 and 252); 262144 x 1001 by what joins vectors, to bf16 211
// us, to fp32 199 (0.47 and 0.88; value by value 503 and 481).  kUnpack: 3, 5 and 8 take
// 125, 121 and 122 us at 1152 columns, 4 119.
constexpr int kUnpack = 4;
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(kQuantizeThreads) dequantize_kernel(const E2m1Matrix q, int d, T *out, int64_t ld) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t r = static_cast<int64_t>(blockIdx.x) / 16 * kE2m1TileRows + warp / 2 * 32 + blockIdx.x % 16 * 2 + warp % 2;
    griddep_launch_dependents();
    griddep_wait();
    if (r >= q.n) return;
    const float s = q.row_scales[r];
    const uint32_t *const codes = reinterpret_cast<const uint32_t *>(q.codes + r * e2m1_pitch(d));
    const int tiles = e2m1_tiles(d);
    T *const row = out + r * ld;
    for (int first = 0; first * 8 < d; first += 32 * kUnpack) {
        uint32_t word[kUnpack], sigma[kUnpack];
#pragma unroll
        for (int k = 0; k < kUnpack; ++k) {
            const int vec = first + 32 * k + lane;
            word[k] = sigma[k] = 0;
            if (vec * 8 >= d) continue;
            word[k] = codes[vec];
            sigma[k] = q.scales[e2m1_scale_at(r, vec / 2, tiles)];
        }
#pragma unroll
        for (int k = 0; k < kUnpack; ++k) {
            const int vec = first + 32 * k + lane;
            if ((first + 32 * k) * 8 >= d) break;  // (the same for all lanes: they exchange)
            const float unit = from_e4m3(sigma[k]) * s;
            float v[8];
            if constexpr (sizeof(T) == 4 && !SHIFTED) {  // a lane writes half a vector, so that the warp's 16 bytes each adjoin
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int from = 16 * h + lane / 2, c = (first + 32 * k + from) * 8 + lane % 2 * 4;
                    const uint32_t half = __shfl_sync(0xFFFFFFFFu, word[k], from) >> (lane % 2 * 16);
                    const float u = __shfl_sync(0xFFFFFFFFu, unit, from);
                    from_e2m1(half & 0xFFFFu, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] *= u;
                    if (c + 4 <= d) {
                        *reinterpret_cast<uint4 *>(row + c) = Vec16<T>::pack(v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (c + i < d) store_value(row + c + i, v[i]);
                    }
                }
            } else {
                from_e2m1(word[k], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= unit;
                if constexpr (SHIFTED) store8_shifted(row, vec, v, d);
                else if (vec * 8 < d) store8(row + 8 * vec, v, d - 8 * vec);
            }
        }
    }
}

template <typename... P, typename... A>
static cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

static vie_status check_shape(const char *fn, int64_t n, int64_t d) {
    if (n < 0 || n > VIE_E2M1_N_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_E2M1_N_MAX);
    if (d < 1 || d > VIE_D_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: d=%lld outside [1, %d]", fn, static_cast<long long>(d), VIE_D_MAX);
    return VIE_OK;
}

// Codes, scales and row scales of n rows.
static vie_status check_e2m1(const char *fn, int64_t n, const void *codes, const void *scales, const float *row_scales) {
    if (n > 0 && (codes == nullptr || scales == nullptr || row_scales == nullptr))
        return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(codes, 16) || !aligned_to(scales, 16) || !aligned_to(row_scales, 4))
        return fail(VIE_ERR_INVALID_ARG, "%s: codes and scales must be 16-byte aligned, row scales 4-byte", fn);
    return VIE_OK;
}

// No result where threads of other rows may still read an input, or write another result.
static vie_status check_apart(const char *fn, const void *result, std::initializer_list<const void *> others) {
    for (const void *p : others)
        if (result != nullptr && result == p)
            return fail(VIE_ERR_INVALID_ARG, "%s: a result in place of an input or of another result", fn);
    return VIE_OK;
}

// The longest rows that a warp takes.
template <typename T, bool SHIFTED>
constexpr int kWarpColumns = SHIFTED && sizeof(T) == 4 ? 1536 : 2048;

// Rows from which on a warp takes each.  A warp's four rows one after the other are a
// latency that few rows do not hide, a CTA per row a cost that many add up; the longer the
// rows, the later the second is the larger, up to rows of 768 columns, and the later where
// rows lie off 16-byte addresses and a warp has more to do for each (us by warps / by CTAs,
// rows of other calls in between, bf16: 64 columns, 2048 rows 2.9 / 2.5, 4096 3.4 / 4.6; 512,
// 8192 8.9 / 8.7; 1152, 6144 12.6 / 9.0, 12288 18.0 / 16.7, 16384 18.6 / 21.7; with values 1024,
// 5120 12.9 / 7.3, 1152, 8192 14.8 / 13.3, 16384 19.9 / 25.8; 401 off, 16384 14.7 / 17.1, with
// values 21.4 / 17.1, 20000 21.8 / 21.0).  Against the quicker one of the two, over 2100 calls of
// 512 to 24576 rows: 0.5 % slower on average, 23 % at the most.  Rows off 16-byte addresses of
// which a lane would keep eight vectors of fp32 are a CTA's however many they are (100000 x
// 1793 266 us by warps, 208 by CTAs).
template <typename T, typename TV, bool SHIFTED>
static bool by_warps(int64_t n, int d) {
    constexpr bool kValues = !std::is_same<TV, None>::value;
    return d <= kWarpColumns<T, SHIFTED> &&
           n >= (2000 + 12 * static_cast<int64_t>(d < 768 ? d : 768)) * (SHIFTED ? kValues ? 3 : 2 : 1);
}

// With the warps that a row's vectors keep busy, or all (nine tenths of the time of a
// kernel that has to ask; eight vectors of fp32 in 192 threads leave an SM 384 of them,
// in 256 with a quarter idle 512: 16000 x 12288 173 us, 150).
template <typename T, typename TV, int NV, bool SHIFTED>
static cudaError_t start_by_cta(const QuantizeParams &p, int64_t rows, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>(rows));
    const int threads = (8 * e2m1_tiles(p.d) / NV + 31) / 32 * 32;
    return threads > (NV == 8 ? 160 : kQuantizeThreads - 32)
               ? launch(quantize_kernel<T, TV, kQuantizeWarps, NV, SHIFTED>, grid, kQuantizeThreads, 0, s, p)
               : launch(quantize_kernel<T, TV, 0, NV, SHIFTED>, grid, threads, 0, s, p);
}

template <typename T, typename TV, bool SHIFTED>
static cudaError_t start_quantize_rows(const QuantizeParams &p, cudaStream_t s) {
    const int64_t rows = (p.n + kE2m1TileRows - 1) / kE2m1TileRows * kE2m1TileRows;  // with those that have scales alone
    if (by_warps<T, TV, SHIFTED>(p.n, p.d)) {
        const dim3 grid(static_cast<unsigned>(rows / 32));
        const size_t smem = static_cast<size_t>(e2m1_tiles(p.d)) * 128;
        auto by_warp = [&](auto kernel) { return launch(kernel, grid, kQuantizeThreads, smem, s, p); };
        if (p.d <= 768) return by_warp(quantize_kernel<T, TV, 1, 3, SHIFTED>);
        if (p.d <= 1024) return by_warp(quantize_kernel<T, TV, 1, 4, SHIFTED>);
        if (p.d <= 1280) return by_warp(quantize_kernel<T, TV, 1, 5, SHIFTED>);
        if constexpr (kWarpColumns<T, SHIFTED> > 1536)
            if (p.d > 1536) return by_warp(quantize_kernel<T, TV, 1, 8, SHIFTED>);
        return by_warp(quantize_kernel<T, TV, 1, 6, SHIFTED>);
    }
    if (p.d <= 2048) return start_by_cta<T, TV, 1, SHIFTED>(p, rows, s);
    if (p.d <= 4096) return start_by_cta<T, TV, 2, SHIFTED>(p, rows, s);
    if (p.d <= 8192) return start_by_cta<T, TV, 4, SHIFTED>(p, rows, s);
    return start_by_cta<T, TV, 8, SHIFTED>(p, rows, s);
}

template <typename T, typename TV>
static cudaError_t start_quantize(const QuantizeParams &p, cudaStream_t s) {
    bool aligned = aligned_to(p.x, 16) && (p.n == 1 || p.ld * sizeof(T) % 16 == 0);
    if constexpr (!std::is_same<TV, None>::value)
        aligned = aligned && aligned_to(p.values, 16) && (p.n == 1 || p.ld_values * sizeof(TV) % 16 == 0);
    return aligned ? start_quantize_rows<T, TV, false>(p, s) : start_quantize_rows<T, TV, true>(p, s);
}

template <typename T>
static cudaError_t start_quantize(const QuantizeParams &p, vie_dtype values_dtype, cudaStream_t s) {
    if (p.values == nullptr) return start_quantize<T, None>(p, s);
    return values_dtype == VIE_DTYPE_BF16 ? start_quantize<T, __nv_bfloat16>(p, s) : start_quantize<T, float>(p, s);
}

static cudaError_t launch_quantize(const QuantizeParams &p, vie_dtype dtype, vie_dtype values_dtype, cudaStream_t s) {
    return dtype == VIE_DTYPE_BF16 ? start_quantize<__nv_bfloat16>(p, values_dtype, s)
                                   : start_quantize<float>(p, values_dtype, s);
}

template <typename T>
static cudaError_t start_dequantize(const E2m1Matrix &q, int d, T *out, int64_t ld, cudaStream_t s) {
    static_assert(kQuantizeWarps == 8, "sixteen CTAs have a tile of rows");
    const dim3 grid(static_cast<unsigned>((q.n + kE2m1TileRows - 1) / kE2m1TileRows * 16));
    const bool aligned = aligned_to(out, 16) && (q.n == 1 || ld * sizeof(T) % 16 == 0);
    return aligned ? launch(dequantize_kernel<T, false>, grid, kQuantizeThreads, 0, s, q, d, out, ld)
                   : launch(dequantize_kernel<T, true>, grid, kQuantizeThreads, 0, s, q, d, out, ld);
}

static vie_status check_logits(const char *fn, int64_t n, int64_t V, int32_t d, const void *x_codes,
                               const void *x_scales, const float *x_row_scales, const void *w_codes,
                               const void *w_scales, const float *w_row_scales, const void *out, vie_dtype out_dtype,
                               int64_t ld_out) {
    vie_status st = check_shape(fn, V, d);
    if (st == VIE_OK && V < 1) st = fail(VIE_ERR_INVALID_ARG, "%s: V=0", fn);
    if (st == VIE_OK && (n < 0 || n > VIE_MANY_MAX))
        st = fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_MANY_MAX);
    if (st == VIE_OK) st = check_e2m1(fn, n, x_codes, x_scales, x_row_scales);
    if (st == VIE_OK) st = check_e2m1(fn, n == 0 ? 0 : V, w_codes, w_scales, w_row_scales);
    if (st == VIE_OK) st = check_matrix(fn, "out", out, out_dtype, n, V, ld_out);
    return st;
}

static vie_status start_logits(const char *fn, const void *x_codes, const void *x_scales, const float *x_row_scales,
                               int64_t n, const void *w_codes, const void *w_scales, const float *w_row_scales,
                               int64_t V, int32_t d, bool w_ready, void *out, vie_dtype out_dtype, int64_t ld_out,
                               cudaStream_t s) {
    E2m1Product p = {};
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    p.x_codes = static_cast<const uint8_t *>(x_codes), p.w_codes = static_cast<const uint8_t *>(w_codes);
    p.x_scales = static_cast<const uint8_t *>(x_scales), p.w_scales = static_cast<const uint8_t *>(w_scales);
    p.x_row_scales = x_row_scales, p.w_row_scales = w_row_scales;
    p.out = out, p.ld = ld_out, p.n = n, p.V = V, p.d = d, p.w_ready = w_ready;
    e = launch_e2m1_logits(p, out_dtype, s);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

}  // namespace vie

using namespace vie;

extern "C" {

vie_status vie_e2m1_bytes(int64_t n, int32_t d, int64_t *code_bytes, int64_t *scale_bytes) {
    const char *fn = "vie_e2m1_bytes";
    const vie_status st = check_shape(fn, n, d);
    if (st != VIE_OK) return st;
    if (code_bytes == nullptr || scale_bytes == nullptr) return fail(VIE_ERR_INVALID_ARG, "%s: NULL result", fn);
    *code_bytes = n * e2m1_pitch(d);
    *scale_bytes = (n + kE2m1TileRows - 1) / kE2m1TileRows * e2m1_tiles(d) * kE2m1TileBytes;
    return VIE_OK;
}

vie_status vie_e2m1_quantize(const void *x, vie_dtype dtype, int64_t n, int32_t d, int64_t ld, void *out_codes,
                             void *out_scales, float *out_row_scales, void *out_values, vie_dtype values_dtype,
                             int64_t ld_values, vie_stream stream) {
    const char *fn = "vie_e2m1_quantize";
    vie_status st = check_shape(fn, n, d);
    if (st == VIE_OK) st = check_matrix(fn, "x", x, dtype, n, d, ld);
    if (st == VIE_OK) st = check_e2m1(fn, n, out_codes, out_scales, out_row_scales);
    if (st == VIE_OK && out_values != nullptr)
        st = check_matrix(fn, "out_values", out_values, values_dtype, n, d, ld_values);
    if (st == VIE_OK && n > 0 && out_values == x && (values_dtype != dtype || (n > 1 && ld_values != ld)))
        st = fail(VIE_ERR_INVALID_ARG, "%s: out_values in place of x with another type or row pitch", fn);
    if (st != VIE_OK || n == 0) return st;
    st = check_apart(fn, x, {out_codes, out_scales, out_row_scales});
    if (st == VIE_OK) st = check_apart(fn, out_values, {out_codes, out_scales, out_row_scales});
    if (st != VIE_OK) return st;
    QuantizeParams p = {};
    p.x = x, p.n = n, p.d = d, p.ld = ld;
    p.codes = static_cast<uint8_t *>(out_codes), p.scales = static_cast<uint8_t *>(out_scales);
    p.row_scales = out_row_scales, p.values = out_values, p.ld_values = ld_values;
    const cudaError_t e = launch_quantize(p, dtype, values_dtype, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_e2m1_dequantize(const void *codes, const void *scales, const float *row_scales, int64_t n, int32_t d,
                               void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream) {
    const char *fn = "vie_e2m1_dequantize";
    vie_status st = check_shape(fn, n, d);
    if (st == VIE_OK) st = check_e2m1(fn, n, codes, scales, row_scales);
    if (st == VIE_OK) st = check_matrix(fn, "out", out, out_dtype, n, d, ld_out);
    if (st == VIE_OK && n > 0) st = check_apart(fn, out, {codes, scales, row_scales});
    if (st != VIE_OK || n == 0) return st;
    const E2m1Matrix q = {static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), row_scales, n};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = out_dtype == VIE_DTYPE_BF16 ? start_dequantize(q, d, static_cast<__nv_bfloat16 *>(out), ld_out, s)
                                                      : start_dequantize(q, d, static_cast<float *>(out), ld_out, s);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_e2m1_logits(const void *x_codes, const void *x_scales, const float *x_row_scales, int64_t n,
                           const void *w_codes, const void *w_scales, const float *w_row_scales, int64_t V, int32_t d,
                           void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream) {
    const char *fn = "vie_e2m1_logits";
    vie_status st = check_logits(fn, n, V, d, x_codes, x_scales, x_row_scales, w_codes, w_scales, w_row_scales, out,
                                 out_dtype, ld_out);
    if (st == VIE_OK && n > 0)
        st = check_apart(fn, out, {x_codes, x_scales, x_row_scales, w_codes, w_scales, w_row_scales});
    if (st != VIE_OK || n == 0) return st;
    return start_logits(fn, x_codes, x_scales, x_row_scales, n, w_codes, w_scales, w_row_scales, V, d, false, out,
                        out_dtype, ld_out, static_cast<cudaStream_t>(stream));
}

vie_status vie_e2m1_quantize_logits(const void *x, vie_dtype dtype, int64_t n, int64_t ld, void *x_codes,
                                    void *x_scales, float *x_row_scales, const void *w_codes, const void *w_scales,
                                    const float *w_row_scales, int64_t V, int32_t d, void *out, vie_dtype out_dtype,
                                    int64_t ld_out, vie_stream stream) {
    const char *fn = "vie_e2m1_quantize_logits";
    vie_status st = check_logits(fn, n, V, d, x_codes, x_scales, x_row_scales, w_codes, w_scales, w_row_scales, out,
                                 out_dtype, ld_out);
    if (st == VIE_OK) st = check_matrix(fn, "x", x, dtype, n, d, ld);
    if (st == VIE_OK && n > 0 && (x_codes == w_codes || x_scales == w_scales || x_row_scales == w_row_scales))
        st = fail(VIE_ERR_INVALID_ARG, "%s: x_* in place of w_*", fn);
    if (st == VIE_OK && n > 0) st = check_apart(fn, x, {x_codes, x_scales, x_row_scales});
    if (st == VIE_OK && n > 0)
        st = check_apart(fn, out, {x_codes, x_scales, x_row_scales, w_codes, w_scales, w_row_scales});
    if (st != VIE_OK || n == 0) return st;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    QuantizeParams p = {};
    p.x = x, p.n = n, p.d = d, p.ld = ld, p.late = 1;
    p.codes = static_cast<uint8_t *>(x_codes), p.scales = static_cast<uint8_t *>(x_scales), p.row_scales = x_row_scales;
    const cudaError_t e = launch_quantize(p, dtype, VIE_DTYPE_F32, s);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    return start_logits(fn, x_codes, x_scales, x_row_scales, n, w_codes, w_scales, w_row_scales, V, d, true, out,
                        out_dtype, ld_out, s);
}

}  // extern "C"
