// vie_e2m1.cu - a head in microscaled 4-bit floating point: quantisation of rows,
// the values that they stand for, and full logits (vie_e2m1.cuh has the format).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

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
};

constexpr int kQuantizeThreads = 256;

// Block b of a row, 0 beyond it.
template <typename T>
__device__ __forceinline__ void load_block(const T *row, int b, int d, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = b * 16 + i < d ? load_value(row + b * 16 + i) : 0.0f;
}

// A warp per row, a block of 16 values per lane, twice: for the row's largest
// magnitude, and for its codes.
template <typename T, typename TV>
__global__ void __launch_bounds__(kQuantizeThreads) quantize_kernel(const QuantizeParams a) {
    const int lane = threadIdx.x & 31;
    const int64_t r = (static_cast<int64_t>(blockIdx.x) * kQuantizeThreads + threadIdx.x) >> 5;
    const int tiles = e2m1_tiles(a.d), code_blocks = 2 * ((a.d + 31) / 32);
    griddep_launch_dependents();
    griddep_wait();
    const bool real = r < a.n;
    const T *row = static_cast<const T *>(a.x) + r * a.ld;
    uint32_t top = 0;
    if (real)
        for (int b = lane; b * 16 < a.d; b += 32) {
            float v[16];
            load_block(row, b, a.d, v);
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const bool finite = top < 0x7F800000u;
    const int E = e2m1_exponent(finite ? top : 0u);
    const float scale = power_of_two(E), inv = power_of_two(-E);
    for (int b = lane; b < 4 * tiles; b += 32) {
        float v[16];
        uint32_t sigma8 = 0;
        float sigma = 0.0f;
        uint32_t codes[2] = {0, 0};
        const bool inside = real && b * 16 < a.d;
        if (inside && finite) {
            load_block(row, b, a.d, v);
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[i] *= inv;
                m = fmaxf(m, fabsf(v[i]));
            }
            sigma8 = to_e4m3(__fdiv_rn(m, 6.0f));
            sigma = from_e4m3(sigma8);
            if (sigma8 != 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __fdiv_rn(v[i], sigma);
                codes[0] = to_e2m1(v);
                codes[1] = to_e2m1(v + 8);
            }
        }
        if (r < (a.n + kE2m1TileRows - 1) / kE2m1TileRows * kE2m1TileRows)
            a.scales[e2m1_scale_at(r, b, tiles)] = static_cast<uint8_t>(sigma8);
        if (real && b < code_blocks)
            *reinterpret_cast<uint2 *>(a.codes + r * e2m1_pitch(a.d) + b * 8) = make_uint2(codes[0], codes[1]);
        if (a.values != nullptr && inside) {
            TV *out = static_cast<TV *>(a.values) + r * a.ld_values + b * 16;
            from_e2m1(codes[0], v);
            from_e2m1(codes[1], v + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (b * 16 + i < a.d) store_value(out + i, finite ? v[i] * sigma * scale : NAN);
        }
    }
    if (lane == 0 && real) a.row_scales[r] = finite ? scale : NAN;
}

struct E2m1Matrix {
    const uint8_t *codes, *scales;
    const float *row_scales;
    int64_t n;
};

__device__ __forceinline__ void e2m1_block(const E2m1Matrix &q, int64_t r, int b, int d, float (&v)[16]) {
    const uint2 c = *reinterpret_cast<const uint2 *>(q.codes + r * e2m1_pitch(d) + b * 8);
    const float sigma = from_e4m3(q.scales[e2m1_scale_at(r, b, e2m1_tiles(d))]);
    from_e2m1(c.x, v);
    from_e2m1(c.y, v + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= sigma;
}

// A thread per block.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const E2m1Matrix q, int d, T *out, int64_t ld) {
    const int blocks = (d + 15) / 16;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, r = i / blocks;
    const int b = static_cast<int>(i % blocks);
    griddep_launch_dependents();
    griddep_wait();
    if (r >= q.n) return;
    float v[16];
    e2m1_block(q, r, b, d, v);
    const float s = q.row_scales[r];
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (b * 16 + j < d) store_value(out + r * ld + b * 16 + j, v[j] * s);
}

template <typename... P, typename... A>
static cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
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

template <typename T>
static cudaError_t start_quantize(const QuantizeParams &p, vie_dtype values_dtype, cudaStream_t s) {
    const int64_t rows = (p.n + kE2m1TileRows - 1) / kE2m1TileRows * kE2m1TileRows;
    const dim3 grid(static_cast<unsigned>(rows * 32 / kQuantizeThreads));
    return values_dtype == VIE_DTYPE_BF16 ? launch(quantize_kernel<T, __nv_bfloat16>, grid, kQuantizeThreads, s, p)
                                          : launch(quantize_kernel<T, float>, grid, kQuantizeThreads, s, p);
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
    if (st != VIE_OK || n == 0) return st;
    QuantizeParams p = {};
    p.x = x, p.n = n, p.d = d, p.ld = ld;
    p.codes = static_cast<uint8_t *>(out_codes), p.scales = static_cast<uint8_t *>(out_scales);
    p.row_scales = out_row_scales, p.values = out_values, p.ld_values = ld_values;
    if (out_values == nullptr) values_dtype = VIE_DTYPE_F32;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == VIE_DTYPE_BF16 ? start_quantize<__nv_bfloat16>(p, values_dtype, s)
                                                  : start_quantize<float>(p, values_dtype, s);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_e2m1_dequantize(const void *codes, const void *scales, const float *row_scales, int64_t n, int32_t d,
                               void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream) {
    const char *fn = "vie_e2m1_dequantize";
    vie_status st = check_shape(fn, n, d);
    if (st == VIE_OK) st = check_e2m1(fn, n, codes, scales, row_scales);
    if (st == VIE_OK) st = check_matrix(fn, "out", out, out_dtype, n, d, ld_out);
    if (st != VIE_OK || n == 0) return st;
    const E2m1Matrix q = {static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), row_scales, n};
    const dim3 grid(static_cast<unsigned>((n * ((d + 15) / 16) + 255) / 256));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e =
        out_dtype == VIE_DTYPE_BF16
            ? launch(dequantize_kernel<__nv_bfloat16>, grid, 256, s, q, d, static_cast<__nv_bfloat16 *>(out), ld_out)
            : launch(dequantize_kernel<float>, grid, 256, s, q, d, static_cast<float *>(out), ld_out);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

vie_status vie_e2m1_logits(const void *x_codes, const void *x_scales, const float *x_row_scales, int64_t n,
                           const void *w_codes, const void *w_scales, const float *w_row_scales, int64_t V, int32_t d,
                           void *out, vie_dtype out_dtype, int64_t ld_out, vie_stream stream) {
    const char *fn = "vie_e2m1_logits";
    vie_status st = check_shape(fn, V, d);
    if (st == VIE_OK && V < 1) st = fail(VIE_ERR_INVALID_ARG, "%s: V=0", fn);
    if (st == VIE_OK && (n < 0 || n > VIE_MANY_MAX))
        st = fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_MANY_MAX);
    if (st == VIE_OK) st = check_e2m1(fn, n, x_codes, x_scales, x_row_scales);
    if (st == VIE_OK) st = check_e2m1(fn, n == 0 ? 0 : V, w_codes, w_scales, w_row_scales);
    if (st == VIE_OK) st = check_matrix(fn, "out", out, out_dtype, n, V, ld_out);
    if (st != VIE_OK || n == 0) return st;
    const E2m1Matrix x = {static_cast<const uint8_t *>(x_codes), static_cast<const uint8_t *>(x_scales), x_row_scales, n};
    const E2m1Matrix w = {static_cast<const uint8_t *>(w_codes), static_cast<const uint8_t *>(w_scales), w_row_scales, V};
    E2m1Product p = {};
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    p.x_scales = x.scales, p.w_scales = w.scales, p.x_row_scales = x.row_scales, p.w_row_scales = w.row_scales;
    p.out = out, p.ld = ld_out, p.n = n, p.V = V, p.d = d;
    e = launch_e2m1_logits(p, x.codes, w.codes, out_dtype, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

}  // extern "C"
