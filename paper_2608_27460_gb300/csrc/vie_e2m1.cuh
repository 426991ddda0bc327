// vie_e2m1.cuh - matrices in microscaled 4-bit floating point: the layout in
// memory, and conversions of blocks of 16 values.
//
// A row x of d values has a power of two s = 2^E, E the least whole number (-126
// at the least) with max |x| <= 6 * 448 * 2^E; each block of 16 values has a scale
// sigma = e4m3(max |x| over it / (6 s)); a value's code is e2m1(x / (s sigma)), and
// stands for code * sigma * s.  Roundings are to nearest, ties to even; a code is
// at most 6 in magnitude (sigma may have been rounded down), and that of a value that
// rounds to 0 is 0 whatever its sign (the code of -0 is not used).  sigma in e4m3 and s
// apart cover what sigma in fp32 would; that s is a power of two makes the
// scaling of values and results exact.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace vie {

constexpr int kE2m1TileRows = 128;    // rows of a tile of scales
constexpr int kE2m1TileBytes = 512;   // 128 rows x 4 scales

// Bytes of a row of codes: two to a byte, the even column in the low half.
__host__ __device__ inline int64_t e2m1_pitch(int d) { return static_cast<int64_t>((d + 31) / 32) * 16; }
__host__ __device__ inline int e2m1_tiles(int d) { return (d + 63) / 64; }
// Where the scale of row r and block b lies: tiles [row / 128][b / 4] of 32 x 4 x 4
// bytes, as the tensor cores' scale memory wants them (row % 32, row / 32 % 4, b % 4).
__host__ __device__ inline int64_t e2m1_scale_at(int64_t r, int b, int tiles) {
    return ((r / kE2m1TileRows) * tiles + b / 4) * kE2m1TileBytes + (r % 32) * 16 + (r / 32 % 4) * 4 + b % 4;
}

// e4m3 of a value >= 0, and back.
__device__ __forceinline__ uint32_t to_e4m3(float v) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
    return r & 0xFFu;
}
__device__ __forceinline__ float from_e4m3(uint32_t b) {
    uint32_t h;  // two halves
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(b)));
    float f;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.f32.f16 %0, lo;\n\t}" : "=f"(f) : "r"(h));
    return f;
}
// Eight values to e2m1 codes, the first in the lowest four bits.
__device__ __forceinline__ uint32_t to_e2m1(const float *v) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r & (((r & 0x77777777u) + 0x77777777u) | 0x77777777u);  // + 7 reaches a sign where the magnitude is not 0
}
// Eight codes to values.
__device__ __forceinline__ void from_e2m1(uint32_t codes, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h;
        asm("{\n\t.reg .b8 a;\n\tcvt.u8.u32 a, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}"
            : "=r"(h)
            : "r"(codes >> (8 * i) & 0xFFu));
        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.f32.f16 %0, lo;\n\tcvt.f32.f16 %1, hi;\n\t}"
            : "=f"(v[2 * i]), "=f"(v[2 * i + 1])
            : "r"(h));
    }
}

// E of a row whose largest magnitude has these bits (finite): max <= 1.3125 * 2^11 * 2^E.
__device__ __forceinline__ int e2m1_exponent(uint32_t top) {
    const int e = static_cast<int>(top >> 23) - 127 - 11 + ((top & 0x7FFFFFu) > 0x280000u ? 1 : 0);
    return e < -126 ? -126 : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

}  // namespace vie
