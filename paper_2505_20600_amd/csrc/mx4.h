// Microscaled 4-bit floating point: the format's arithmetic and the launchers'
// descriptors (mx4.hip, mx4_linear.hip, block_ops_api.hip).
//
// A row of K elements (K a multiple of 32) is K/2 bytes of codes, element 2i in
// the low half of byte i, and K/32 exponent bytes b, one per 32 elements: value =
// code * 2^(b - 127). Codes are e2m1: sign, two exponent bits (bias 1), one
// mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, neither infinities
// nor NaN; b = 255 makes its 32 elements NaN. This is what the scaled matrix
// instructions take: a lane's 16 bytes of codes are 32 consecutive elements of
// one row, and its exponent byte theirs.
#pragma once

#include "common.h"
#include "kernels.h"

namespace ms {

constexpr int kMxBlock = 32;        // elements per exponent byte

// Exponent byte of a block whose largest |x| has the float32 bits `u` (finite): the
// smallest power of two s with |x| <= 7 s = 1.75 * 2^2 s, at least 2^-126 and at most
// 2^125 (6 * 2^125 is the largest value a code then has, finite in bf16 and float32);
// 1 for zeros. What lies in (6 s, 7 s] rounds to 6 s, with the error of a grid that
// went on to 8 s.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t u) {
    const int e = (int)((u + 0x1fffffu) >> 23) - 2;    // a mantissa above 0.75 carries into the exponent
    return u == 0 ? 127u : (uint32_t)min(max(e, 1), 252);
}

// 2^(127 - b) for b in 1..252.
__device__ __forceinline__ float mx4_ratio(uint32_t b) { return __uint_as_float((254u - b) << 23); }

// The exponent byte's value 2^(b - 127): b = 0 is the subnormal 2^-127, b = 255 NaN.
__device__ __forceinline__ float mx4_scale(uint32_t b) {
    return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7fc00000u : b << 23);
}

// Eight values times ratio -> eight codes, round to nearest even, |x ratio| above 6 to 6.
__device__ __forceinline__ uint32_t mx4_encode8(const float x[8], float ratio) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i] * ratio, -6.f, 6.f);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
    return w;
}

// Product of packed codes. a: the activations [M][K], w: the weights [N][K].
struct Mx4LinearDesc {
    const uint8_t *a, *as;      // codes [M][K / 2], exponent bytes [M][K / 32]
    const uint8_t *w, *ws;      // codes [N][K / 2], exponent bytes [N][K / 32]
    GemmDesc g;                 // shape, bias, residual, output, epilogue, ksplit and part; kchunk in 256-element steps
    int form;                   // set by plan_mx4_linear
    int waves;                  // of a workgroup of the form for few rows
};

// Outputs of a workgroup: 16 x 16, or tiles of 64, 128 or 256 rows and columns.
enum { kMx4Rows = 0, kMx4Tile64, kMx4Tile128, kMx4Tile256 };

hipError_t launch_mx4_quantize(int dtype, const void* x, long rows, int cols, long ld, uint8_t* codes, uint8_t* scales,
                               hipStream_t s);
hipError_t launch_mx4_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, long rows, int cols, void* x,
                                 long ld, hipStream_t s);
// Sets the form and the K split from the shape and what the caller's buffer for parts holds.
void plan_mx4_linear(Mx4LinearDesc& d, size_t part_floats);
hipError_t launch_mx4_linear(int dtype, const Mx4LinearDesc& d, hipStream_t s);

}  // namespace ms
