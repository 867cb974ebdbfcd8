// Rows to and from microscaled 4-bit codes (the format: mx4.h).
//
// Both are bound by the wide side's bytes. A lane has eight consecutive elements,
// 16 bytes of bf16 or 32 of float32, and one word of codes, so that a wave reads or
// writes 1 KB (2 KB) and 256 bytes in a row; the four lanes of a block of 32 share its
// largest magnitude through two exchanges.
#include <algorithm>

#include "mx4.h"

namespace ms {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ void load8(const T* p, float v[8]) {
    if constexpr (sizeof(T) == 2) {
        const vec16 r = ld16(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    } else {
        load4<float>(p, v);
        load4<float>(p + 4, v + 4);
    }
}

// Pieces of eight elements, `per_row` to a row. grid.x covers a row's pieces, grid.y the rows in turn.
template <typename T>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(const T* __restrict__ x, long rows, int per_row, long ld,
                                                                uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const long n = rows * per_row;
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long)gridDim.x * kThreads) {
        const long r = i / per_row;
        const int c = (int)(i - r * per_row);
        float v[8];
        load8<T>(x + r * ld + c * 8, v);
        uint32_t u = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) u = max(u, __float_as_uint(v[k]) & 0x7fffffffu);
        // rows hold whole blocks, so the four lanes of a block are all here
        u = max(u, (uint32_t)__shfl_xor((int)u, 1, kWave));
        u = max(u, (uint32_t)__shfl_xor((int)u, 2, kWave));
        const bool finite = u < 0x7f800000u;    // an infinity or NaN anywhere: the block is NaN, its codes zeros
        const uint32_t b = finite ? mx4_exponent(u) : 255u;
        const uint32_t w = finite ? mx4_encode8(v, mx4_ratio(b)) : 0u;
        codes[i] = w;
        if (c % 4 == 0) scales[i / 4] = (uint8_t)b;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                  long rows, int per_row, T* __restrict__ x, long ld) {
    const long n = rows * per_row;
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long)gridDim.x * kThreads) {
        const long r = i / per_row;
        const int c = (int)(i - r * per_row);
        const uint32_t w = codes[i];
        const float s = mx4_scale(scales[i / 4]);
        T* const p = x + r * ld + c * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const auto f = k == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0)
                         : k == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1)
                         : k == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2)
                                  : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
            v[2 * k] = f[0] * s;        // exact: a power of two; below 2^-126 a subnormal of both types
            v[2 * k + 1] = f[1] * s;
        }
        if constexpr (sizeof(T) == 2) {
            vec16 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o.w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
            st16(p, o);
        } else {
            store4<float>(p, v);
            store4<float>(p + 4, v + 4);
        }
    }
}

unsigned blocks_for(long pieces) { return (unsigned)std::min<long>((pieces + kThreads - 1) / kThreads, 1 << 20); }

}  // namespace

hipError_t launch_mx4_quantize(int dtype, const void* x, long rows, int cols, long ld, uint8_t* codes, uint8_t* scales,
                               hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int per = cols / 8;
    const dim3 grid(blocks_for(rows * per)), block(kThreads);
    uint32_t* const c = reinterpret_cast<uint32_t*>(codes);
    if (dtype == kBF16)
        hipLaunchKernelGGL(mx4_quantize_kernel<bf16_t>, grid, block, 0, s, static_cast<const bf16_t*>(x), rows, per, ld, c, scales);
    else
        hipLaunchKernelGGL(mx4_quantize_kernel<float>, grid, block, 0, s, static_cast<const float*>(x), rows, per, ld, c, scales);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, long rows, int cols, void* x,
                                 long ld, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int per = cols / 8;
    const dim3 grid(blocks_for(rows * per)), block(kThreads);
    const uint32_t* const c = reinterpret_cast<const uint32_t*>(codes);
    if (dtype == kBF16)
        hipLaunchKernelGGL(mx4_dequantize_kernel<bf16_t>, grid, block, 0, s, c, scales, rows, per, static_cast<bf16_t*>(x), ld);
    else
        hipLaunchKernelGGL(mx4_dequantize_kernel<float>, grid, block, 0, s, c, scales, rows, per, static_cast<float*>(x), ld);
    return hipGetLastError();
}

}  // namespace ms
