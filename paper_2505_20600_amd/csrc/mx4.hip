// Rows to and from microscaled 4-bit codes (the format: mx4.h).
//
// Both are bound by the wide side's bytes. A lane has eight consecutive elements,
// 16 bytes of bf16 or 32 of float32, and one word of codes, so that a wave reads or
// writes 1 KB (2 KB) and 256 bytes in a row; the four lanes of a block of 32 share its
// largest magnitude through two exchanges. At 16384 rows of 4096, bf16: codes in 27 us and read back in 26 us where
// the last-level cache holds the rows (6.3 and 6.5 TB/s, a copy there 7.0), 32 and 34 us over buffers that no cache holds (5.3 and
// 5.0, a copy 5.3); float32 there 53 us (5.8) and 62 us (4.9).
#include <algorithm>

#include "mx4.h"

namespace ms {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ void unpack8(const vec16 (&r)[sizeof(T) / 2], float v[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            v[2 * i] = __uint_as_float(r[0].w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[0].w[i] & 0xffff0000u);
        } else {
            v[i] = __uint_as_float(r[0].w[i]);
            v[4 + i] = __uint_as_float(r[1].w[i]);
        }
    }
}

// Element index of piece i of `per_row` to a row; rows without gaps need no division.
__device__ __forceinline__ long place(long i, int per_row, long ld) {
    if (ld == (long)per_row * 8) return i * 8;
    const long r = i / per_row;
    return r * ld + (i - r * per_row) * 8;
}

// Pieces of eight elements, U to a lane at a time, their loads ahead of all else.
template <typename T, int U>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(const T* __restrict__ x, long n, int per_row, long ld,
                                                                uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    for (long i0 = (long)blockIdx.x * U * kThreads + threadIdx.x; i0 < n; i0 += (long)gridDim.x * U * kThreads) {
        vec16 raw[U][sizeof(T) / 2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const T* const p = x + place(min(i0 + u * kThreads, n - 1), per_row, ld);
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h) raw[u][h] = ld16(p + h * 16 / (int)sizeof(T));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long i = i0 + u * kThreads;
            if (i >= n) break;
            float v[8];
            unpack8<T>(raw[u], v);
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
            // rows hold whole blocks, so the four lanes of a block are all here
            m = max(m, (uint32_t)__shfl_xor((int)m, 1, kWave));
            m = max(m, (uint32_t)__shfl_xor((int)m, 2, kWave));
            const bool finite = m < 0x7f800000u;    // an infinity or NaN anywhere: the block is NaN, its codes zeros
            const uint32_t b = finite ? mx4_exponent(m) : 255u;
            codes[i] = finite ? mx4_encode8(v, mx4_ratio(b)) : 0u;
            if (i % 4 == 0) scales[i / 4] = (uint8_t)b;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                  long n, int per_row, T* __restrict__ x, long ld) {
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long)gridDim.x * kThreads) {
        const uint32_t w = codes[i];
        const float s = mx4_scale(scales[i / 4]);
        T* const p = x + place(i, per_row, ld);
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

// Workgroups for n pieces, u to a lane at a time.
unsigned blocks_for(long n, int u) { return (unsigned)std::min<long>((n + u * kThreads - 1) / (u * kThreads), 1 << 20); }

template <typename T, int U>
void quantize(const void* x, long n, int per, long ld, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    hipLaunchKernelGGL((mx4_quantize_kernel<T, U>), dim3(blocks_for(n, U)), dim3(kThreads), 0, s, static_cast<const T*>(x), n, per, ld,
                       reinterpret_cast<uint32_t*>(codes), scales);
}

}  // namespace

hipError_t launch_mx4_quantize(int dtype, const void* x, long rows, int cols, long ld, uint8_t* codes, uint8_t* scales,
                               hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int per = cols / 8;
    const long n = rows * per;
    // bf16 pieces are one load: four at once where there are enough to fill the CUs with them. 16384 rows of 4096, in the cache,
    // take 26 us instead of 30, 2048 rows of 1152 would take 3.9 instead of 3.6; in float32 four at once gain nothing (48 us both ways).
    if (dtype != kBF16) quantize<float, 1>(x, n, per, ld, codes, scales, s);
    else if (n < 1 << 20) quantize<bf16_t, 1>(x, n, per, ld, codes, scales, s);
    else quantize<bf16_t, 4>(x, n, per, ld, codes, scales, s);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, long rows, int cols, void* x,
                                 long ld, hipStream_t s) {
    if (rows == 0) return hipSuccess;
    const int per = cols / 8;
    const long n = rows * per;
    const dim3 grid(blocks_for(n, 1)), block(kThreads);
    const uint32_t* const c = reinterpret_cast<const uint32_t*>(codes);
    if (dtype == kBF16)
        hipLaunchKernelGGL(mx4_dequantize_kernel<bf16_t>, grid, block, 0, s, c, scales, n, per, static_cast<bf16_t*>(x), ld);
    else
        hipLaunchKernelGGL(mx4_dequantize_kernel<float>, grid, block, 0, s, c, scales, n, per, static_cast<float*>(x), ld);
    return hipGetLastError();
}

}  // namespace ms
