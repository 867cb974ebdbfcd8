// What the bf16 attention kernels share: the matrix instruction, the layout of
// K and V tiles in LDS, the transpose read of V, the softmax's constants.
#pragma once

#include "common.h"

namespace ms {

__device__ __forceinline__ f32x4_t mfma32(bf16x8_t a, bf16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

constexpr float kRescaleLog2 = 8.0f;   // softmax weights may reach 2^8 before a rescale
// Score accumulators start at minus the running maximum, but not beyond this: a score
// far above the maximum so far would be rounded to the digits of the latter (a first
// key tile near the type's lowest value left the others' scores none). 2^14 leaves them
// 2^-10, below the rounding of the weights, and a tile's ordinary path as it was.
constexpr float kStartMax = 16384.0f;

// 16-byte chunk swizzles of a V and of a K row (XOR of the chunk index; see
// the kernel comment).
template <int ROWB>
__device__ __forceinline__ int v_swz(int r) {
    if constexpr (ROWB == 128) return 2 * ((r >> 1) & 3) + ((r >> 3) & 1);
    else if constexpr (ROWB == 256) return 2 * (r & 7) + ((r >> 3) & 1);
    else return 0;
}
template <int ROWB>
__device__ __forceinline__ int k_swz(int r) {
    if constexpr (ROWB == 256) return r & 15;
    else if constexpr (ROWB == 128) return (r >> 1) & 7;
    else if constexpr (ROWB % 128 == 64) return (r >> 1) & 3;
    else return 0;
}

typedef const __attribute__((address_space(3))) uint8_t* lds_cptr;

__device__ __forceinline__ bf16x4_t ld_tr16(lds_cptr p) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(p));
    return __builtin_bit_cast(bf16x4_t, v);
}

}  // namespace ms
