// Descriptor and launcher of the per-head norms, rotation and K/V scatter (qk_norm_rope.hip).
#pragma once

#include "common.h"

namespace ms {

struct QkNormRopeDesc {
    const void* qkv;            // [M] rows of (H + 2 G) heads, ld elements apart
    void* q;                    // [M][H][hd]
    void* kv;                   // [kv_rows][2][G][hd]
    const void *q_gain, *k_gain;// [hd], NULL: not normalised
    const float* table;         // [n_pos][rot / 2][2] cos, sin; NULL: not rotated
    const int32_t* pos;         // [M] table rows, NULL: m; outside 0..n_pos - 1: not rotated
    const int32_t* rows;        // [M] rows of kv, NULL: m; outside 0..kv_rows - 1: K and V are not written
    long ld, kv_rows;
    int M, H, G, hd, rot, n_pos;
    bool halves;                // pairs (i, i + rot / 2) instead of (2 i, 2 i + 1)
    float eps;
    int parts;                  // set by launch_qk_norm_rope: waves that share a row's heads
};

hipError_t launch_qk_norm_rope(int dtype, const QkNormRopeDesc& d, hipStream_t s);

}  // namespace ms
