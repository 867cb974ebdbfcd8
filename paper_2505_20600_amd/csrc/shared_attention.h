// Attention of a batch over one shared prefix: descriptor and launchers
// (shared_attention.hip, block_ops_api.hip).
#pragma once

#include "common.h"

namespace ms {

constexpr int kSharedMaxBatch = 128;

struct SharedAttnDesc {
    const void* q;              // [M][heads * group * hd]
    void* o;                    // the same
    const void* kv;             // prefix [T][2][heads * hd]
    const uint64_t* bits;       // [batch][words] hidden prefix tokens, 64 to a word; NULL: none
    const int32_t* seg_start;   // [batch + 1] packed rows of each request, NULL: one request, every row
    const void* fresh;          // own rows [fresh_rows][2][heads * hd], NULL: none
    const int32_t* fresh_start; // [batch + 1] own rows of each request
    int fresh_rows, batch, T, words, M, heads, group, hd;
    float scale_log2;           // log2(e) times the score scale
    int tile;                   // query slots per workgroup: 16 or 32, or in bf16 128
    int nsplit;                 // key ranges; > 1: partials in part_o / part_ml
    float* part_o;              // [nsplit][M][heads * group * hd], each range's output over its own sum
    float* part_ml;             // [nsplit][M][heads * group][2]: its maximum (log2 domain) and sum
};

// Hidden tokens as bits: bit t % 64 of bits[b][t / 64] is set where mask[b][t] is not 0, and past the last token.
hipError_t launch_shared_bits(const uint8_t* mask, int batch, int T, uint64_t* bits, hipStream_t s);
// Sets the form and the key ranges from the sizes. The caller may lower nsplit to what its buffers hold.
void plan_shared_attention(int dtype, SharedAttnDesc& a);
hipError_t launch_shared_attention(int dtype, const SharedAttnDesc& a, hipStream_t s);
// Joins the key ranges' parts into the output; nothing where there is one range.
hipError_t launch_shared_join(int dtype, const SharedAttnDesc& a, hipStream_t s);

}  // namespace ms
