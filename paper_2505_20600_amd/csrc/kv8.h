// 8-bit K/V cache: the format's arithmetic and the launchers' descriptors
// (kv8.hip, kv8_attention.hip, kv8_api.hip; the step in maskstep.hip).
//
// A cache holds e4m3 codes (no infinities, NaN 0x7f, largest 448) in
// [cache][token][K, V][head][head_dim] order and one exponent byte b per
// (cache, block of 2^lblock tokens, K or V, head): value = code * 2^(b - 127).
// The scale is a power of two, so a value is exact in bf16 and float32 (within
// their ranges) and v_cvt_scalef32 applies it in the conversion; e4m3 is a
// floating format, so a finer scale would only shift where its largest and
// smallest codes lie.
#pragma once

#include "common.h"

namespace ms {

constexpr int kKv8MaxSegments = 128;   // packed query segments per attention call

// One float with the exponent byte's value 2^(b - 127): b = 0 is the subnormal
// 2^-127, b = 255 NaN.
__device__ __forceinline__ float kv8_scale(uint32_t b) {
    return __uint_as_float(b == 0 ? 0x00400000u : b == 255 ? 0x7fc00000u : b << 23);
}

// Exponent byte that values of the magnitudes up to |x| 2^(from - 127) need (`u`: the bits of
// |x|, finite): the smallest power of two s >= 2^-126 with |x| 2^(from - 127) <= 448 s =
// 1.75 * 2^8 s; 0 for x = 0. A block takes the largest need among its values, and the scale 1
// (kv8_block_exponent) where all are zero.
__device__ __forceinline__ uint32_t kv8_need(uint32_t u, int from) {
    const int e = (int)((u + 0x1fffffu) >> 23) + from - 135;    // a mantissa above 0.75 carries into the exponent
    return u == 0 ? 0u : (uint32_t)max(e, 1);
}
__device__ __forceinline__ uint32_t kv8_block_exponent(uint32_t need) { return need == 0 ? 127u : need; }

__device__ __forceinline__ bool kv8_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Two codes (bytes 0-1 or 2-3 of w) -> two packed bf16 / two floats, scaled.
template <bool HI>
__device__ __forceinline__ uint32_t kv8_to_bf16x2(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HI));
}
template <bool HI>
__device__ __forceinline__ float2 kv8_to_f32x2(uint32_t w, float s) {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, HI);
    return make_float2(v[0], v[1]);
}

// What x 2^(from - 127) is multiplied by, as x, for codes at the exponent byte b >= its need: 2^(from - b),
// at least 2^-127 (below that every x of a code is far below half the smallest code, and so is its
// product) and at most 2^127 (a code other than 0 never takes more than 2^17). Exact where the product is
// a normal float32; what is not is below half the smallest code.
__device__ __forceinline__ float kv8_ratio(int from, uint32_t b) {
    const int e = min(from - (int)b + 127, 254);
    return __uint_as_float(e <= 0 ? 0x00400000u : (uint32_t)e << 23);
}

// Four values times ratio -> four codes, round to nearest even; at most 448 for finite x; NaN and
// infinities become NaN.
__device__ __forceinline__ uint32_t kv8_encode4(const float x[4], float ratio) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = kv8_finite(x[i]) ? x[i] * ratio : __uint_as_float(0x7fc00000u);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    return (uint32_t)w;
}

// Which cached tokens of which caches the requests of a batch read.
struct Kv8Select {
    const int32_t* codes_of;    // [batch] cache of each request's codes, NULL: request b has cache b
    const int32_t* scales_of;   // [batch] the same of its scales
    const int32_t* keys;        // [batch][ld_keys] token numbers, NULL: tokens 0, 1, ...
    const int32_t* n_keys;      // [batch] listed tokens, NULL: ld_keys (every token)
    int ld_keys;
    int batch;
};

struct Kv8Cache {
    uint8_t* codes;         // [n_caches][T][2][heads * hd]
    uint8_t* scales;        // [n_scales][blocks][2][heads]
    int n_caches, n_scales; // scale tables may be indexed apart from the codes
    int T, heads, hd, lblock, blocks;
};

struct Kv8AttnDesc {
    Kv8Cache c;
    Kv8Select sel;
    const void* q;              // [M][heads * group * hd]
    void* o;                    // the same
    const int32_t* seg_start;   // [nseg + 1] packed rows of each segment
    const int32_t* seg_req;     // [nseg] request of each segment, NULL: segment s is request s
    int nseg, M, group;
    const void* kv;             // fresh rows [kv_rows][2][heads * hd], NULL: none
    const int32_t* f_rows;      // rows of kv in list order, NULL: entry i is row i
    const int32_t* f_start;     // [batch] first list entry of each request
    const int32_t* f_end;       // [batch] and the one past its last
    long kv_rows;               // rows of kv
    int f_list;                 // entries of the list
    float scale_log2;           // log2(e) times the score scale
    int tile;                   // query slots per workgroup: 16, or in bf16 32 or 128
    int nsplit;                 // key ranges; > 1: partials in part_o / part_ml
    float* part_o;              // [nsplit][M][heads * group * hd], each range's output over its own sum
    float* part_ml;             // [nsplit][M][heads * group][2]: its maximum (log2 domain) and sum
};

// One request's keys: the listed cached tokens, then the fresh rows. Every
// index that comes from device memory is bounded here or where it is used.
struct Kv8Req {
    const uint8_t* codes;
    const uint8_t* scales;
    const int32_t* keys;
    int nk;         // cached tokens
    int f0, nf;     // fresh list entries [f0, f0 + nf)
};

// `codes`, `scales`: the request's cache numbers (0 where it has none).
__device__ __forceinline__ Kv8Req kv8_request(const Kv8Cache& c, const Kv8Select& sel, int b, int& codes, int& scales) {
    Kv8Req r{nullptr, nullptr, nullptr, 0, 0, 0};
    const int cc = sel.codes_of ? sel.codes_of[b] : b;
    const int sc = sel.scales_of ? sel.scales_of[b] : b;
    const int n = sel.n_keys ? min(max(sel.n_keys[b], 0), sel.ld_keys) : sel.ld_keys;
    const bool known = cc >= 0 && cc < c.n_caches && sc >= 0 && sc < c.n_scales;
    codes = known ? cc : 0;
    scales = known ? sc : 0;
    r.codes = c.codes + (long)codes * c.T * 2 * c.heads * c.hd;
    r.scales = c.scales + (long)scales * c.blocks * 2 * c.heads;
    r.keys = sel.keys ? sel.keys + (long)b * sel.ld_keys : nullptr;
    r.nk = known ? n : 0;
    return r;
}
__device__ __forceinline__ Kv8Req kv8_request(const Kv8Cache& c, const Kv8Select& sel, int b) {
    int cc, sc;
    return kv8_request(c, sel, b, cc, sc);
}

__device__ __forceinline__ void kv8_fresh(const Kv8AttnDesc& a, int b, Kv8Req& r) {
    if (!a.kv) return;
    r.f0 = min(max(a.f_start[b], 0), a.f_list);
    r.nf = min(max(a.f_end[b], r.f0), a.f_list) - r.f0;
}

// Unmasked tokens of every request in ascending order: keys[b][0 .. n_keys[b]).
hipError_t launch_kv8_keys(const uint8_t* mask, int batch, int T, int32_t* keys, int ld_keys, int32_t* n_keys,
                           hipStream_t s);
// The same for a step context from its inverse map inv [batch][n_text + N] (packed row of a
// token, < 0: not recomputed): the image tokens that are not recomputed, and the recomputed
// tokens' flat rows b * (n_text + N) + t, request b's list entries [start[b], end[b]).
hipError_t launch_kv8_step_lists(const int32_t* inv, int batch, int N, int n_text, int32_t* keys, int32_t* n_keys,
                                 int32_t* fresh, int32_t* start, int32_t* end, hipStream_t s);
// K/V rows [..][2][heads * hd] -> codes and scales. src_row NULL: token t of
// cache c is row c * row_stride + t; else row src_row[c][t] where that lies in
// [0, kv_rows), and the token keeps its value elsewhere.
// kv8_quantize_fits: whether one launch can have the whole.
bool kv8_quantize_fits(int dtype, const Kv8Cache& c);
hipError_t launch_kv8_quantize(int dtype, const Kv8Cache& c, const void* kv, long row_stride, const int32_t* src_row,
                               long kv_rows, hipStream_t s);
// kv[b * row_stride + t] = the listed tokens' values.
hipError_t launch_kv8_dequantize(int dtype, const Kv8Cache& c, const Kv8Select& sel, void* kv, long row_stride,
                                 hipStream_t s);
// Sets the form and the key ranges for a call over about `keys` keys per request (from its
// sizes; its tables are not read). The caller may lower nsplit to what its buffers hold.
void plan_kv8_attention(int dtype, Kv8AttnDesc& a, long keys);
hipError_t launch_kv8_attention(int dtype, const Kv8AttnDesc& a, hipStream_t s);
// Joins the key ranges' parts into the output; nothing where there is one range.
hipError_t launch_kv8_join(int dtype, const Kv8AttnDesc& a, hipStream_t s);

}  // namespace ms
