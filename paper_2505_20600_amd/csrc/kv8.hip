// Writing and reading an 8-bit K/V cache, and the lists of unmasked tokens.
#include <algorithm>

#include "kernels.h"
#include "kv8.h"

namespace ms {
namespace {

constexpr int kThreads = 256;

// 16 bytes of a K/V row, and the codes of as many values.
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    __device__ __forceinline__ static float at(const vec16& v, int i) {
        const uint32_t w = v.w[i >> 1];
        return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
    }
    // largest magnitude, as the bits of a float32 (infinities and NaN above every finite one)
    __device__ __forceinline__ static uint32_t most(const vec16& v) {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        auto mag = [&](int i) { return __builtin_bit_cast(u16x2, v.w[i] & 0x7fff7fffu); };
        const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(0), mag(1)),
                                                  __builtin_elementwise_max(mag(2), mag(3)));
        return (uint32_t)max(m[0], m[1]) << 16;
    }
    // codes of finite values at a power-of-two scale that holds them, round to nearest even
    __device__ __forceinline__ static void encode(const vec16& v, float scale, uint32_t (&c)[2]) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef short s16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s16x2 o = {0, 0};
            o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(bf16x2, v.w[2 * k]), scale, false);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(bf16x2, v.w[2 * k + 1]), scale, true);
            c[k] = __builtin_bit_cast(uint32_t, o);
        }
    }
    // the values that codes stand for; a bf16 value beyond the type's range is infinite
    __device__ __forceinline__ static vec16 decode(const uint32_t (&c)[2], float s) {
        return vec16{{kv8_to_bf16x2<false>(c[0], s), kv8_to_bf16x2<true>(c[0], s), kv8_to_bf16x2<false>(c[1], s),
                      kv8_to_bf16x2<true>(c[1], s)}};
    }
};
template <> struct Piece<float> {
    static constexpr int N = 4;
    __device__ __forceinline__ static float at(const vec16& v, int i) { return __uint_as_float(v.w[i]); }
    __device__ __forceinline__ static uint32_t most(const vec16& v) {
        const uint32_t m = 0x7fffffffu;
        return max(max(v.w[0] & m, v.w[1] & m), max(v.w[2] & m, v.w[3] & m));
    }
    __device__ __forceinline__ static void encode(const vec16& v, float scale, uint32_t (&c)[1]) {
        typedef short s16x2 __attribute__((ext_vector_type(2)));
        s16x2 o = {0, 0};
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, at(v, 0), at(v, 1), scale, false);
        o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, at(v, 2), at(v, 3), scale, true);
        c[0] = __builtin_bit_cast(uint32_t, o);
    }
    __device__ __forceinline__ static vec16 decode(const uint32_t (&c)[1], float s) {
        const float2 x = kv8_to_f32x2<false>(c[0], s), y = kv8_to_f32x2<true>(c[0], s);
        return vec16{{__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(y.x), __float_as_uint(y.y)}};
    }
};

// Past the caches: what is read or written once.
__device__ __forceinline__ vec16 load_stream(const void* p) {
    return __builtin_bit_cast(vec16, __builtin_nontemporal_load(static_cast<const u32x4_t*>(p)));
}
__device__ __forceinline__ void store_stream(void* p, const vec16& v) {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), static_cast<u32x4_t*>(p));
}
template <bool STREAM, int N>
__device__ __forceinline__ void store_codes(uint32_t* p, const uint32_t (&w)[N]) {
    typedef uint32_t u32xn_t __attribute__((ext_vector_type(N)));
    u32xn_t v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = w[i];
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32xn_t*>(p));
    else *reinterpret_cast<u32xn_t*>(p) = v;
}

// A workgroup takes NV rows per wave of a cache (a block of tokens or, of small blocks,
// several), K or V, and as many heads as 64 lanes of 16 bytes cover: lane = column, the waves
// take the rows in turn, so that a load is a contiguous kilobyte of a row and each value is read
// once, kept in registers until the exponent byte that its block needs is known (LDS, one
// maximum per block and head). Bound by memory. Over buffers that no cache holds, where a copy
// takes 5.65 TB/s: 8 caches of 4096 tokens of 16 heads of 72 (227 MB) 58 us, 3.9 TB/s (its groups of
// heads share lines of codes), 4 of 24 heads of 128 (302 MB) 51 us, 5.9 TB/s, 8 of 16 heads of 64 in
// float32 (335 MB) 55 us, 6.1 TB/s; the first over the same buffers again and again 44 us. A wave per
// (block, head) tile, lanes over its 144-byte rows and the values unpacked to float32, took 58 us
// there; loads through the caches 50. Codes go past the caches where a group's row of them is whole
// 64-byte lines (at head_dim 128 55 -> 51 us; at 72, where neighbouring groups share lines, 44 -> 49).
// Rewriting: kept rows need what their codes' largest magnitude needs at the old scale, and are
// encoded by the ratio of the two scales. Two loads one after the other (which row, then the row),
// three barriers and the stores, on the workgroups with a new row: one cache of 4096 tokens of 16
// heads of 72 a tenth of them in four runs 9.0 us, half 8.4, all 10.1, in float32 of 64 columns 6.2, 8.3,
// 8.9; a fifth of the tokens of 8 such caches in runs 19, scattered over every block 52 (166 MB).
// Except for blocks of 64 the rewriting forms ask for eight waves per SIMD: the compiler then
// keeps its scalar registers few enough for them (blocks of 128, that scattered fifth 72 -> 57 us, one
// cache's tenth 10.7 -> 11.0; blocks of 32 58 -> 52). Blocks of 64 run as well without (52 and 51 us,
// the tenth 9.0 and 9.3).
template <typename T, int NV, int WAVES, bool REWRITE, bool STREAM>
__global__ __launch_bounds__(WAVES * kWave, REWRITE && WAVES * NV != 64 ? 8 : 1) void quantize_kernel(
    Kv8Cache c, const T* __restrict__ kv, long row_stride, const int32_t* __restrict__ src_row, long kv_rows,
    int heads_per_group, int groups, int row_groups) {
    constexpr int CW = Piece<T>::N, R = WAVES * NV, kGroup = WAVES * kWave;
    __shared__ uint32_t s_need[R][kWave];   // [block of the rows][head of the group]: exponent byte, kNotFinite beside NaN and infinities
    constexpr uint32_t kNotFinite = 256;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    unsigned at = blockIdx.x;
    const int group = at % groups;
    at /= groups;
    const int which = at % 2;
    at /= 2;
    const int t0 = (int)(at % row_groups) * R, cache = at / row_groups;
    const int C = c.hd / CW, dkv = c.heads * c.hd;
    const int head0 = group * heads_per_group, heads = min(heads_per_group, c.heads - head0);
    const int h = lane / C;                 // head of the group
    const bool mine = lane < heads * C;
    const int col = which * dkv + head0 * c.hd + lane * CW;
    const int rows = min(R, c.T - t0);
    uint8_t* const codes = c.codes + ((long)cache * c.T + t0) * 2 * dkv + col;
    uint8_t* const scales = c.scales + ((long)cache * c.blocks + (t0 >> c.lblock)) * 2 * c.heads + which * c.heads + head0 + h;

    // which rows are new, one lane a row, and which are in a block with a new one
    uint64_t fresh[(R + kWave - 1) / kWave], touched[(R + kWave - 1) / kWave];
    if constexpr (REWRITE) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < (R + kWave - 1) / kWave; ++j) {
            const int r = j * kWave + lane;
            const int v = r < rows ? src_row[(long)cache * c.T + t0 + r] : -1;
            fresh[j] = __ballot(v >= 0 && v < kv_rows);
            any |= fresh[j] != 0;
        }
        if (!any) return;
        const int block = 1 << c.lblock;
#pragma unroll
        for (int j = 0; j < (R + kWave - 1) / kWave; ++j) {
            const int r = (j * kWave + lane) >> c.lblock << c.lblock;   // this row's block begins here
            uint64_t m = fresh[r / kWave] >> (r % kWave);
            if (block < kWave) m &= (1ull << block) - 1;
            else if (block > kWave) m = fresh[0] | fresh[(R + kWave - 1) / kWave - 1];
            touched[j] = __ballot(m != 0 && j * kWave + lane < rows);
        }
    }
    for (int i = threadIdx.x; i < (R >> c.lblock ? R >> c.lblock : 1) * kWave; i += kGroup) (&s_need[0][0])[i] = 0u;

    // REWRITE: a kept row holds its codes' values unscaled, `from` their scale's exponent byte (127
    // for new rows, whose values stand for themselves): scaled values reach from 2^-136 to 448 times
    // 2^127, beyond both ends of bf16 and float32
    vec16 v[NV];
    int from[REWRITE ? NV : 1];
    auto row_of = [&](int i) { return i * WAVES + wave; };
    auto bit = [&](const uint64_t* m, int r) { return (m[R > kWave ? r / kWave : 0] >> (r % kWave)) & 1; };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int r = row_of(i);
        v[i] = vec16{{0u, 0u, 0u, 0u}};
        if constexpr (REWRITE) {
            from[i] = 127;
            if (!mine || !bit(touched, r)) continue;
            if (bit(fresh, r)) {
                v[i] = ld16(kv + (long)src_row[(long)cache * c.T + t0 + r] * 2 * dkv + col);
            } else {
#pragma unroll
                for (int k = 0; k < CW / 4; ++k) v[i].w[k] = reinterpret_cast<const uint32_t*>(codes + (long)r * 2 * dkv)[k];
                from[i] = scales[(long)(r >> c.lblock) * 2 * c.heads];
            }
        } else if (mine && r < rows) {
            v[i] = load_stream(kv + ((long)cache * row_stride + t0 + r) * 2 * dkv + col);
        }
    }
    if constexpr (REWRITE) {    // the kept rows' codes, when all loads are under way
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int r = row_of(i);
            if (bit(fresh, r) || !bit(touched, r)) continue;
            uint32_t w[CW / 4];
#pragma unroll
            for (int k = 0; k < CW / 4; ++k) w[k] = v[i].w[k];
            v[i] = Piece<T>::decode(w, 1.0f);
            const bool nan = from[i] == 255;    // a scale of NaN
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i].w[k] = nan ? 0xffffffffu : v[i].w[k];
            from[i] = nan ? 127 : from[i];
        }
    }
    // this lane's largest need per block to s_need, from the bits of each row's largest magnitude
    auto scale_from = [&](int i) { return REWRITE ? from[REWRITE ? i : 0] : 127; };
    auto needs = [&](auto of_row) {
        auto need = [&](uint32_t u, int b) { return u >= 0x7f800000u ? kNotFinite : kv8_need(u, b); };
        uint32_t most = 0, kept = 0;    // of a block's new and kept rows; the latter have one scale
        int kept_from = 127;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int r = row_of(i);
            const uint32_t u = of_row(i);
            if (!REWRITE || bit(fresh, r)) {
                most = max(most, u);
            } else if (bit(touched, r)) {
                kept = max(kept, u);
                kept_from = scale_from(i);
            }
            if (i + 1 == NV || row_of(i + 1) >> c.lblock != r >> c.lblock) {
                uint32_t n = need(most, 127);
                if constexpr (REWRITE) n = max(n, need(kept, kept_from));
                if (mine) atomicMax(&s_need[r >> c.lblock][h], n);
                most = kept = 0;
            }
        }
    };
    __syncthreads();
    needs([&](int i) { return Piece<T>::most(v[i]); });
    __syncthreads();
    bool odd = false;       // infinities or NaN somewhere
    for (int i = threadIdx.x; i < (R >> c.lblock ? R >> c.lblock : 1) * kWave; i += kGroup) odd |= (&s_need[0][0])[i] == kNotFinite;
    odd = __syncthreads_or(odd);
    if (odd) {              // the scale is that of the finite values
        for (int i = threadIdx.x; i < (R >> c.lblock ? R >> c.lblock : 1) * kWave; i += kGroup) (&s_need[0][0])[i] = 0u;
        __syncthreads();
        needs([&](int i) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < CW; ++e) {
                const float x = Piece<T>::at(v[i], e);
                m = max(m, kv8_finite(x) ? __float_as_uint(fabsf(x)) : 0u);
            }
            return m;
        });
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int r = row_of(i);
        if (!mine || (REWRITE ? !bit(touched, r) : r >= rows)) continue;
        const uint32_t b = kv8_block_exponent(s_need[r >> c.lblock][h]);
        uint32_t* const p = reinterpret_cast<uint32_t*>(codes + (long)r * 2 * dkv);
        uint32_t w[CW / 4];
        if (odd || REWRITE) {
            const float ratio = kv8_ratio(scale_from(i), b);
#pragma unroll
            for (int k = 0; k < CW / 4; ++k) {
                const float x[4] = {Piece<T>::at(v[i], 4 * k), Piece<T>::at(v[i], 4 * k + 1), Piece<T>::at(v[i], 4 * k + 2),
                                    Piece<T>::at(v[i], 4 * k + 3)};
                w[k] = kv8_encode4(x, ratio);
            }
        } else {
            Piece<T>::encode(v[i], kv8_scale(b), w);
        }
        store_codes<STREAM>(p, w);
        // the first row of a block, the first lane of a head
        if ((r & ((1 << c.lblock) - 1)) == 0 && lane % C == 0) scales[(long)(r >> c.lblock) * 2 * c.heads] = (uint8_t)b;
    }
}

// Values of the listed tokens: a workgroup takes `rows` of a request's list, its threads 16
// bytes of output each (two such stores of every other 16 bytes were 10% slower), four at a
// time so that their loads are in flight together. Bound by memory: 4 x ~3100 listed tokens of
// 24 heads of 128 (233 MB) 36 us, 6.4 TB/s, over the same buffers again and again; with stores
// through the caches 57. Over buffers that no cache holds 43 (a copy of as much 41), in float32 of 64
// columns (189 MB) 37.
template <typename T>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(Kv8Cache c, Kv8Select sel, T* __restrict__ kv,
                                                              long row_stride, int rows) {
    constexpr int N = 4, CW = Piece<T>::N;
    const int b = blockIdx.y, first = blockIdx.x * rows;
    const Kv8Req r = kv8_request(c, sel, b);
    const unsigned dkv = c.heads * c.hd, per_row = 2 * dkv / CW;
    const unsigned n = (unsigned)min(rows, max(r.nk - first, 0)) * per_row;
    for (unsigned i0 = threadIdx.x; i0 < n; i0 += N * kThreads) {
        int t[N];
        unsigned col[N];
        uint32_t code[N][CW / 4];
        float s[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const unsigned i = i0 + j * kThreads, at = i / per_row;
            col[j] = (i - at * per_row) * CW;
            t[j] = -1;
            if (i < n) t[j] = r.keys ? r.keys[first + at] : first + (int)at;
            if (t[j] >= c.T) t[j] = -1;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int tj = max(t[j], 0);
            const uint32_t* const p = reinterpret_cast<const uint32_t*>(r.codes + (long)tj * 2 * dkv + col[j]);
#pragma unroll
            for (int k = 0; k < CW / 4; ++k) code[j][k] = p[k];
            // K heads, then V heads
            s[j] = kv8_scale(r.scales[(long)(tj >> c.lblock) * 2 * c.heads + col[j] / c.hd]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (t[j] < 0) continue;
            store_stream(kv + ((long)b * row_stride + t[j]) * 2 * dkv + col[j], Piece<T>::decode(code[j], s[j]));
        }
    }
}

// Ascending numbers of a request's tokens whose mask byte is zero: one workgroup
// per request, kScanThreads tokens at a time, their places from a prefix sum. A pass takes 0.6
// us (a load, two barriers): 4096 tokens 4.1 us, 128 requests of them 4.6, 2^17 tokens 80 us, 2^20 630.
constexpr int kScanThreads = 1024;
__global__ __launch_bounds__(kScanThreads) void keys_kernel(const uint8_t* __restrict__ mask, int T,
                                                            int32_t* __restrict__ keys, int ld_keys,
                                                            int32_t* __restrict__ n_keys) {
    __shared__ int s_wave[kScanThreads / kWave];
    const int b = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int base = 0;
    for (int t0 = 0; t0 < T; t0 += kScanThreads) {
        const int t = t0 + threadIdx.x;
        const bool take = t < T && mask[(long)b * T + t] == 0;
        const uint64_t m = __ballot(take);
        if (lane == 0) s_wave[wave] = __popcll(m);
        __syncthreads();
        int before = base, total = 0;
#pragma unroll
        for (int w = 0; w < kScanThreads / kWave; ++w) {
            const int v = s_wave[w];
            before += w < wave ? v : 0;
            total += v;
        }
        if (take) keys[(long)b * ld_keys + before + __popcll(m & ((1ull << lane) - 1))] = t;
        base += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) n_keys[b] = base;
}

// Both lists of a request from its inverse map; see launch_kv8_step_lists.
__global__ __launch_bounds__(kScanThreads) void step_lists_kernel(const int32_t* __restrict__ inv, int N, int n_text,
                                                                  int32_t* __restrict__ keys, int32_t* __restrict__ n_keys,
                                                                  int32_t* __restrict__ fresh, int32_t* __restrict__ start,
                                                                  int32_t* __restrict__ end) {
    __shared__ int s_cached[kScanThreads / kWave], s_fresh[kScanThreads / kWave];
    const int b = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, T = n_text + N;
    const long row0 = (long)b * T;
    int cached = 0, news = 0;
    for (int t0 = 0; t0 < T; t0 += kScanThreads) {
        const int t = t0 + threadIdx.x;
        const bool in = t < T, recomputed = in && inv[row0 + t] >= 0, keep = in && !recomputed && t >= n_text;
        const uint64_t mc = __ballot(keep), mf = __ballot(recomputed), below = (1ull << lane) - 1;
        if (lane == 0) {
            s_cached[wave] = __popcll(mc);
            s_fresh[wave] = __popcll(mf);
        }
        __syncthreads();
        int c = cached, f = news;
#pragma unroll
        for (int w = 0; w < kScanThreads / kWave; ++w) {
            if (w < wave) {
                c += s_cached[w];
                f += s_fresh[w];
            }
            cached += s_cached[w];
            news += s_fresh[w];
        }
        if (keep) keys[(long)b * N + c + __popcll(mc & below)] = t - n_text;
        if (recomputed) fresh[row0 + f + __popcll(mf & below)] = (int)(row0 + t);
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        n_keys[b] = cached;
        start[b] = (int)row0;
        end[b] = (int)row0 + news;
    }
}

// How a cache is divided among workgroups.
struct QuantizeGrid {
    int groups, per_group;      // groups of heads, even ones of at most 64 lanes
    int rows, row_groups;
    long workgroups;
};
QuantizeGrid quantize_grid(int dtype, const Kv8Cache& c) {
    QuantizeGrid g;
    const int most = kWave / (c.hd / (dtype == kBF16 ? Piece<bf16_t>::N : Piece<float>::N));
    g.groups = (c.heads + most - 1) / most;
    g.per_group = (c.heads + g.groups - 1) / g.groups;
    g.rows = std::max(1 << c.lblock, 16);
    g.row_groups = (c.T + g.rows - 1) / g.rows;
    g.workgroups = (long)c.n_caches * g.row_groups * 2 * g.groups;
    return g;
}

template <typename T, bool REWRITE, bool STREAM>
void launch_quantize(const Kv8Cache& c, const QuantizeGrid& g, const void* kv, long row_stride, const int32_t* src_row,
                     long kv_rows, hipStream_t s) {
    const dim3 grid((unsigned)g.workgroups);
    const T* p = static_cast<const T*>(kv);
#define MS_ROWS(r, nv, waves)                                                                                          \
    case r: hipLaunchKernelGGL((quantize_kernel<T, (nv), (waves), REWRITE, STREAM>), grid, dim3((waves) * kWave), 0, s, c, p, row_stride, \
                               src_row, kv_rows, g.per_group, g.groups, g.row_groups); break;
    switch (g.rows) {
        MS_ROWS(16, 4, 4) MS_ROWS(32, 4, 8) MS_ROWS(64, 8, 8) MS_ROWS(128, 8, 16)
    }
#undef MS_ROWS
}

template <typename T>
void launch_quantize(const Kv8Cache& c, const QuantizeGrid& g, const void* kv, long row_stride, const int32_t* src_row,
                     long kv_rows, hipStream_t s) {
    if (src_row) launch_quantize<T, true, false>(c, g, kv, row_stride, src_row, kv_rows, s);
    else if (g.per_group * c.hd % 64 == 0) launch_quantize<T, false, true>(c, g, kv, row_stride, src_row, kv_rows, s);
    else launch_quantize<T, false, false>(c, g, kv, row_stride, src_row, kv_rows, s);
}

}  // namespace

hipError_t launch_kv8_keys(const uint8_t* mask, int batch, int T, int32_t* keys, int ld_keys, int32_t* n_keys,
                           hipStream_t s) {
    hipLaunchKernelGGL(keys_kernel, dim3(batch), dim3(kScanThreads), 0, s, mask, T, keys, ld_keys, n_keys);
    return hipGetLastError();
}

hipError_t launch_kv8_step_lists(const int32_t* inv, int batch, int N, int n_text, int32_t* keys, int32_t* n_keys,
                                 int32_t* fresh, int32_t* start, int32_t* end, hipStream_t s) {
    hipLaunchKernelGGL(step_lists_kernel, dim3(batch), dim3(kScanThreads), 0, s, inv, N, n_text, keys, n_keys, fresh, start, end);
    return hipGetLastError();
}

// 16 threads or fewer per row of a workgroup: fewer than the 2^32 threads that end a launch.
bool kv8_quantize_fits(int dtype, const Kv8Cache& c) {
    const QuantizeGrid g = quantize_grid(dtype, c);
    return g.workgroups * g.rows < 1l << 28;
}

hipError_t launch_kv8_quantize(int dtype, const Kv8Cache& c, const void* kv, long row_stride, const int32_t* src_row,
                               long kv_rows, hipStream_t s) {
    const QuantizeGrid g = quantize_grid(dtype, c);
    if (dtype == kBF16) launch_quantize<bf16_t>(c, g, kv, row_stride, src_row, kv_rows, s);
    else launch_quantize<float>(c, g, kv, row_stride, src_row, kv_rows, s);
    return hipGetLastError();
}

hipError_t launch_kv8_dequantize(int dtype, const Kv8Cache& c, const Kv8Select& sel, void* kv, long row_stride,
                                 hipStream_t s) {
    if (sel.ld_keys == 0) return hipSuccess;
    const int rows = std::max(1, (int)(4 * kThreads * 16 / (2 * c.heads * c.hd * (dtype == kBF16 ? 2 : 4))));   // about one pass
    const dim3 grid((sel.ld_keys + rows - 1) / rows, sel.batch), block(kThreads);
    if (dtype == kBF16)
        hipLaunchKernelGGL(dequantize_kernel<bf16_t>, grid, block, 0, s, c, sel, static_cast<bf16_t*>(kv), row_stride, rows);
    else
        hipLaunchKernelGGL(dequantize_kernel<float>, grid, block, 0, s, c, sel, static_cast<float*>(kv), row_stride, rows);
    return hipGetLastError();
}

}  // namespace ms
