// Writing and reading an 8-bit K/V cache, and the lists of unmasked tokens.
#include <algorithm>

#include "kernels.h"
#include "kv8.h"

namespace ms {
namespace {

constexpr int kThreads = 256;

// Eight consecutive elements of a K/V row.
template <typename T> struct Chunk8;
template <> struct Chunk8<bf16_t> {
    vec16 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = ld16(p); }
    __device__ __forceinline__ float at(int i) const {
        const uint32_t w = v.w[i >> 1];
        return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
    }
    // the bits of the values that codes stand for; a bf16 value beyond the type's range is infinite
    __device__ __forceinline__ void decode(uint2 c, float s) {
        v.w[0] = kv8_to_bf16x2<false>(c.x, s);
        v.w[1] = kv8_to_bf16x2<true>(c.x, s);
        v.w[2] = kv8_to_bf16x2<false>(c.y, s);
        v.w[3] = kv8_to_bf16x2<true>(c.y, s);
    }
    __device__ __forceinline__ void store(bf16_t* p) const { st16(p, v); }
};
template <> struct Chunk8<float> {
    float f[8];
    __device__ __forceinline__ void load(const float* p) {
        load4<float>(p, f);
        load4<float>(p + 4, f + 4);
    }
    __device__ __forceinline__ float at(int i) const { return f[i]; }
    __device__ __forceinline__ void decode(uint2 c, float s) {
        const float2 a = kv8_to_f32x2<false>(c.x, s), b = kv8_to_f32x2<true>(c.x, s);
        const float2 d = kv8_to_f32x2<false>(c.y, s), e = kv8_to_f32x2<true>(c.y, s);
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
        f[4] = d.x; f[5] = d.y; f[6] = e.x; f[7] = e.y;
    }
    __device__ __forceinline__ void store(float* p) const {
        store4<float>(p, f);
        store4<float>(p + 4, f + 4);
    }
};

// One tile = the rows of one block of tokens, K or V, one head: 2^lblock x
// head_dim values in chunks of eight. `lanes` lanes of a wave (a power of two)
// hold one tile in registers, NV chunks each, so the values are read once:
// largest magnitude over the tile, exponent byte, codes. Bound by memory.
template <typename T, int NV, bool REWRITE>
__global__ __launch_bounds__(kThreads) void quantize_kernel(Kv8Cache c, const T* __restrict__ kv, long row_stride,
                                                            const int32_t* __restrict__ src_row, long kv_rows,
                                                            int lanes, long tiles) {
    const int sub = threadIdx.x % lanes;
    const long tile = (long)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
    if (tile >= tiles) return;   // whole groups of lanes; the shuffles below stay within a group
    const int head = (int)(tile % c.heads);
    const int which = (int)(tile / c.heads % 2);
    const long sb = tile / (2 * c.heads);
    const int blk = (int)(sb % c.blocks);
    const int cache = (int)(sb / c.blocks);
    const int C = c.hd / 8, dkv = c.heads * c.hd;
    const int t0 = blk << c.lblock;
    const int rows = min(1 << c.lblock, c.T - t0);
    const int chunks = rows * C;
    const int col0 = which * dkv + head * c.hd;
    uint8_t* const codes = c.codes + ((long)cache * c.T + t0) * 2 * dkv + col0;
    uint8_t* const sp = c.scales + ((long)cache * c.blocks + blk) * 2 * c.heads + which * c.heads + head;

    const int step_r = lanes / C, step_c = lanes % C;
    Chunk8<T> v[NV];
    // REWRITE: a kept chunk holds its codes' values unscaled, to be multiplied in float32
    // (a bf16 would lose the bits of scaled values below 2^-126)
    float mul[REWRITE ? NV : 1];
    auto value = [&](int i, int e) { return REWRITE ? v[i].at(e) * mul[REWRITE ? i : 0] : v[i].at(e); };
    if constexpr (REWRITE) {
        const int32_t* const src = src_row + (long)cache * c.T + t0;
        const float s = kv8_scale(*sp);
        bool any = false;
        int r = sub / C, col = sub % C;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (sub + i * lanes < chunks) {
                const int from = src[r];
                if (from >= 0 && from < kv_rows) {
                    any = true;
                    mul[i] = 1.0f;
                    v[i].load(kv + (long)from * 2 * dkv + col0 + col * 8);
                } else {
                    mul[i] = s;
                    v[i].decode(*reinterpret_cast<const uint2*>(codes + (long)r * 2 * dkv + col * 8), 1.0f);
                }
            }
            r += step_r;
            col += step_c;
            if (col >= C) { col -= C; ++r; }
        }
        int hit = any;
        for (int o = lanes / 2; o > 0; o >>= 1) hit |= __shfl_xor(hit, o, kWave);
        if (!hit) return;   // no new row in this block: codes and scale stay as they are
    } else {
        const T* const src = kv + ((long)cache * row_stride + t0) * 2 * dkv + col0;
        int r = sub / C, col = sub % C;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (sub + i * lanes < chunks) v[i].load(src + (long)r * 2 * dkv + col * 8);
            r += step_r;
            col += step_c;
            if (col >= C) { col -= C; ++r; }
        }
    }
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (sub + i * lanes < chunks) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = value(i, e);
                amax = fmaxf(amax, kv8_finite(x) ? fabsf(x) : 0.f);
            }
        }
    for (int o = lanes / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o, kWave));
    const uint32_t b = kv8_exponent(amax);
    const float inv = kv8_inverse(b);
    int r = sub / C, col = sub % C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (sub + i * lanes < chunks) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = value(i, e);
            *reinterpret_cast<uint2*>(codes + (long)r * 2 * dkv + col * 8) =
                make_uint2(kv8_encode4(x, inv), kv8_encode4(x + 4, inv));
        }
        r += step_r;
        col += step_c;
        if (col >= C) { col -= C; ++r; }
    }
    if (sub == 0) *sp = (uint8_t)b;
}

// Values of the listed tokens: a thread takes eight codes of a row. Bound by memory.
template <typename T>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(Kv8Cache c, Kv8Select sel, T* __restrict__ kv,
                                                              long row_stride) {
    const int b = blockIdx.y;
    const Kv8Req r = kv8_request(c, sel, b);
    const int dkv = c.heads * c.hd, per_row = 2 * dkv / 8;
    const long n = (long)r.nk * per_row;
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long)gridDim.x * kThreads) {
        const int at = (int)(i / per_row), ch = (int)(i - (long)at * per_row);
        const int t = r.keys ? r.keys[at] : at;
        if (t < 0 || t >= c.T) continue;
        const int head2 = ch * 8 / c.hd;   // K heads, then V heads
        const float s = kv8_scale(r.scales[(long)(t >> c.lblock) * 2 * c.heads + head2]);
        Chunk8<T> v;
        v.decode(*reinterpret_cast<const uint2*>(r.codes + (long)t * 2 * dkv + ch * 8), s);
        v.store(kv + ((long)b * row_stride + t) * 2 * dkv + ch * 8);
    }
}

// Ascending numbers of a request's tokens whose mask byte is zero: one workgroup
// per request, kScanThreads tokens at a time, their places from a prefix sum.
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

template <typename T, bool REWRITE>
void launch_quantize(const Kv8Cache& c, const void* kv, long row_stride, const int32_t* src_row, long kv_rows,
                     hipStream_t s) {
    const int per_tile = (1 << c.lblock) * (c.hd / 8);
    int lanes = 1;
    while (lanes < kWave && lanes < per_tile) lanes *= 2;
    const int nv = (per_tile + lanes - 1) / lanes;
    const long tiles = (long)c.n_caches * c.blocks * 2 * c.heads;
    const long per_group = kThreads / lanes;
    const dim3 grid((unsigned)((tiles + per_group - 1) / per_group)), block(kThreads);
    const T* p = static_cast<const T*>(kv);
#define MS_NV(n)                                                                                                    \
    hipLaunchKernelGGL((quantize_kernel<T, n, REWRITE>), grid, block, 0, s, c, p, row_stride, src_row, kv_rows, lanes, \
                       tiles)
    if (nv <= 1) MS_NV(1);
    else if (nv <= 2) MS_NV(2);
    else if (nv <= 4) MS_NV(4);
    else if (nv <= 8) MS_NV(8);
    else if (nv <= 16) MS_NV(16);
    else MS_NV(32);
#undef MS_NV
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

hipError_t launch_kv8_quantize(int dtype, const Kv8Cache& c, const void* kv, long row_stride, const int32_t* src_row,
                               long kv_rows, hipStream_t s) {
    if (dtype == kBF16) {
        if (src_row) launch_quantize<bf16_t, true>(c, kv, row_stride, src_row, kv_rows, s);
        else launch_quantize<bf16_t, false>(c, kv, row_stride, src_row, kv_rows, s);
    } else {
        if (src_row) launch_quantize<float, true>(c, kv, row_stride, src_row, kv_rows, s);
        else launch_quantize<float, false>(c, kv, row_stride, src_row, kv_rows, s);
    }
    return hipGetLastError();
}

hipError_t launch_kv8_dequantize(int dtype, const Kv8Cache& c, const Kv8Select& sel, void* kv, long row_stride,
                                 hipStream_t s) {
    const long most = (long)sel.ld_keys * (2 * c.heads * c.hd / 8);
    if (most == 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<long>((most + kThreads - 1) / kThreads, 1 << 16), sel.batch), block(kThreads);
    if (dtype == kBF16)
        hipLaunchKernelGGL(dequantize_kernel<bf16_t>, grid, block, 0, s, c, sel, static_cast<bf16_t*>(kv), row_stride);
    else
        hipLaunchKernelGGL(dequantize_kernel<float>, grid, block, 0, s, c, sel, static_cast<float*>(kv), row_stride);
    return hipGetLastError();
}

}  // namespace ms
