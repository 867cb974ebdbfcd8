// Row products of microscaled 4-bit operands (the format: mx4.h):
// out = epilogue(A W^T + bias), A [M][K] activations, W [N][K] weights.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 codes, each
// group of 32 by its two scales, and sums in float32. Lane l holds 32 codes (16
// bytes) of row l % 16, columns 32 (l / 16) on, and their exponent byte. W is the
// first operand, so that a lane's four results are four neighbouring columns of
// one output row.
#include "gelu.h"
#include "mx4.h"

namespace ms {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = 256;              // K elements per step
constexpr int kRowB = kStep / 2;        // bytes of a staged row
constexpr uint32_t kAbsent = 0xfff00000u;

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4_t mfma_mx4(const vec16& w, const vec16& a, f32x4_t c, int sw, int sa) {
    i32x8_t x = {}, y = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = (int)w.w[i];
        y[i] = (int)a.w[i];
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, sw, 0, sa);
}

// Permutation of a staged row's eight 16-byte chunks: 16 rows' reads of one chunk take every bank in turn.
__device__ __forceinline__ int k_chunk(int r) { return (r >> 1) & 7; }

// Four columns n.. of row m: to the output with the epilogue, or to the K range's part.
template <typename T, int EPI>
__device__ __forceinline__ void finish(const GemmDesc& g, int m, int n, int split, const f32x4_t& acc) {
    float v[4] = {acc[0], acc[1], acc[2], acc[3]};
    if (g.ksplit > 1) {
        store4<float>(g.part + ((long)split * g.M + m) * g.N + n, v);
        return;
    }
    float b[4];
    load4<T>(static_cast<const T*>(g.bias) + n, b);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] += b[r];
    if constexpr (EPI == kEpiBiasGelu) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = gelu(v[r]);
    }
    if constexpr (EPI == kEpiBiasResid) {
        load4<T>(static_cast<const T*>(g.R) + (long)m * g.N + n, b);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += b[r];
    }
    store4<T>(static_cast<T*>(g.C) + (long)m * g.N + n, v);
}

template <typename T, int EPI>
__global__ __launch_bounds__(kThreads) void mx4_linear_kernel(Mx4LinearDesc d) {
    constexpr int BM = 128, BN = 128, STAGEB = (BM + BN) * kRowB;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * STAGEB];
    const GemmDesc& g = d.g;
    const uint32_t lds0 = lds_addr(smem);
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int grp = lane / 16, l16 = lane % 16;
    const int mt = (g.M + BM - 1) / BM, nt = (g.N + BN - 1) / BN;
    const int lb = xcd_logical_block(blockIdx.x, mt * nt * g.ksplit);
    const int m0 = lb % mt * BM, n0 = lb / mt % nt * BN, split = lb / (mt * nt);
    const uint32_t rowb = (uint32_t)g.K / 2, blocks = (uint32_t)g.K / kMxBlock;
    const int rows_a = min(BM, g.M - m0), rows_w = min(BN, g.N - n0);
    const u32x4_t ra = raw_rsrc(d.a + (long)m0 * rowb, (uint32_t)rows_a * rowb), rw = raw_rsrc(d.w + (long)n0 * rowb, (uint32_t)rows_w * rowb);
    const __amdgpu_buffer_rsrc_t sa = make_rsrc(d.as + (long)m0 * blocks, (uint32_t)rows_a * blocks), sw = make_rsrc(d.ws + (long)n0 * blocks, (uint32_t)rows_w * blocks);
    const int steps = (g.K + kStep - 1) / kStep;
    const int t0 = split * g.kchunk, t1 = min(steps, t0 + g.kchunk);

    // stage: BM rows of A, then BN of W, a row's 16-byte chunks permuted by the row
    auto issue = [&](int t, int st) {
#pragma unroll
        for (int i = 0; i < (BM + BN) / 8 / 4; ++i) {
            const int q = i * 4 + wave, r = (q * 8 + lane / 8) % BM;
            const int c = t * 8 + ((lane % 8) ^ k_chunk(r));
            const uint32_t off = c < (int)blocks ? (uint32_t)r * rowb + c * 16 : kAbsent;
            dma_buf16(q < BM / 8 ? ra : rw, off, 0, lds0 + st * STAGEB + q * 1024);
        }
    };
    const int wm = wave % 2 * 64, wn = wave / 2 * 64;
    int xa[2][4], xw[2][4];
    auto scales = [&](int t) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = t * 8 + k * 4 + grp;
                const bool in = c < (int)blocks;
                xa[k][i] = __builtin_amdgcn_raw_buffer_load_b8(sa, in ? (wm + i * 16 + l16) * blocks + c : kAbsent, 0, 0);
                xw[k][i] = __builtin_amdgcn_raw_buffer_load_b8(sw, in ? (wn + i * 16 + l16) * blocks + c : kAbsent, 0, 0);
            }
    };
    f32x4_t acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (t0 < t1) {
        scales(t0);
        issue(t0, 0);
    }
    for (int t = t0; t < t1; ++t) {
        int ca[2][4], cw[2][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ca[k][i] = xa[k][i];
                cw[k][i] = xw[k][i];
            }
        wait_all();
        barrier_only();
        if (t + 1 < t1) {
            scales(t + 1);
            issue(t + 1, (t + 1 - t0) & 1);
        }
        const uint8_t* const s = smem + ((t - t0) & 1) * STAGEB;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            vec16 fa[4], fw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = ((k * 4 + grp) ^ k_chunk(l16)) * 16;
                fa[i] = ld16(s + (wm + i * 16 + l16) * kRowB + c);
                fw[i] = ld16(s + (BM + wn + i * 16 + l16) * kRowB + c);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma_mx4(fw[i], fa[j], acc[i][j], cw[k][i], ca[k][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = n0 + wn + i * 16 + grp * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + wm + j * 16 + l16;
            if (m < g.M && n < g.N) finish<T, EPI>(g, m, n, split, acc[i][j]);
        }
    }
}

template <typename T>
hipError_t launch(const Mx4LinearDesc& d, hipStream_t s) {
    const GemmDesc& g = d.g;
    const dim3 grid((unsigned)(((g.M + 127) / 128) * ((g.N + 127) / 128) * g.ksplit)), block(kThreads);
    switch (g.epilogue) {
        case kEpiBias: hipLaunchKernelGGL((mx4_linear_kernel<T, kEpiBias>), grid, block, 0, s, d); break;
        case kEpiBiasResid: hipLaunchKernelGGL((mx4_linear_kernel<T, kEpiBiasResid>), grid, block, 0, s, d); break;
        case kEpiBiasGelu: hipLaunchKernelGGL((mx4_linear_kernel<T, kEpiBiasGelu>), grid, block, 0, s, d); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

void plan_mx4_linear(Mx4LinearDesc& d, size_t part_floats) {
    GemmDesc& g = d.g;
    const int steps = (g.K + kStep - 1) / kStep;
    d.form = 0;
    g.ksplit = 1;
    g.kchunk = steps;
}

hipError_t launch_mx4_linear(int dtype, const Mx4LinearDesc& d, hipStream_t s) {
    if (d.g.M == 0) return hipSuccess;
    hipError_t e = dtype == kBF16 ? launch<bf16_t>(d, s) : launch<float>(d, s);
    return e == hipSuccess ? launch_gemm_reduce(dtype, d.g, s) : e;
}

}  // namespace ms
