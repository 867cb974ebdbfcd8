// Row products of microscaled 4-bit operands (the format: mx4.h):
// out = epilogue(A W^T + bias), A [M][K] activations, W [N][K] weights.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 codes, each
// group of 32 by its two scales, and sums in float32. Lane l holds 32 codes (16
// bytes) of row l % 16, columns 32 (l / 16) on, and their exponent byte. W is the
// first operand, so that a lane's four results are four neighbouring columns of
// one output row.
#include <algorithm>
#include <cmath>

#include "gelu.h"
#include "mx4.h"

namespace ms {
namespace {

constexpr int kStep = 256;              // K elements per step
constexpr int kRowB = kStep / 2;        // bytes of a staged row
constexpr int kStepBlocks = kStep / kMxBlock;
constexpr uint32_t kAbsent = 0xfff00000u;

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// w's scale in byte OW of sw, a's in byte OA of sa.
template <int OW, int OA>
__device__ __forceinline__ f32x4_t mfma_mx4(const vec16& w, const vec16& a, f32x4_t c, int sw, int sa) {
    i32x8_t x = {}, y = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = (int)w.w[i];
        y[i] = (int)a.w[i];
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, OW, sw, OA, sa);
}
// The same with byte numbers that are constants once loops are unrolled.
template <int OW>
__device__ __forceinline__ f32x4_t mfma_mx4_a(const vec16& w, const vec16& a, f32x4_t c, int sw, int sa, int oa) {
    switch (oa) {
        case 0: return mfma_mx4<OW, 0>(w, a, c, sw, sa);
        case 1: return mfma_mx4<OW, 1>(w, a, c, sw, sa);
        case 2: return mfma_mx4<OW, 2>(w, a, c, sw, sa);
        default: return mfma_mx4<OW, 3>(w, a, c, sw, sa);
    }
}
__device__ __forceinline__ f32x4_t mfma_mx4_b(const vec16& w, const vec16& a, f32x4_t c, int sw, int ow, int sa, int oa) {
    switch (ow) {
        case 0: return mfma_mx4_a<0>(w, a, c, sw, sa, oa);
        case 1: return mfma_mx4_a<1>(w, a, c, sw, sa, oa);
        case 2: return mfma_mx4_a<2>(w, a, c, sw, sa, oa);
        default: return mfma_mx4_a<3>(w, a, c, sw, sa, oa);
    }
}

// Permutation of a staged row's eight 16-byte chunks: 16 rows' reads of one chunk take every bank in turn.
__device__ __forceinline__ int k_chunk(int r) { return (r >> 1) & 7; }

// Four columns n.. of row m to the output, with the epilogue.
template <typename T, int EPI>
__device__ __forceinline__ void finish(const GemmDesc& g, int m, int n, float v[4]) {
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

// First row, first column and K range of a workgroup's tile.
template <int BM, int BN>
__device__ __forceinline__ void tile_of(const GemmDesc& g, int& m0, int& n0, int& split) {
    const int mt = (g.M + BM - 1) / BM, nt = (g.N + BN - 1) / BN;
    const int lb = xcd_logical_block(blockIdx.x, mt * nt * g.ksplit);
    split = lb / (mt * nt);
    // groups of group_m row tiles, the column tiles of a group side by side: what an XCD works on stays in its L2
    const int in = lb % (mt * nt), per = g.group_m * nt, first = in / per * g.group_m;
    const int gm = min(g.group_m, mt - first), at = in % per;
    m0 = (first + at % gm) * BM;
    n0 = at / gm * BN;
}

// Four neighbouring elements as they lie.
template <typename T>
struct alignas(4 * sizeof(T)) Four {
    T v[4];
};

// A wave's MI x NI blocks of 16 x 16 outputs from (m0, n0) on: 16 rows at a time through LDS, so that it loads and
// stores whole lines of a row. A barrier for the workgroup; `smem` is the stages' memory. The residual is under way
// before it: fetched block by block, 8192 x 4096 x 16384 took 288 us instead of 269, 8192 x 4608 x 1152 77 instead of 62.
template <typename T, int EPI, int MI, int NI>
__device__ __forceinline__ void write_tile(const GemmDesc& g, int m0, int n0, int split, const f32x4_t (&acc)[NI][MI], uint8_t* smem,
                                           int wave, int lane) {
    constexpr int OLD = NI * 16 + 4;                    // floats of a row in LDS
    constexpr int COLS = NI * 4, ROWS = kWave / COLS;   // lanes of four columns per row, rows at a time
    static_assert(kWave % COLS == 0, "output lanes");
    constexpr int PASSES = 16 / ROWS;
    constexpr int AHEAD = sizeof(T) == 2 ? MI : 2;      // blocks whose residual is on its way, as many as the registers hold
    const int grp = lane / 16, l16 = lane % 16, col = lane % COLS * 4, n = n0 + col, row0 = lane / COLS;
    const bool whole = g.ksplit == 1, in = n < g.N;
    Four<T> res[MI][PASSES];
    auto fetch = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < PASSES; ++r) {
            const int m = m0 + j * 16 + row0 + r * ROWS;
            res[j][r] = Four<T>{};
            if (whole && in && m < g.M) res[j][r] = *reinterpret_cast<const Four<T>*>(static_cast<const T*>(g.R) + (long)m * g.N + n);
        }
    };
    if constexpr (EPI == kEpiBiasResid) {
#pragma unroll
        for (int j = 0; j < MI; ++j)
            if (j < AHEAD) fetch(j);
    }
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (whole && in) load4<T>(static_cast<const T*>(g.bias) + n, bias);
    __syncthreads();    // every wave is past its last read of the stages
    float* const so = reinterpret_cast<float*>(smem) + wave * 16 * OLD;
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        const int m = m0 + j * 16 + row0;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            store4<float>(so + l16 * OLD + i * 16 + grp * 4, v);
        }
        asm volatile("" ::: "memory");      // LDS operations of a wave are done in order
        if constexpr (EPI == kEpiBiasResid) {
            if (j > 0 && j + AHEAD - 1 < MI) fetch(j + AHEAD - 1);
        }
        float v[PASSES][4];
#pragma unroll
        for (int r = 0; r < PASSES; ++r) load4<float>(so + (row0 + r * ROWS) * OLD + col, v[r]);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int r = 0; r < PASSES; ++r) {
            if (!in || m + r * ROWS >= g.M) continue;
            if (!whole) {
                store4<float>(g.part + ((long)split * g.M + m + r * ROWS) * g.N + n, v[r]);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[r][e] += bias[e];
                if constexpr (EPI == kEpiBiasGelu) v[r][e] = gelu(v[r][e]);
                if constexpr (EPI == kEpiBiasResid) v[r][e] += Elt<T>::to_f32(res[j][r].v[e]);
            }
            store4<T>(static_cast<T*>(g.C) + (long)(m + r * ROWS) * g.N + n, v[r]);
        }
    }
}

// Tiles of BM x BN outputs by WM x WN waves, steps of 256 elements of K in two stages of LDS. Codes land
// there by direct loads; a step's scales (8 bytes a row) come through registers, a thread to a row, and are laid
// out so that a lane finds those of its row and columns for two fragments and both halves of the step in one word.
// 8192 x 4096 x 16384 in tiles of 256 takes 269 to 280 us by the card where such calls follow each other (290 to 300 among other
// work, up to 340 after an idle card), 3.9 to 4.1 PFLOP/s of the 7.1 to 7.7 that the instruction reaches alone:
// matrix cores busy 41%, the rest is the stream of operands into a CU (direct loads cost it about four cycles per 128-byte
// line, 512 of them a step) and its LDS reads, which two stages and one workgroup per CU overlap in part. A ring of three
// regions with the next step's fragments and scales (through LDS as well) read under the last products took 271 us too, 283
// against 283 at 8192 x 8192 x 8192, 49 against 53 at 8192 x 4608 x 1152: 1.4% over 16 sizes, not worth a second kernel.
template <int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int NT = WM * WN * kWave;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;      // 16 x 16 outputs of a wave
    static constexpr int CODEB = (BM + BN) * kRowB, SCALEB = (BM + BN) * kStepBlocks;
    static constexpr int STAGEB = CODEB + SCALEB;
    static constexpr int OUTB = WM * WN * 16 * (NI * 16 + 4) * 4;
    static constexpr int LDSB = 2 * STAGEB > OUTB ? 2 * STAGEB : OUTB;
    static constexpr int COPIES = (BM + BN) / 8;                    // of 1 KB
    static_assert(COPIES % (WM * WN) == 0 && BM % 64 == 0 && BN % 64 == 0 && BM + BN <= NT && MI % 2 == 0 && NI % 2 == 0, "tile");
};

template <typename T, int EPI, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave) void mx4_linear_kernel(Mx4LinearDesc d) {
    using C = Tile<BM, BN, WM, WN>;
    constexpr int MI = C::MI, NI = C::NI;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[C::LDSB];
    const GemmDesc& g = d.g;
    const uint32_t lds0 = lds_addr(smem);
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int grp = lane / 16, l16 = lane % 16;
    int m0, n0, split;
    tile_of<BM, BN>(g, m0, n0, split);
    const uint32_t rowb = (uint32_t)g.K / 2;
    const int blocks = g.K / kMxBlock;
    const int rows_a = min(BM, g.M - m0), rows_w = min(BN, g.N - n0);
    const u32x4_t ra = raw_rsrc(d.a + (long)m0 * rowb, (uint32_t)rows_a * rowb), rw = raw_rsrc(d.w + (long)n0 * rowb, (uint32_t)rows_w * rowb);
    const int steps = (g.K + kStep - 1) / kStep;
    const int t0 = split * g.kchunk, t1 = min(steps, t0 + g.kchunk);

    // stage: BM rows of A, then BN of W, a row's 16-byte chunks permuted by the row; then the scales
    constexpr int PER = C::COPIES / (WM * WN);
    uint32_t voff[PER];
    int chunk[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int q = i * WM * WN + wave, r = (q < BM / 8 ? q : q - BM / 8) * 8 + lane / 8;
        chunk[i] = (lane % 8) ^ k_chunk(r);
        voff[i] = (uint32_t)r * rowb + chunk[i] * 16;
    }
    auto issue = [&](int t, int st) {
        const bool whole = (t + 1) * kStepBlocks <= blocks;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * WM * WN + wave;
            const uint32_t off = whole || t * kStepBlocks + chunk[i] < blocks ? voff[i] + (uint32_t)t * kRowB : kAbsent;
            dma_buf16(q < BM / 8 ? ra : rw, off, 0, lds0 + st * C::STAGEB + q * 1024);
        }
    };
    // this thread's row of scales: eight bytes of step t, zeros past K and past the last row
    const bool row_of_a = tid < BM;
    const int srow = row_of_a ? tid : tid - BM;
    const bool has_row = tid < BM + BN && srow < (row_of_a ? rows_a : rows_w);
    const uint8_t* const sp = (row_of_a ? d.as + (long)(m0 + (has_row ? srow : 0)) * blocks : d.ws + (long)(n0 + (has_row ? srow : 0)) * blocks);
    auto load_scales = [&](int t, uint32_t (&v)[2]) {
        v[0] = v[1] = 0;
        if (!has_row || t >= t1) return;
        const uint8_t* const p = sp + t * kStepBlocks;
        const int n = min(kStepBlocks, blocks - t * kStepBlocks);
        if (n == kStepBlocks) {
            __builtin_memcpy(v, p, 8);      // of any alignment
        } else {
#pragma unroll
            for (int i = 0; i < kStepBlocks; ++i)
                if (i < n) v[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
        }
    };
    // [64 rows][lane group][row % 16][row / 16][half of the step]
    const uint32_t sdst = (uint32_t)(tid / 64 * 512 + tid % 16 * 8 + tid % 64 / 16 * 2);
    auto store_scales = [&](const uint32_t (&v)[2], int st) {
        if (tid >= BM + BN) return;
        uint8_t* const p = smem + st * C::STAGEB + C::CODEB + sdst;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *reinterpret_cast<uint16_t*>(p + k * 128) = (uint16_t)((v[0] >> (8 * k) & 0xff) | (v[1] >> (8 * k) & 0xff) << 8);
    };
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);
    auto scale_at = [&](int row) { return (uint32_t)(row / 64 * 512 + grp * 128 + l16 * 8 + row % 64 / 32 * 4); };

    f32x4_t acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    uint32_t next[2];
    if (t0 < t1) {
        load_scales(t0, next);
        issue(t0, 0);
        store_scales(next, 0);
        load_scales(t0 + 1, next);
    }
    for (int t = t0; t < t1; ++t) {
        wait_all();     // step t has landed, and this wave's reads of the stage refilled below are done
        barrier_only();
        const int st = (t - t0) & 1;
        if (t + 1 < t1) {
            store_scales(next, st ^ 1);
            issue(t + 1, st ^ 1);
            load_scales(t + 2, next);
        }
        const uint8_t* const s = smem + st * C::STAGEB;
        uint32_t sa[MI / 2], sw[NI / 2];
#pragma unroll
        for (int j = 0; j < MI / 2; ++j) sa[j] = *reinterpret_cast<const uint32_t*>(s + C::CODEB + scale_at(wm + j * 32));
#pragma unroll
        for (int i = 0; i < NI / 2; ++i) sw[i] = *reinterpret_cast<const uint32_t*>(s + C::CODEB + scale_at(BM + wn + i * 32));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            vec16 fa[MI], fw[NI];
            const int c = ((k * 4 + grp) ^ k_chunk(l16)) * 16;
#pragma unroll
            for (int j = 0; j < MI; ++j) fa[j] = ld16(s + (wm + j * 16 + l16) * kRowB + c);
#pragma unroll
            for (int i = 0; i < NI; ++i) fw[i] = ld16(s + (BM + wn + i * 16 + l16) * kRowB + c);
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < MI; ++j)
                    acc[i][j] = mfma_mx4_b(fw[i], fa[j], acc[i][j], (int)sw[i / 2], i % 2 * 2 + k, (int)sa[j / 2], j % 2 * 2 + k);
        }
    }
    write_tile<T, EPI, MI, NI>(g, m0 + wm, n0 + wn, split, acc, smem, wave, lane);
}

// Few rows: 16 x 16 outputs per workgroup of up to 16 waves; every wave has 256-element steps of its own (step wave +
// waves i) and loads its fragments from global memory, so that the weights' rows are on their way at once; the waves'
// sums meet in LDS. Bound by latency, and with large weights by its loads, a lane's scale one byte of a line of its own: one row of
// 3456 x 1152 3.0 us, of 4096 x 16384 12.3 us (36 MB of weights, 2.9 TB/s), 3.5 and 12.9 us with weights that no cache holds.
template <typename T, int EPI>
__global__ __launch_bounds__(1024) void mx4_rows_kernel(Mx4LinearDesc d) {
    constexpr int OLD = 20;
    __shared__ __attribute__((aligned(16))) float smem[16 * 16 * OLD];
    const GemmDesc& g = d.g;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), waves = blockDim.x / kWave;
    const int grp = lane / 16, l16 = lane % 16;
    const int nt = (g.N + 15) / 16;
    const int n0 = (int)(blockIdx.x % nt) * 16, m0 = (int)(blockIdx.x / nt) * 16;
    const uint32_t rowb = (uint32_t)g.K / 2;
    const int blocks = g.K / kMxBlock, steps = (g.K + kStep - 1) / kStep;
    const int rows_a = min(16, g.M - m0), rows_w = min(16, g.N - n0);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(d.a + (long)m0 * rowb, (uint32_t)rows_a * rowb), rw = make_rsrc(d.w + (long)n0 * rowb, (uint32_t)rows_w * rowb);
    const __amdgpu_buffer_rsrc_t qa = make_rsrc(d.as + (long)m0 * blocks, (uint32_t)(rows_a * blocks)), qw = make_rsrc(d.ws + (long)n0 * blocks, (uint32_t)(rows_w * blocks));
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    struct Frag {
        vec16 w[2], a[2];
        int sw[2], sa[2];
    };
    auto load = [&](int t, Frag& f) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int b = t * kStepBlocks + k * 4 + grp;
            const bool in = t < steps && b < blocks;        // else zeros
            const uint32_t at = in ? (uint32_t)l16 * rowb + b * 16 : kAbsent;
            const int sat = in ? l16 * blocks + b : (int)kAbsent;
            f.w[k] = buf_ld16(rw, at, 0);
            f.a[k] = buf_ld16(ra, at, 0);
            f.sw[k] = __builtin_amdgcn_raw_buffer_load_b8(qw, sat, 0, 0);
            f.sa[k] = __builtin_amdgcn_raw_buffer_load_b8(qa, sat, 0, 0);
        }
    };
    auto multiply = [&](const Frag& f) {
#pragma unroll
        for (int k = 0; k < 2; ++k) acc = mfma_mx4<0, 0>(f.w[k], f.a[k], acc, f.sw[k], f.sa[k]);
    };
    Frag f0, f1;
    load(wave, f0);
    for (int t = wave; t < steps; t += 2 * waves) {
        load(t + waves, f1);        // past the last step: zeros
        multiply(f0);
        load(t + 2 * waves, f0);
        multiply(f1);
    }
    const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
    store4<float>(smem + (wave * 16 + l16) * OLD + grp * 4, v);
    __syncthreads();
    if (tid < 64) {         // a thread per row and four columns
        const int row = tid / 4, n = n0 + tid % 4 * 4, m = m0 + row;
        if (m < g.M && n < g.N) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < waves; ++w) {
                float p[4];
                load4<float>(smem + (w * 16 + row) * OLD + tid % 4 * 4, p);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] += p[r];
            }
            finish<T, EPI>(g, m, n, v);
        }
    }
}

template <typename T, int EPI>
hipError_t launch(const Mx4LinearDesc& d, hipStream_t s) {
    const GemmDesc& g = d.g;
    auto tiles = [&](int bm, int bn) { return dim3((unsigned)((long)((g.M + bm - 1) / bm) * ((g.N + bn - 1) / bn) * g.ksplit)); };
    switch (d.form) {
        case kMx4Rows: hipLaunchKernelGGL((mx4_rows_kernel<T, EPI>), tiles(16, 16), dim3(d.waves * kWave), 0, s, d); break;
        case kMx4Tile64: hipLaunchKernelGGL((mx4_linear_kernel<T, EPI, 64, 64, 2, 2>), tiles(64, 64), dim3(256), 0, s, d); break;
        case kMx4Tile128: hipLaunchKernelGGL((mx4_linear_kernel<T, EPI, 128, 128, 2, 2>), tiles(128, 128), dim3(256), 0, s, d); break;
        case kMx4Tile256: hipLaunchKernelGGL((mx4_linear_kernel<T, EPI, 256, 256, 4, 2>), tiles(256, 256), dim3(512), 0, s, d); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch(const Mx4LinearDesc& d, hipStream_t s) {
    switch (d.g.epilogue) {
        case kEpiBias: return launch<T, kEpiBias>(d, s);
        case kEpiBiasResid: return launch<T, kEpiBiasResid>(d, s);
        case kEpiBiasGelu: return launch<T, kEpiBiasGelu>(d, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

// Form and K split: the least modelled time. A form with tiles of its side takes, with k workgroups on the fullest of 256
// CUs (at most as many as fit) and `full` of the CUs busy, in us
//   a + rounds (steps (s0 + s1 k + s2 full) + o0 + o1 k)
// for `steps` of 256 columns in its K range, and a K split 2.2 + 1.37e-6 per range and output more. The form for few
// rows takes its steps in up to 16 waves at once. Fitted to 6105 measured times (21 widths and depths, 128 to 16384, by 20 row counts,
// 1 to 8192, each form, 1 to 16 ranges); the chosen pair takes 1.015 times the fastest on average, 1.38 times at most (one row of
// 4096 x 16384, with a workspace, 14.9 us in 16 ranges of tiles of 64; the form for few rows has 12.3). In
// us, as graphs of one card, rows / 64 / 128 / 256: 16 x 1152 x 1152 4.6 / 6.0 / 8.6 / 15, 410 x 4608 x 1152 - / 8.4 / 10.5 / 17, 3000 x 2304 x 768 - / 12.2 /
// 11.5 / 14.7, 8192 x 4096 x 16384 - / 588 / 350 / 276; 64 x 4096 x 16384 in 1 / 2 / 4 / 8 / 16 ranges 40 / 25 / 17 / 16 / 19.
void plan_mx4_linear(Mx4LinearDesc& d, size_t part_floats) {
    GemmDesc& g = d.g;
    const int steps = (g.K + kStep - 1) / kStep;
    d.form = kMx4Rows;
    d.waves = std::min(16, steps);
    g.ksplit = 1;
    g.kchunk = steps;
    g.group_m = 4;
    if (g.M == 0) return;
    struct Form {
        int form, side, most;
        double a, s0, s1, s2, o0, o1;
    };
    static const Form forms[] = {{kMx4Tile64, 64, 4, 3.67, 0.235, 0.161, 0.149, 0.0, 0.44},
                                 {kMx4Tile128, 128, 2, 3.95, 0.468, 0.247, 0.267, 0.0, 1.48},
                                 {kMx4Tile256, 256, 1, 2.9, 0.868, 0.668, 0.484, 4.36, 0.769}};
    const double mn = (double)g.M * g.N;
    double least = 1e30;
    if (g.M <= 256) {
        const double tiles = (double)((g.M + 15) / 16) * ((g.N + 15) / 16);
        least = 2.35 + 1.06 * ((steps + d.waves - 1) / d.waves) + 2.53e-6 * tiles * g.K + 0.061 * std::ceil(tiles / 256) * d.waves + 0.82e-6 * g.M * g.K;
    }
    for (const Form& f : forms) {
        const long tiles = (long)((g.M + f.side - 1) / f.side) * ((g.N + f.side - 1) / f.side);
        int before = 0;
        for (int want : {1, 2, 3, 4, 6, 8, 12, 16}) {
            const int chunk = (steps + want - 1) / want, n = (steps + chunk - 1) / chunk;
            if (n == before || want > steps) continue;
            before = n;
            if (n > 1 && ((size_t)n > part_floats / ((size_t)g.M * g.N) || tiles * n >= (1l << 22))) break;
            const double q = std::ceil(tiles * n / 256.0), k = std::min(q, (double)f.most), rounds = std::max(1.0, q / f.most);
            const double full = std::min(1.0, tiles * n / 256.0);
            double us = f.a + rounds * (chunk * (f.s0 + f.s1 * k + f.s2 * full) + f.o0 + f.o1 * k);
            if (n > 1) us += 2.2 + 1.37e-6 * n * mn;
            if (us < least) {
                least = us;
                d.form = f.form;
                g.ksplit = n;
                g.kchunk = chunk;
            }
        }
    }
}

hipError_t launch_mx4_linear(int dtype, const Mx4LinearDesc& d, hipStream_t s) {
    if (d.g.M == 0) return hipSuccess;
    hipError_t e = dtype == kBF16 ? launch<bf16_t>(d, s) : launch<float>(d, s);
    return e == hipSuccess ? launch_gemm_reduce(dtype, d.g, s) : e;
}

}  // namespace ms
