// Attention over an 8-bit K/V cache: packed query rows of a batch over the
// listed cached tokens of their request (codes and scales) and its fresh K/V
// rows (the model's type), one softmax over both. A row without any key is 0.
//
// A query slot is a (packed row, query head of one K/V head's group) pair, so
// query heads that share a K/V head share its tiles. A request's keys form
// tiles: the listed cached tokens first, then the fresh rows. Tiles are staged
// through registers: lane l of a wave holds tile key l's token number (read one
// tile ahead), the row's offset and its two scales; the threads fetch the rows'
// chunks by those offsets, convert codes to bf16 with their scales (exact: a
// scale is a power of two) on the way to LDS, and the products run on bf16
// matrix instructions in the layout of attention.hip: S^T = K Q^T leaves the
// weights in the operand layout of O^T = V^T P^T, V is read transposed by
// ds_read_b64_tr_b16, rows of ones in V^T give the denominator. Absent keys
// (past a list's end, numbers out of range) are zero rows with score -inf.
// Scores, maxima, sums and the parts of key ranges are float32. bf16 rounds
// twice: the weights, the matrix cores' operand of the second product (both
// numerator and denominator take the rounded ones), and the output.
#include <algorithm>
#include <cmath>

#include "attn_tiles.h"
#include "kernels.h"
#include "kv8.h"

namespace ms {
namespace {

constexpr int kThreads = 256;

// LDS operations of the wave done (vector-memory loads may stay in flight).
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xc07f); }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Which query slots and key tiles a workgroup has.
struct Work {
    int row0;       // first packed row of the segment
    int slots;      // query slots of the segment
    int q0;         // first slot of this tile
    int kvh;        // K/V head
    int split;
    int t0, t1;     // key tiles
    int ntc;        // cached tiles of the request
    Kv8Req r;
};

// Slot tile `tile` of all segments, K/V head and key range; false: past the last tile.
template <int QT, int KT>
__device__ __forceinline__ bool find_work(const Kv8AttnDesc& a, int tile, int kvh, int split, Work& w) {
    // lane l reads what belongs to segment l (then l + 64), all at once
    const int lane = threadIdx.x % kWave;
    for (int s0 = 0; s0 < a.nseg; s0 += kWave) {
        const int s = min(s0 + lane, a.nseg - 1);
        const int b = a.seg_req ? a.seg_req[s] : s;
        const bool known = b >= 0 && b < a.sel.batch;
        const int bs = known ? b : 0;
        const int r0 = min(max(a.seg_start[s], 0), a.M), r1 = min(max(a.seg_start[s + 1], r0), a.M);
        int cc, sc, f0 = 0, nf = 0;
        int nk = kv8_request(a.c, a.sel, bs, cc, sc).nk;
        if (a.kv) {
            Kv8Req f{};
            kv8_fresh(a, bs, f);
            f0 = f.f0;
            nf = f.nf;
        }
        if (!known) nk = nf = 0;
        const int own = s0 + lane < a.nseg ? ((r1 - r0) * a.group + QT - 1) / QT : 0;
        int upto = own;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int v = __shfl_up(upto, o, kWave);
            if (lane >= o) upto += v;
        }
        const uint64_t past = __ballot(upto > tile);
        if (!past) {
            tile -= __builtin_amdgcn_readlane(upto, kWave - 1);
            continue;
        }
        const int at = uniform(__ffsll((unsigned long long)past) - 1);
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
        w.row0 = of(r0);
        w.slots = (of(r1) - w.row0) * a.group;
        w.q0 = (tile - of(upto - own)) * QT;
        w.kvh = kvh;
        w.split = split;
        w.r.nk = of(nk);
        w.r.f0 = of(f0);
        w.r.nf = of(nf);
        w.r.codes = a.c.codes + (long)of(cc) * a.c.T * 2 * a.c.heads * a.c.hd;
        w.r.scales = a.c.scales + (long)of(sc) * a.c.blocks * 2 * a.c.heads;
        w.r.keys = a.sel.keys ? a.sel.keys + (long)of(bs) * a.sel.ld_keys : nullptr;
        w.ntc = (w.r.nk + KT - 1) / KT;
        const uint32_t nt = w.ntc + (w.r.nf + KT - 1) / KT;   // below 2^24; times 64 ranges below 2^32
        w.t0 = (int)(nt * split / a.nsplit);
        w.t1 = (int)(nt * (split + 1) / a.nsplit);
        return true;
    }
    return false;
}

// Row index of a query slot's (row, query head) in [M][n_heads].
__device__ __forceinline__ long slot_row(const Kv8AttnDesc& a, const Work& w, int slot) {
    const int HG = a.c.heads * a.group;
    if (a.group == 1) return (long)(w.row0 + slot) * HG + w.kvh;
    const int r = slot / a.group;
    return (long)(w.row0 + r) * HG + w.kvh * a.group + (slot - r * a.group);
}

// Staging of KT-key tiles by NT threads, of the listed cached tokens or (FRESH)
// of the fresh rows. A thread keeps one chunk column of CW elements and takes the
// rows r0, r0 + RS, ... of the K rows followed by the V rows, so that its
// addresses differ by constants. Loads are unconditional (absent keys load
// nothing or a row that is then zeroed) and their results untouched until the
// next step, so that no branch or use makes a wave wait for what it has just
// issued.
template <int HD, int KT, int NT, bool FRESH>
struct Stager {
    static constexpr int CW = HD % 16 == 0 ? 16 : HD % 24 == 0 ? 24 : 8;
    static constexpr int CR = HD / CW;                  // chunks per row
    static constexpr int RS = NT / CR;                  // rows per pass
    static constexpr int NCH = (2 * KT + RS - 1) / RS;  // passes
    static constexpr int NV = FRESH ? CW / 8 : (CW + 15) / 16;   // 16-byte loads per chunk (the last of 24 codes: 8 bytes)
    static constexpr int ROWB = HD * 2;
    static constexpr int TILEB = KT * ROWB;
    static constexpr int KPAD = 32;                     // zeros past the K tile, read by padding slots of the last QK step
    static constexpr int TRASH = 2 * TILEB + KPAD;      // 64 bytes past the tiles, never read
    static constexpr int STAGEB = TRASH + 64;
    static constexpr bool SWZ = ROWB == 128 || ROWB == 256 || ROWB % 128 == 64;
    static constexpr int gcd16(int x) { return x % 16 == 0 ? 16 : x % 8 == 0 ? 8 : x % 4 == 0 ? 4 : x % 2 == 0 ? 2 : 1; }
    static constexpr int PER = SWZ ? 16 / gcd16(RS) : 1;    // the swizzles repeat every 16 rows
    static constexpr int ND = PER < NCH ? PER : NCH;
    // Offset of an absent key: past every cache's end and every scale table's, so that codes and
    // exponent bytes read as zeros. (An absent key with some present token's scale would be NaN
    // where that is NaN, and 0 weight times NaN in the second product.)
    static constexpr uint32_t kAbsent = 0xfff00000u;

    __amdgpu_buffer_rsrc_t rsrc, rscale, rlist;
    int lane, r0;
    int count;              // keys of this kind
    bool listed;            // whether rlist holds their numbers
    uint32_t row_bytes;     // of a token's codes
    uint32_t kcol, vcol;    // first element of this thread's K and V chunks within a token's row
    uint32_t dk[ND], dv[ND];// LDS offsets of the chunk of row r0 + i RS within a stage, less i RS rows
    vec16 raw[NCH][NV];
    uint32_t sk, sv;        // this lane's key: its scales' exponent bytes
    int num;                // list entry of this lane's key in the next tile to issue
    uint64_t valid;         // present keys of the tile in raw

    // pass i's row among the V rows: compile-time where no pass straddles the border
    __device__ __forceinline__ bool in_v(int i) const {
        if (i * RS >= KT) return true;
        if ((i + 1) * RS <= KT) return false;
        return r0 + i * RS >= KT;
    }
    __device__ __forceinline__ bool in_tile(int i) const { return (NT % CR == 0 && (i + 1) * RS <= 2 * KT) || r0 + i * RS < 2 * KT; }
    // tile key of pass i (any lane number past the tile's end)
    __device__ __forceinline__ int key(int i) const { return r0 + i * RS - (in_v(i) ? KT : 0); }

    __device__ __forceinline__ void init(const Kv8AttnDesc& a, const Work& w, int tid) {
        lane = threadIdx.x % kWave;
        const int dkv = a.c.heads * HD;
        row_bytes = 2 * dkv;
        count = FRESH ? w.r.nf : w.r.nk;
        const int32_t* const l = FRESH ? (a.f_rows ? a.f_rows + w.r.f0 : nullptr) : w.r.keys;
        listed = l != nullptr;
        rlist = make_rsrc(l, listed ? (uint32_t)count * 4u : 0u);
        if constexpr (!FRESH) {
            rsrc = make_rsrc(w.r.codes, (uint32_t)a.c.T * row_bytes);
            rscale = make_rsrc(w.r.scales, (uint32_t)a.c.blocks * 2u * a.c.heads);
        }
        r0 = tid / CR;
        const int col = tid % CR;
        if (r0 >= RS) r0 = 2 * KT;      // NT % CR threads have no chunk
        kcol = w.kvh * HD + col * CW;
        vcol = kcol + dkv;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int r = r0 + i * RS;
            dk[i] = r0 * ROWB + (((col * (CW / 8)) ^ k_swz<ROWB>(r % 16)) * 16);
            dv[i] = r0 * ROWB + (((col * (CW / 8)) ^ v_swz<ROWB>((r + 2 * KT - KT) % 16)) * 16) + KPAD;
        }
    }
    // reads the list entry of this lane's key of tile t
    __device__ __forceinline__ void fetch_index(int t) {
        num = (int)__builtin_amdgcn_raw_buffer_load_b32(rlist, (t * KT + lane) * 4, 0, 0);   // past the end: 0
    }
    // starts the loads of tile t, whose numbers fetch_index has read; past the last tile of the range (`end`) every key is absent
    __device__ __forceinline__ void issue(const Kv8AttnDesc& a, const Work& w, int t, int end) {
        const int i = t * KT + lane;
        const int v = listed ? num : (FRESH ? w.r.f0 : 0) + i;
        const bool there = t < end && lane < KT && i < count && v >= 0 && (FRESH ? v < a.kv_rows : v < a.c.T);
        valid = __ballot(there);
        if constexpr (!FRESH) {
            const uint32_t off = there ? (uint32_t)v * row_bytes : kAbsent;
            const int so = there ? (v >> a.c.lblock) * (2 * a.c.heads) + w.kvh : (int)kAbsent;
            sk = __builtin_amdgcn_raw_buffer_load_b8(rscale, so, 0, 0);
            sv = __builtin_amdgcn_raw_buffer_load_b8(rscale, so, a.c.heads, 0);
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const uint32_t o = (uint32_t)__shfl((int)off, key(i), kWave) + (in_v(i) ? vcol : kcol);
                if constexpr (CW >= 16) raw[i][0] = buf_ld16(rsrc, o, 0);
                if constexpr (CW % 16 == 8) {
                    const auto v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)(o + CW - 8), 0, 0);
                    raw[i][NV - 1].w[0] = v[0];
                    raw[i][NV - 1].w[1] = v[1];
                }
            }
        } else {
            const int row = there ? v : 0;
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const long from = __shfl(row, key(i), kWave);
                const bf16_t* p = static_cast<const bf16_t*>(a.kv) + from * row_bytes + (in_v(i) ? vcol : kcol);
#pragma unroll
                for (int j = 0; j < NV; ++j) raw[i][j] = ld16(p + 8 * j);
            }
        }
    }
    // the tile in raw, as bf16, to the stage at smem
    __device__ __forceinline__ void store(uint8_t* smem) {
        if constexpr (!FRESH) {
            // the two scales as the upper halves of their float32 values
            const uint32_t both = (__float_as_uint(kv8_scale(sk)) >> 16) | __float_as_uint(kv8_scale(sv));
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const uint32_t pr = (uint32_t)__shfl((int)both, key(i), kWave);
                const float s = __uint_as_float(in_v(i) ? pr & 0xffff0000u : pr << 16);
                vec16 o[CW / 8];
#pragma unroll
                for (int j = 0; j < CW / 8; ++j) {
                    const uint32_t c0 = raw[i][j / 2].w[2 * (j % 2)], c1 = raw[i][j / 2].w[2 * (j % 2) + 1];
                    o[j].w[0] = kv8_to_bf16x2<false>(c0, s);
                    o[j].w[1] = kv8_to_bf16x2<true>(c0, s);
                    o[j].w[2] = kv8_to_bf16x2<false>(c1, s);
                    o[j].w[3] = kv8_to_bf16x2<true>(c1, s);
                }
                put(i, o, smem);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const bool there = (valid >> (key(i) & 63)) & 1;
                vec16 o[CW / 8];
#pragma unroll
                for (int j = 0; j < CW / 8; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[j].w[k] = there ? raw[i][j].w[k] : 0u;
                put(i, o, smem);
            }
        }
    }
    // a thread without a row in this pass writes past the stage's tiles instead of branching
    __device__ __forceinline__ void put(int i, const vec16 (&o)[CW / 8], uint8_t* smem) {
        const uint32_t d = in_v(i) ? dv[i % ND] : dk[i % ND], there = in_tile(i);
        const uint32_t at = there ? d + i * RS * ROWB : TRASH;
        st16(smem + at, o[0]);
        if constexpr (CW == 16) st16(smem + (at ^ 16), o[1]);
        if constexpr (CW == 24) {   // rows without a swizzle
            st16(smem + at + 16, o[1]);
            st16(smem + at + 32, o[2]);
        }
    }
};

// Staging of the fresh rows' 64-key tiles by the four waves of a workgroup with
// direct-to-LDS loads: they need no conversion. Absent keys' rows read as zeros.
template <int HD, int KT, typename S>
struct FreshDma {
    static constexpr int ROWB = HD * 2, TILEB = KT * ROWB;
    static constexpr int INSTR = TILEB / 1024;          // 1 KB copies per tile
    static constexpr int NQ = 2 * INSTR;                // K then V
    static constexpr int IPW = (NQ + 3) / 4;            // copies per wave (most)
    static_assert(TILEB % 1024 == 0, "tile copies");
    u32x4_t rsrc;
    __amdgpu_buffer_rsrc_t rlist;
    int lane, wave, count, f0;
    bool listed;
    uint32_t row_bytes;
    int rl[IPW];
    uint32_t col[IPW], dst[IPW];
    int num;
    uint64_t valid;

    __device__ __forceinline__ void init(const Kv8AttnDesc& a, const Work& w, int wave_, int lane_) {
        lane = lane_;
        wave = wave_;
        count = w.r.nf;
        f0 = w.r.f0;
        const int32_t* const l = a.f_rows ? a.f_rows + f0 : nullptr;
        listed = l != nullptr;
        rlist = make_rsrc(l, listed ? (uint32_t)count * 4u : 0u);
        row_bytes = 4u * a.c.heads * HD;
        rsrc = raw_rsrc(a.kv, (uint32_t)a.kv_rows * row_bytes);
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int q = min(i * 4 + wave, NQ - 1);
            const bool isv = q >= INSTR;
            const int pos = (q % INSTR) * 1024 + lane * 16, r = pos / ROWB;
            rl[i] = r;
            col[i] = (isv ? row_bytes / 2 : 0u) + w.kvh * ROWB + (((pos % ROWB) / 16) ^ (isv ? v_swz<ROWB>(r) : k_swz<ROWB>(r))) * 16;
            dst[i] = uniform((isv ? TILEB + S::KPAD : 0) + (q % INSTR) * 1024);
        }
    }
    __device__ __forceinline__ void fetch_index(int t) {
        num = (int)__builtin_amdgcn_raw_buffer_load_b32(rlist, (t * KT + lane) * 4, 0, 0);   // past the end: 0
    }
    // tile t into the stage at LDS address `lds`
    __device__ __forceinline__ void issue(const Kv8AttnDesc& a, int t, int end, uint32_t lds) {
        const int i = t * KT + lane, v = listed ? num : f0 + i;
        const bool there = t < end && i < count && v >= 0 && v < a.kv_rows;
        valid = __ballot(there);
        const uint32_t off = there ? (uint32_t)v * row_bytes : S::kAbsent;
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const uint32_t o = (uint32_t)__shfl((int)off, rl[i], kWave) + col[i];
            if (i * 4 + wave < NQ) dma_buf16(rsrc, o, 0, lds + dst[i]);
        }
    }
};

// The four waves' sums of 16 slots, each relative to its own maximum (so [wave][slot][OLD]
// and sml [wave][slot]), to the output or the key range's part.
template <typename T, int HD, int OLD>
__device__ __forceinline__ void join_waves(const Kv8AttnDesc& a, const Work& w, const float* so, const float2* sml, int tid,
                                           int slot) {
    const int s = tid / 16;
    if (slot >= w.slots) return;
    float m = -INFINITY, f[4], sum = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) m = fmaxf(m, sml[v * 16 + s].x);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const float2 ml = sml[v * 16 + s];
        f[v] = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
        sum += f[v] * ml.y;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const long row = slot_row(a, w, slot), part = (long)w.split * a.M * a.c.heads * a.group + row;
    for (int c = (tid % 16) * 4; c < HD; c += 64) {
        float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float4 x = *reinterpret_cast<const float4*>(so + (v * 16 + s) * OLD + c);
            o[0] += f[v] * x.x; o[1] += f[v] * x.y; o[2] += f[v] * x.z; o[3] += f[v] * x.w;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] *= inv;
        if (a.nsplit == 1) store4<T>(static_cast<T*>(a.o) + row * HD + c, o);
        else store4<float>(a.part_o + part * HD + c, o);
    }
    if (a.nsplit > 1 && tid % 16 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * part) = make_float2(m, sum);
}

// Workgroups of the SHARED form that the registers let a CU hold.
constexpr int shared_per_cu(int hd) { return hd <= 16 ? 4 : hd <= 72 ? 3 : 2; }
// The same of the forms for few slots.
constexpr int few_per_cu(int hd, int slots) { return slots == 16 ? (hd <= 48 || hd == 64 ? 4 : hd <= 80 ? 3 : 2) : hd <= 32 ? 4 : hd <= 64 ? 3 : 2; }

// bf16. SHARED: 128 query slots, 32 per wave; the four waves share 64-key tiles in two stages, so
// that a key is converted once for 128 slots. Bound by the waves' own work on a tile (converting,
// softmax, products, each a sixth to a third of it, and little of one wave's under another's): 8
// requests of 123 to 2458 rows over 4096 keys of 16 heads of 72 (129 GFLOP) 215 to 230 us, 4 of 922
// to 2150 rows over 4608 keys of 24 heads of 128 (327 GFLOP) 375 us, 0.6 and 0.87 PFLOP/s; the
// matrix cores are busy 37% and 44% of the time. 256 slots (eight waves) gained 3 to 7% on long
// segments and lost more on short ones.
// Not SHARED: 16 or 32 slots, all of them in every wave, and every wave has key tiles of its own (32
// keys, tile t0 + wave + 4 i); the four partial results are joined at the end. Bound by the way of
// the codes through registers and LDS: 8 requests of 4 to 48 rows over 4096 keys of 16 heads of 72
// (77 MB, not in a cache) 30 us, 2.5 TB/s; 24 requests over 4096 keys of 16 heads of 64 4.5 TB/s.
template <int HD, int QT_>
struct Bf16Cfg {
    static constexpr int QT = QT_;
    static constexpr bool SHARED = QT == 128;
    static constexpr int KT = SHARED ? 64 : 32;
    static constexpr int NQB = QT == 16 ? 1 : 2;        // 16-slot blocks per wave
    static constexpr int NT = SHARED ? kThreads : kWave;
    static constexpr int STAGES = SHARED ? 2 : 1;
    using S = Stager<HD, KT, NT, false>;
    using F = Stager<HD, KT, NT, true>;
    static constexpr int NKS = KT / 16;
    static constexpr int NK32 = (HD + 31) / 32;
    static constexpr bool KTAIL = HD % 32 != 0;
    static constexpr bool SUM_IN_PAD = HD % 16 != 0;
    static constexpr int NREAL = (HD + 15) / 16;
    static constexpr int NHS = NREAL + (SUM_IN_PAD ? 0 : 1);
    static constexpr int LDSB = (SHARED ? STAGES : 4) * S::STAGEB;
};

template <int HD, int QT>
__global__ __launch_bounds__(kThreads, QT == 128 ? shared_per_cu(HD) : few_per_cu(HD, QT)) void attend_bf16_kernel(Kv8AttnDesc a, int qtiles) {
    using C = Bf16Cfg<HD, QT>;
    constexpr bool SHARED = C::SHARED;
    using S = typename C::S;
    constexpr int NQB = C::NQB, NKS = C::NKS;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[C::LDSB + 16];
    const uint32_t lds0 = lds_addr(smem);
    const uint32_t ones_rel = C::LDSB;                  // 8 bytes of bf16 ones (SUM_IN_PAD)

    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave);
    const int grp = lane / 16, l16 = lane % 16;
    // SHARED: a head's slot tiles side by side, so that an XCD's L2 serves a head's codes to
    // all of them. Else the heads of a (tile, range) pair side by side, which read neighbouring
    // parts of the same rows, and the pairs dealt out to the XCDs in turn: the tiles that no
    // segment fills come last and would leave whole XCDs idle in a contiguous split.
    Work w;
    if constexpr (SHARED) {
        const int lb = xcd_logical_block(blockIdx.x, qtiles * a.nsplit * a.c.heads);
        if (!find_work<C::QT, C::KT>(a, lb % qtiles, lb / (qtiles * a.nsplit), lb / qtiles % a.nsplit, w)) return;
    } else {
        const int i = blockIdx.x / kXcds, pair = i / a.c.heads * kXcds + blockIdx.x % kXcds;
        if (!find_work<C::QT, C::KT>(a, pair / a.nsplit, i % a.c.heads, pair % a.nsplit, w)) return;
    }
    constexpr int step = SHARED ? 1 : 4;

    // constant LDS: the K pads' zeros and the ones block
    constexpr int NSTG = SHARED ? C::STAGES : 4;
    if (tid < 2 * NSTG) *reinterpret_cast<uint4*>(smem + (tid / 2) * S::STAGEB + S::TILEB + (tid % 2) * 16) = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 2 * NSTG) *reinterpret_cast<uint2*>(smem + C::LDSB) = make_uint2(0x3f803f80u, 0x3f803f80u);

    // Q^T fragments (B operand), their sign that of the score scale
    bf16x8_t qf[NQB][C::NK32];
    const bf16_t* __restrict__ q = static_cast<const bf16_t*>(a.q);
    const int wq0 = w.q0 + (SHARED ? wave * 32 : 0);
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        const int slot = wq0 + qb * 16 + l16;
        const bf16_t* qp = q + slot_row(a, w, slot) * HD;
#pragma unroll
        for (int kc = 0; kc < C::NK32; ++kc) {
            vec16 v = {{0u, 0u, 0u, 0u}};
            if (slot < w.slots && kc * 32 + grp * 8 < HD) v = ld16(qp + kc * 32 + grp * 8);
#pragma unroll
            for (int j = 0; j < 4; ++j) v.w[j] ^= flip;
            qf[qb][kc] = __builtin_bit_cast(bf16x8_t, v);
        }
    }

    // fragment read offsets inside a stage (bytes)
    const int fK = k_swz<S::ROWB>(l16);
    uint32_t koff[C::NK32];
#pragma unroll
    for (int kc = 0; kc < C::NK32; ++kc) koff[kc] = l16 * S::ROWB + (((4 * kc + grp) ^ fK) * 16);
    // last QK step of a head_dim that is not a multiple of 32 (its rows are not swizzled): lanes
    // whose slots lie past the row read the stage's block of zeros
    static_assert(!C::KTAIL || !S::SWZ, "tail offsets");
    const bool in_row = (C::NK32 - 1) * 64 + grp * 16 < S::ROWB;
    const int rowA = 4 * grp + (l16 >> 2);
    const int fV = v_swz<S::ROWB>(rowA);
    uint32_t voffh[C::NREAL];
#pragma unroll
    for (int h = 0; h < C::NREAL; ++h) {
        const int hd = 16 * h + 4 * (l16 & 3);
        voffh[h] = S::TILEB + S::KPAD + rowA * S::ROWB + (((hd / 8) ^ fV) * 16) + (hd % 8) * 2;
    }
    const bool ones_lane = C::SUM_IN_PAD && (16 * (C::NREAL - 1) + 4 * (l16 & 3)) >= HD;

    f32x4_t oacc[NQB][C::NHS];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
        for (int h = 0; h < C::NHS; ++h) oacc[qb][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const float cs = fabsf(a.scale_log2), rescale_at = kRescaleLog2 / cs;
    float m_run[NQB];
    f32x4_t negm[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        m_run[qb] = -INFINITY;
        negm[qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    bool beyond = true;
    const bf16x8_t onesf = __builtin_bit_cast(bf16x8_t, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
    constexpr uint64_t kAll = C::KT == 64 ? ~0ull : (1ull << (C::KT % 64)) - 1;

    auto qk = [&](uint32_t sbase, f32x4_t (&sacc)[NQB][NKS]) {
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) sacc[qb][ks] = negm[qb];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
#pragma unroll
            for (int kc = 0; kc < C::NK32; ++kc) {
                uint32_t at = koff[kc] + ks * 16 * S::ROWB;
                if (C::KTAIL && kc == C::NK32 - 1) at = in_row ? at : (uint32_t)S::TILEB;
                const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(smem + sbase + at);
#pragma unroll
                for (int qb = 0; qb < NQB; ++qb) sacc[qb][ks] = mfma32(kf, qf[qb][kc], sacc[qb][ks]);
            }
        }
    };
    auto drop_absent = [&](uint64_t present, f32x4_t (&sacc)[NQB][NKS]) {
        if (present != kAll) {
            const uint64_t mine = present >> (grp * 4);
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!((mine >> (ks * 16 + r)) & 1)) {
#pragma unroll
                        for (int qb = 0; qb < NQB; ++qb) sacc[qb][ks][r] = -INFINITY;
                    }
        }
    };
    // online softmax in place: sacc becomes the weights; running maxima and accumulators
    // updated, a rescale only where a score exceeds its slot's maximum by more than 2^8
    auto softmax = [&](f32x4_t (&sacc)[NQB][NKS]) {
        float mx[NQB];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            mx[qb] = sacc[qb][0][0];
#pragma unroll
            for (int i = 1; i < 4 * NKS; ++i) mx[qb] = fmaxf(mx[qb], sacc[qb][i / 4][i % 4]);
        }
        float most = mx[0];
#pragma unroll
        for (int qb = 1; qb < NQB; ++qb) most = fmaxf(most, mx[qb]);
        if (beyond || __any(most > rescale_at)) {
            bool far = false;
#pragma unroll
            for (int qb = 0; qb < NQB; ++qb) {
                const float rm = rows_max(mx[qb]);
                const bool none = m_run[qb] == -INFINITY;
                const float was = none ? -INFINITY : m_run[qb] + negm[qb][0];
                const float up = fmaxf(rm, was);
                const bool still = up == -INFINITY;
                const float corr = none ? 0.f : fast_exp2((was - up) * cs);
#pragma unroll
                for (int h = 0; h < C::NHS; ++h) oacc[qb][h] *= corr;
                m_run[qb] = fmaxf(m_run[qb], rm - negm[qb][0]);
                const float n = m_run[qb] == -INFINITY ? 0.f : -fminf(fmaxf(m_run[qb], -kStartMax), kStartMax);
                negm[qb] = f32x4_t{n, n, n, n};
                far |= fabsf(m_run[qb]) > kStartMax;
                const float off = still ? 0.f : up;
#pragma unroll
                for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sacc[qb][ks][r] -= off;
            }
            beyond = __any(far);
        }
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                for (int r = 0; r < 4; ++r) sacc[qb][ks][r] = fast_exp2(sacc[qb][ks][r] * cs);
    };
    auto pv = [&](uint32_t sbase, f32x4_t (&sacc)[NQB][NKS]) {
        // without a swizzle the blocks of 16 columns lie 32 bytes apart, an offset of the reads
        constexpr int NB = S::SWZ ? C::NREAL : 1;
        uint32_t vbase[NB];
#pragma unroll
        for (int h = 0; h < NB; ++h) {
            vbase[h] = lds0 + sbase + voffh[h];
            asm volatile("" : "+v"(vbase[h]));   // keep the sum: offsets are added per read
        }
#pragma unroll
        for (int c = 0; c < C::KT / 32; ++c) {
            bf16x8_t vf[C::NHS];
#pragma unroll
            for (int h = 0; h < C::NHS; ++h) {
                if (h >= C::NREAL) {
                    vf[h] = onesf;
                } else {
                    const lds_cptr vb = (lds_cptr)(uintptr_t)vbase[S::SWZ ? h : 0] + (S::SWZ ? 0 : 32 * h);
                    lds_cptr p0 = vb + (32 * c) * S::ROWB, p1 = vb + (32 * c + 16) * S::ROWB;
                    if (h == C::NREAL - 1 && ones_lane) { p0 = (lds_cptr)(uintptr_t)(lds0 + ones_rel); p1 = p0; }
                    const bf16x4_t lo = ld_tr16(p0), hi = ld_tr16(p1);
                    vf[h] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
            }
            bf16x8_t pf[NQB];
#pragma unroll
            for (int qb = 0; qb < NQB; ++qb) {
                uint4 p;
                p.x = pack_bf16x2(sacc[qb][2 * c][0], sacc[qb][2 * c][1]);
                p.y = pack_bf16x2(sacc[qb][2 * c][2], sacc[qb][2 * c][3]);
                p.z = pack_bf16x2(sacc[qb][2 * c + 1][0], sacc[qb][2 * c + 1][1]);
                p.w = pack_bf16x2(sacc[qb][2 * c + 1][2], sacc[qb][2 * c + 1][3]);
                pf[qb] = __builtin_bit_cast(bf16x8_t, p);
            }
#pragma unroll
            for (int h = 0; h < C::NHS; ++h)
#pragma unroll
                for (int qb = 0; qb < NQB; ++qb) oacc[qb][h] = mfma32(vf[h], pf[qb], oacc[qb][h]);
        }
    };

    f32x4_t sa[NQB][NKS];
    const bool active = wq0 < w.slots;
    // Tiles [from, to) of one kind: tile t is in LDS, tile t + step in registers or on its way
    // there while t is multiplied; its conversion stands between the two products, under the
    // matrix instructions.
    auto run = [&](auto st, int from, int to, int skip) __attribute__((always_inline)) {
        if constexpr (!SHARED) from += (wave - skip) & 3;   // the waves go on in turn from one kind to the next
        if (from >= to) return;   // the whole workgroup, or a wave that waits for no other
        st.init(a, w, SHARED ? tid : lane);
        auto stage = [&](int n) { return (uint32_t)(SHARED ? (n & 1) * S::STAGEB : wave * S::STAGEB); };
        st.fetch_index(from);
        st.issue(a, w, from, to);
        st.fetch_index(from + step);
        uint64_t present = st.valid;
        st.store(smem + stage(0));
        st.issue(a, w, from + step, to);
        st.fetch_index(from + 2 * step);
        int n = 0;
        for (int t = from; t < to; t += step, ++n) {
            wait_lds();
            if constexpr (SHARED) barrier_only();
            else __builtin_amdgcn_wave_barrier();
            const uint64_t now = present;
            auto next = [&]() {
                present = st.valid;
                st.store(smem + stage(n + 1));
                st.issue(a, w, t + 2 * step, to);
                st.fetch_index(t + 3 * step);
            };
            if constexpr (SHARED) {
                if (!active) {
                    next();
                    continue;
                }
                // under the matrix instructions of QK, or before them at head_dim 72, the largest with
                // three workgroups per CU, which the registers saved make room for. In us, under / before:
                // 12 x 1024 rows of 16 heads over 4096 keys at 24 195 / 196, 40 234 / 237, 48 241 / 243, 56
                // 257 / 264, 72 320 / 305; 8 x 900 rows at 56 179 / 182, at 72 264 / 215
                if constexpr (S::SWZ || HD <= 64 || shared_per_cu(HD) != 3) {
                    qk(stage(n), sa);
                    next();
                } else {
                    next();
                    __builtin_amdgcn_sched_barrier(0);
                    qk(stage(n), sa);
                }
                drop_absent(now, sa);
                softmax(sa);
                pv(stage(n), sa);
            } else {
                qk(stage(n), sa);
                drop_absent(now, sa);
                softmax(sa);
                pv(stage(n), sa);
                asm volatile("" ::: "memory");
                next();
            }
        }
        if constexpr (SHARED) {
            wait_lds();
            barrier_only();   // the stages may be written again
        }
    };
    // the same of the fresh rows in the SHARED form: their loads land in LDS
    auto run_dma = [&](int from, int to) {
        if (from >= to) return;
        FreshDma<HD, 64, S> st;
        st.init(a, w, wave, lane);
        st.fetch_index(from);
        st.issue(a, from, to, lds0);
        st.fetch_index(from + 1);
        for (int t = from, n = 0; t < to; ++t, ++n) {
            const uint64_t now = st.valid;
            wait_all();   // tile t has landed, and this wave's reads of the stage refilled below are done
            barrier_only();
            if (t + 1 < to) {
                st.issue(a, t + 1, to, lds0 + ((n + 1) & 1) * S::STAGEB);
                st.fetch_index(t + 2);
            }
            if (!active) continue;
            qk((n & 1) * S::STAGEB, sa);
            drop_absent(now, sa);
            softmax(sa);
            pv((n & 1) * S::STAGEB, sa);
        }
    };
    __syncthreads();   // constant LDS
    const int c0 = min(w.t0, w.ntc), c1 = min(w.t1, w.ntc);
    run(typename C::S{}, c0, c1, 0);
    if (w.r.nf > 0) {
        const int f0 = max(w.t0 - w.ntc, 0), f1 = max(w.t1 - w.ntc, 0);
        if constexpr (SHARED) run_dma(f0, f1);
        else run(typename C::F{}, f0, f1, c1 - c0);
    }

    float l[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        if constexpr (C::SUM_IN_PAD) {
            // the last 8 rows of the last subtile are the ones rows: lane groups 2-3 hold them
            const float t0 = grp >= 2 ? oacc[qb][C::NHS - 1][0] : 0.f;
            auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(t0), __float_as_uint(t0), false, false);
            l[qb] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
        } else {
            l[qb] = oacc[qb][C::NHS - 1][0];
        }
    }
    const long range = (long)w.split * a.M * a.c.heads * a.group;
    __syncthreads();   // every wave is past its last read of the stages
    if constexpr (SHARED) {
        // through LDS: rows of a slot in 16-byte vectors, chunks swizzled by the slot where rows are a power of two
        constexpr int CH = HD / 8, CF = HD / 4;
        constexpr int SWM = (CH & (CH - 1)) == 0 ? (CH >= 16 ? 15 : CH - 1) : 0;
        constexpr int SWF = (CF & (CF - 1)) == 0 ? (CF >= 16 ? 15 : CF - 1) : 0;
        uint8_t* const so = smem + wave * 32 * S::ROWB * (a.nsplit == 1 ? 1 : 2);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            const float inv_l = l[qb] == 0.f ? 0.f : 1.0f / l[qb];
            const int rl = qb * 16 + l16;
#pragma unroll
            for (int h = 0; h < C::NHS; ++h) {
                const int cidx = h * 16 + grp * 4;
                if (cidx < HD) {
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = oacc[qb][h][r] * inv_l;
                    if (a.nsplit == 1)
                        store4<bf16_t>(reinterpret_cast<bf16_t*>(so + rl * S::ROWB + (((cidx / 8) ^ (rl & SWM)) * 16) + (cidx % 8) * 2), v);
                    else
                        store4<float>(reinterpret_cast<float*>(so + rl * 2 * S::ROWB) + ((cidx / 4) ^ (rl & SWF)) * 4, v);
                }
            }
            const int slot = wq0 + rl;
            if (a.nsplit > 1 && grp == 0 && slot < w.slots)
                *reinterpret_cast<float2*>(a.part_ml + 2 * (range + slot_row(a, w, slot))) = make_float2(m_run[qb] * cs, l[qb]);
        }
        __syncthreads();
        if (a.nsplit == 1) {
            for (int k = lane; k < 32 * CH; k += kWave) {
                const int rl = k / CH, c = k % CH;
                if (wq0 + rl < w.slots)
                    st16(static_cast<bf16_t*>(a.o) + slot_row(a, w, wq0 + rl) * HD + c * 8,
                         ld16(so + rl * S::ROWB + ((c ^ (rl & SWM)) * 16)));
            }
        } else {
            for (int k = lane; k < 32 * CF; k += kWave) {
                const int rl = k / CF, c = k % CF;
                if (wq0 + rl < w.slots)
                    st16(a.part_o + (range + slot_row(a, w, wq0 + rl)) * HD + c * 4,
                         ld16(so + rl * 2 * S::ROWB + ((c ^ (rl & SWF)) * 16)));
            }
        }
    } else {
        // the four waves' sums, each relative to its own maximum, joined through LDS 16 slots at a time
        constexpr int OLD = HD + 4;
        float* const so = reinterpret_cast<float*>(smem);
        float2* const sml = reinterpret_cast<float2*>(so + 4 * 16 * OLD);
        static_assert((4 * 16 * OLD + 4 * 16 * 2) * 4 <= C::LDSB, "join fits the stages");
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            if (qb > 0) __syncthreads();
#pragma unroll
            for (int h = 0; h < C::NREAL; ++h) {
                const int cidx = h * 16 + grp * 4;
                if (cidx < HD) {
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = oacc[qb][h][r];
                    store4<float>(so + (wave * 16 + l16) * OLD + cidx, v);
                }
            }
            if (grp == 0) sml[wave * 16 + l16] = make_float2(m_run[qb] * cs, l[qb]);
            __syncthreads();
            join_waves<bf16_t, HD, OLD>(a, w, so, sml, tid, w.q0 + qb * 16 + tid / 16);
        }
    }
}

// float32: 16 query slots, every wave has 32-key tiles of its own, joined at the end, as in
// the bf16 form for few slots. Bound by the float32 matrix instructions (HD of them per tile
// and wave, 32 cycles each, against ~300 cycles of staging), so the same form serves many slots.
template <int HD, bool FRESH>
struct StagerF32 {
    static constexpr int KT = 32;
    static constexpr int CW = HD % 16 == 0 ? 16 : 8;
    static constexpr int CR = HD / CW, RS = kWave / CR, NCH = (2 * KT + RS - 1) / RS;
    static constexpr int NV = FRESH ? CW / 4 : 1;       // 16-byte loads per chunk
    // words per row: 4 P = 16 or 48 mod 64 keeps the four rows that a transposed V read takes in different banks
    static constexpr int P = HD + 4;
    static constexpr int TRASH = 2 * KT * P;            // words past the K and V rows: spare chunks, reads past the last row
    static constexpr int WORDS = TRASH + 16;
    static constexpr uint32_t kAbsent = 0xfff00000u;    // as in Stager

    __amdgpu_buffer_rsrc_t rsrc, rscale, rlist;
    int lane, r0, col, count;
    bool listed;
    uint32_t row_elts, kcol;    // elements of a token's K and V rows; first K element of this lane's chunk
    vec16 raw[NCH][NV];
    uint32_t sk, sv;
    int num;
    uint64_t valid;

    __device__ __forceinline__ bool in_v(int i) const { return r0 + i * RS >= KT; }
    __device__ __forceinline__ int key(int i) const { return r0 + i * RS - (in_v(i) ? KT : 0); }

    __device__ __forceinline__ void init(const Kv8AttnDesc& a, const Work& w, int lane_) {
        lane = lane_;
        row_elts = 2 * a.c.heads * HD;
        count = FRESH ? w.r.nf : w.r.nk;
        const int32_t* const l = FRESH ? (a.f_rows ? a.f_rows + w.r.f0 : nullptr) : w.r.keys;
        listed = l != nullptr;
        rlist = make_rsrc(l, listed ? (uint32_t)count * 4u : 0u);
        if constexpr (FRESH) {
            rsrc = make_rsrc(a.kv, (uint32_t)a.kv_rows * row_elts * 4u);
        } else {
            rsrc = make_rsrc(w.r.codes, (uint32_t)a.c.T * row_elts);
            rscale = make_rsrc(w.r.scales, (uint32_t)a.c.blocks * 2u * a.c.heads);
        }
        r0 = lane / CR;
        col = lane % CR;
        if (r0 >= RS) r0 = 2 * KT;      // kWave % CR lanes have no chunk
        kcol = w.kvh * HD + col * CW;
    }
    __device__ __forceinline__ void fetch_index(int t) {
        num = (int)__builtin_amdgcn_raw_buffer_load_b32(rlist, (t * KT + lane) * 4, 0, 0);   // past the end: 0
    }
    __device__ __forceinline__ void issue(const Kv8AttnDesc& a, const Work& w, int t, int end) {
        const int i = t * KT + lane;
        const int v = listed ? num : (FRESH ? w.r.f0 : 0) + i;
        const bool there = t < end && lane < KT && i < count && v >= 0 && (FRESH ? v < a.kv_rows : v < a.c.T);
        valid = __ballot(there);
        const uint32_t off = there ? (uint32_t)v * row_elts * (FRESH ? 4u : 1u) : kAbsent;   // absent rows read as zeros
        if constexpr (!FRESH) {
            const int so = there ? (v >> a.c.lblock) * (2 * a.c.heads) + w.kvh : (int)kAbsent;
            sk = __builtin_amdgcn_raw_buffer_load_b8(rscale, so, 0, 0);
            sv = __builtin_amdgcn_raw_buffer_load_b8(rscale, so, a.c.heads, 0);
        }
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const uint32_t e = kcol + (in_v(i) ? row_elts / 2 : 0u);
            const uint32_t o = (uint32_t)__shfl((int)off, key(i), kWave) + e * (FRESH ? 4u : 1u);
            if constexpr (FRESH) {
#pragma unroll
                for (int j = 0; j < NV; ++j) raw[i][j] = buf_ld16(rsrc, o + 16 * j, 0);
            } else if constexpr (CW == 16) {
                raw[i][0] = buf_ld16(rsrc, o, 0);
            } else {
                const auto v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)o, 0, 0);
                raw[i][0].w[0] = v[0];
                raw[i][0].w[1] = v[1];
            }
        }
    }
    __device__ __forceinline__ void store(float* smem) {
        uint32_t both = 0;
        if constexpr (!FRESH) both = (__float_as_uint(kv8_scale(sk)) >> 16) | __float_as_uint(kv8_scale(sv));
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int r = r0 + i * RS;
            float* const p = smem + (r < 2 * KT ? r * P + col * CW : TRASH);
            if constexpr (FRESH) {
#pragma unroll
                for (int j = 0; j < NV; ++j) st16(p + 4 * j, raw[i][j]);
            } else {
                const uint32_t pr = (uint32_t)__shfl((int)both, key(i), kWave);
                const float s = __uint_as_float(in_v(i) ? pr & 0xffff0000u : pr << 16);
#pragma unroll
                for (int j = 0; j < CW / 4; ++j) {
                    const float2 x = kv8_to_f32x2<false>(raw[i][0].w[j], s), y = kv8_to_f32x2<true>(raw[i][0].w[j], s);
                    const float v[4] = {x.x, x.y, y.x, y.y};
                    store4<float>(p + 4 * j, v);
                }
            }
        }
    }
};

// float32: 16 query slots in every wave, 32-key tiles of its own per wave as in the bf16 forms for
// few slots, products on the float32 matrix instructions. Bound by them and by the staging in
// turn at few rows: 205 rows of 4 heads of 64 over 1024 keys (0.21 GFLOP) 14.5 us with the join, of
// which two launches are 8; 3 requests of 137 to 661 rows over 1687 keys of 26 heads of 64 (12.3 GFLOP)
// 180 us, 69 TFLOP/s, each key staged for every 16 rows. Two workgroups per CU hold 70 KB of LDS each.
template <int HD>
__global__ __launch_bounds__(kThreads, 2) void attend_f32_kernel(Kv8AttnDesc a) {
    using S = StagerF32<HD, false>;
    constexpr int KT = S::KT, P = S::P, NJ = (HD + 15) / 16;
    constexpr int OLD = NJ * 16 + 4;
    constexpr int JOIN = 4 * 16 * OLD + 4 * 16 * 2;     // words of the waves' sums
    __shared__ __attribute__((aligned(16))) float smem[4 * S::WORDS > JOIN ? 4 * S::WORDS : JOIN];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), grp = lane / 16, l16 = lane % 16;
    const int i = blockIdx.x / kXcds, pair = i / a.c.heads * kXcds + blockIdx.x % kXcds;
    Work w;
    if (!find_work<16, KT>(a, pair / a.nsplit, i % a.c.heads, pair % a.nsplit, w)) return;
    float* const sw = smem + wave * S::WORDS;

    // Q^T operand: slot l16, head_dim 16 j + 4 grp + e for the instruction (j, e)
    float qf[NJ][4];
    const int slot = w.q0 + l16;
    const float* const q = static_cast<const float*>(a.q) + slot_row(a, w, slot) * HD;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (slot < w.slots && j * 16 + grp * 4 < HD) load4<float>(q + j * 16 + grp * 4, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[j][e] = v[e];
    }
    f32x4_t oacc[NJ];
#pragma unroll
    for (int h = 0; h < NJ; ++h) oacc[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    auto multiply = [&](uint64_t present) __attribute__((always_inline)) {
        // S^T: keys 16 ks + 4 grp + r of slot l16, in the log2 domain
        float sc[2][4];
        float mx = -INFINITY;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float k[4] = {0.f, 0.f, 0.f, 0.f};
                if (HD % 16 == 0 || j + 1 < NJ || j * 16 + grp * 4 < HD) load4<float>(sw + (ks * 16 + l16) * P + j * 16 + grp * 4, k);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc = Elt<float>::mma(k[e], qf[j][e], acc);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool there = (present >> (ks * 16 + grp * 4 + r)) & 1;
                sc[ks][r] = there ? acc[r] * a.scale_log2 : -INFINITY;
                mx = fmaxf(mx, sc[ks][r]);
            }
        }
        const float m_new = fmaxf(m_run, rows_max(mx));
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float corr = m_run == -INFINITY ? 0.f : fast_exp2(m_run - ref);
        m_run = m_new;
        l_run *= corr;
#pragma unroll
        for (int h = 0; h < NJ; ++h) oacc[h] *= corr;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[ks][r] = fast_exp2(sc[ks][r] - ref);
                l_run += sc[ks][r];
            }
        // O^T += V^T P^T; a last block of eight columns multiplies what lies behind the row too, into rows that are not used
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int h = 0; h < NJ; ++h)
                    oacc[h] = Elt<float>::mma(sw[(KT + ks * 16 + grp * 4 + r) * P + h * 16 + l16], sc[ks][r], oacc[h]);
    };
    auto run = [&](auto st, int from, int to, int skip) __attribute__((always_inline)) {
        from += (wave - skip) & 3;   // the waves go on in turn from one kind to the next
        if (from >= to) return;
        st.init(a, w, lane);
        st.fetch_index(from);
        st.issue(a, w, from, to);
        st.fetch_index(from + 4);
        uint64_t present = st.valid;
        st.store(sw);
        st.issue(a, w, from + 4, to);
        st.fetch_index(from + 8);
        for (int t = from; t < to; t += 4) {
            wait_lds();
            __builtin_amdgcn_wave_barrier();
            multiply(present);
            asm volatile("" ::: "memory");
            present = st.valid;
            st.store(sw);
            st.issue(a, w, t + 8, to);
            st.fetch_index(t + 12);
        }
    };
    const int c0 = min(w.t0, w.ntc), c1 = min(w.t1, w.ntc);
    run(S{}, c0, c1, 0);
    if (w.r.nf > 0) run(StagerF32<HD, true>{}, max(w.t0 - w.ntc, 0), max(w.t1 - w.ntc, 0), c1 - c0);

    const float l = rows_sum(l_run);
    __syncthreads();
    float* const so = smem;
    float2* const sml = reinterpret_cast<float2*>(so + 4 * 16 * OLD);
#pragma unroll
    for (int h = 0; h < NJ; ++h) {
        const float v[4] = {oacc[h][0], oacc[h][1], oacc[h][2], oacc[h][3]};
        store4<float>(so + (wave * 16 + l16) * OLD + h * 16 + grp * 4, v);
    }
    if (grp == 0) sml[wave * 16 + l16] = make_float2(m_run, l);
    __syncthreads();
    join_waves<float, HD, OLD>(a, w, so, sml, tid, w.q0 + tid / 16);
}

// Join of the key ranges: range s has the weight l_s 2^(m_s - m); rows of no
// segment are left alone, rows of no key get 0. One wave per (row, head): lane s
// holds range s's maximum and sum, then hd / 4 lanes take four columns each and as
// many groups of them as the wave holds take the ranges in turn, so that a row
// costs two rounds of loads however many ranges there are.
constexpr int kMaxRanges = 64;
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(Kv8AttnDesc a) {
    const int HG = a.c.heads * a.group, hd = a.c.hd, lane = threadIdx.x % kWave;
    const int lo = min(max(a.seg_start[0], 0), a.M), hi = min(max(a.seg_start[a.nseg], 0), a.M);
    const long plane = (long)a.M * HG;
    const long sr = (long)lo * HG + (long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;   // (row, head)
    if (sr >= (long)hi * HG) return;
    const int CL = hd / 4, groups = kWave / CL, grp = lane / CL, col = lane % CL;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < a.nsplit) ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (lane * plane + sr));
    const float m = wave_max(ml.x);
    const float f = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m) * ml.y;
    const float L = wave_sum(f);
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    const float* const po = a.part_o + sr * hd + col * 4;
#pragma unroll 8
    for (int s0 = 0; s0 < a.nsplit; s0 += groups) {
        const int s = s0 + grp;
        const float fs = __shfl(f, s, kWave);
        if (grp < groups && s < a.nsplit) {
            const float4 p = *reinterpret_cast<const float4*>(po + s * plane * hd);
            acc[0] += fs * p.x; acc[1] += fs * p.y; acc[2] += fs * p.z; acc[3] += fs * p.w;
        }
    }
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < groups; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] += __shfl(acc[r], (g * CL + col) % kWave, kWave);
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] *= inv;
    if (lane < CL) store4<T>(static_cast<T*>(a.o) + sr * hd + col * 4, o);
}

// Slot tiles, the segments' last ones counted as full.
int slot_tiles(const Kv8AttnDesc& a, int tile) {
    return (int)std::min<long>((long)a.M * a.group / tile + a.nseg, (long)a.M * a.group);
}

// Whether a split into n ranges stays below the 2^32 threads that end a launch: the attention's
// (its pairs of tile and range rounded up to the XCDs) and the join's, a wave per row and head.
bool ranges_fit(const Kv8AttnDesc& a, int tile, int n) {
    constexpr long most = (1l << 32) / kThreads;
    return ((long)slot_tiles(a, tile) * n + kXcds) * a.c.heads < most &&
           (long)a.M * a.c.heads * a.group / (kThreads / kWave) + 1 < most;
}

template <int QT>
void launch_bf16(const Kv8AttnDesc& a, hipStream_t s) {
    const int qtiles = slot_tiles(a, QT);
    const int pairs = qtiles * a.nsplit;
    const dim3 grid((unsigned)(QT == 128 ? pairs : (pairs + kXcds - 1) / kXcds * kXcds) * a.c.heads), block(kThreads);
    switch (a.c.hd) {
#define MS_HD(n) case n: hipLaunchKernelGGL((attend_bf16_kernel<n, QT>), grid, block, 0, s, a, qtiles); break;
        MS_HD(8) MS_HD(16) MS_HD(24) MS_HD(32) MS_HD(40) MS_HD(48) MS_HD(56) MS_HD(64)
        MS_HD(72) MS_HD(80) MS_HD(88) MS_HD(96) MS_HD(104) MS_HD(112) MS_HD(120) MS_HD(128)
#undef MS_HD
    }
}

void launch_f32(const Kv8AttnDesc& a, hipStream_t s) {
    const int qtiles = slot_tiles(a, 16);
    const int pairs = qtiles * a.nsplit;
    const dim3 grid((unsigned)(pairs + kXcds - 1) / kXcds * kXcds * a.c.heads), block(kThreads);
    switch (a.c.hd) {
#define MS_HD(n) case n: hipLaunchKernelGGL(attend_f32_kernel<n>, grid, block, 0, s, a); break;
        MS_HD(8) MS_HD(16) MS_HD(24) MS_HD(32) MS_HD(40) MS_HD(48) MS_HD(56) MS_HD(64)
#undef MS_HD
    }
}

}  // namespace

// Query slots per workgroup and key ranges: the pair with the least modelled time, from the
// segments' mean length (how many slot tiles ragged segments fill: half a tile more each than
// rows / tile). `base` workgroups per range of `steps` key steps; up to the `most` that a CU
// holds run at once, k on the fullest one.
//  16 and 32 slots (waves with key tiles of their own): a step is 128 keys and takes 0.0015 +
//   0.009 k us per column of head_dim, a quarter more where rows are not whole 16-byte
//   chunks, whatever the slots: staging bounds it. float32: 0.016 k, its matrix instructions.
//  128 slots: a step is 64 keys; k workgroups take the tile's matrix instructions times
//   (0.014 + 0.010 k) us together, and a longer start and end.
//  No less than the codes' bytes at 4.5 TB/s. More than one range: the join's launch, and the
//  parts written and read.
// Fitted to 5159 measured times (16 shapes of 1 to 64 requests of 500 to 16000 keys, head_dim 32 to
// 128, 1 to 1600 rows, equal and ragged, every form, 1 to 64 ranges): the chosen pair takes 1.05
// times the fastest on average, 1.40 times at most (profiles/kv8_attention_plan_times.txt). In us at the best count of ranges, 16 / 32 / 128 slots: 8 requests
// over 4096 keys of 16 heads of 64, 16 rows each 22 / 23 / 29, 32 rows 29 / 24 / 33, 64 rows 47 / 33 /
// 37, 128 rows - / 52 / 46; 4 over 24 heads of 128, 32 rows 43 / 32 / 42, 96 rows - / 69 / 55; one of
// 128 rows over 1024 keys of 12 heads of 64 - / 12 / 14. Ranges: 8 x 16 rows of 16 heads of 72
// in 1 / 2 / 4 / 8 / 16 take 40 / 28 / 25 / 31 / 36, one row of 12 heads of 64 25 in one and 10 in 12;
// 8 x 123 to 2458 rows of 16 heads of 72 in 1 / 2 / 3 232 / 253 / 257.
void plan_kv8_attention(int dtype, Kv8AttnDesc& a, long keys) {
    a.tile = 16;
    a.nsplit = 1;
    if (a.M == 0) return;
    const int heads = a.c.heads, hd = a.c.hd;
    const long rows = (long)a.M * a.group, segs = std::min(a.nseg, a.M), per = (rows + segs - 1) / segs;
    const double mfmas = 8 * ((hd + 31) / 32) + 4 * ((hd + 15) / 16 + (hd % 16 == 0));
    const double bytes = 2.0 * segs * keys * heads * hd / 4.5e6;
    double least = 1e30;
    for (int tile : {16, 32, 128}) {
        if (tile > 16 && (dtype != kBF16 || per <= tile / 4)) break;
        const double tiles = segs == 1 ? (double)((per + tile - 1) / tile) : segs * std::max(1.0, (double)(per - 1) / tile + 0.5);
        const double base = tiles * heads;
        const long steps = std::max(1l, tile == 128 ? (keys + 63) / 64 : (keys + 127) / 128);
        const int most = tile == 128 ? shared_per_cu(hd) : dtype == kBF16 ? few_per_cu(hd, tile) : 2;
        for (int n : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (n > steps || n > kMaxRanges || (n > 1 && !ranges_fit(a, tile, n))) break;
            const double groups = base * n, slots = 256.0 * most, k = std::min(std::ceil(groups / 256), (double)most);
            const double step = tile == 128 ? mfmas * (0.014 + 0.010 * k)
                : dtype != kBF16 ? k * hd * 0.016 : (hd * (hd % 16 ? 1.25 : 1.0) + 2) * (0.0015 + 0.009 * k);
            const double round = (steps + n - 1) / n * step;    // as many as run at once
            double us = (tile == 128 ? 10.5 : 7.3) + std::max(bytes, groups > slots ? round * (groups / slots + 0.25) : round);
            if (n > 1) us += 2.6 + (8.0 * n + 2) * rows * heads * hd / 2.7e6;
            if (us < least) {
                least = us;
                a.tile = tile;
                a.nsplit = n;
            }
        }
    }
}

hipError_t launch_kv8_attention(int dtype, const Kv8AttnDesc& a, hipStream_t s) {
    if (a.M == 0) return hipSuccess;
    if (dtype == kBF16) {
        if (a.tile == 16) launch_bf16<16>(a, s);
        else if (a.tile == 32) launch_bf16<32>(a, s);
        else launch_bf16<128>(a, s);
    } else {
        launch_f32(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_kv8_join(int dtype, const Kv8AttnDesc& a, hipStream_t s) {
    if (a.M == 0 || a.nsplit == 1) return hipSuccess;
    const long n = (long)a.M * a.c.heads * a.group;
    const dim3 grid((unsigned)((n + kThreads / kWave - 1) / (kThreads / kWave))), block(kThreads);
    if (dtype == kBF16) hipLaunchKernelGGL(join_kernel<bf16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(join_kernel<float>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace ms
