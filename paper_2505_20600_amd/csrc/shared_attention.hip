// Attention of a batch whose requests share a long prefix: packed query rows over
// one prefix's K/V rows, less the tokens that the row's request hides, and over
// the request's own K/V rows, one softmax over both. A row without any key is 0.
//
// A query slot is a (packed row, query head of one K/V head's group) pair. Slots of
// all requests stand in one row and are cut into tiles that go across requests, so
// that a prefix tile is fetched and multiplied once for as many slots as a tile
// has, however few rows each request brings. What a request does not see is a
// matter of each score: every lane has the hidden tokens of its slot's request as one
// word per key tile. Own rows lie behind each other in the order of the requests; a
// slot tile walks over those of its first to its last request, and a slot sees its
// own request's.
//
// Tiles of K and V rows land in LDS by direct loads. The products run in the layout
// of attention.hip: S^T = K Q^T leaves the weights in the operand layout of O^T =
// V^T P^T, V is read transposed by ds_read_b64_tr_b16, rows of ones in V^T give the
// denominator. Scores, maxima, sums and the parts of key ranges are float32. bf16
// rounds twice: the weights, the matrix cores' operand of the second product (numerator
// and denominator take the same rounded ones), and the output.
//
// A hidden key's weight is 0, and 0 times an infinity or NaN in its V row is NaN: a
// slot whose result is not finite is computed again over the keys that it sees, one
// wave at a slot (recompute). So is one whose sums of finite values, the weights above 1 and not yet divided by their own
// sum, leave float32: the second computation and the join keep weights that sum to at most 1.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_tiles.h"
#include "kernels.h"
#include "shared_attention.h"

namespace ms {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// A workgroup's query slots and key tiles.
struct Work {
    int row0;       // first packed row of all
    int slots;      // slots in all
    int q0;         // first slot of this tile
    int kvh;        // K/V head
    int split;
    int t0, t1;     // key tiles: those of the prefix, then the own ones
    int ntp;        // prefix tiles
    int first, last;    // requests of the tile
    int f0, f1;     // their own rows
};

// The tables of a workgroup's requests in LDS: where each one's rows start, and its own rows.
struct Tables {
    int32_t row[kSharedMaxBatch + 1];
    int32_t own[kSharedMaxBatch + 1];
};

// Request of packed row r: the last one of [lo, hi) that starts at or before it, lo where none does (any of them where starts do
// not ascend).
__device__ __forceinline__ int request_of(const Tables& t, int r, int lo, int hi) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.row[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same of all requests, a lane to two of them, for a row that the whole wave asks for.
__device__ __forceinline__ int request_of_all(const SharedAttnDesc& a, const Tables& t, int r) {
    static_assert(kSharedMaxBatch == 2 * kWave, "requests");
    if (a.batch == 1) return 0;
    const int lane = threadIdx.x % kWave;
    const uint64_t lower = __ballot(lane < a.batch && t.row[lane] <= r);
    const uint64_t upper = a.batch > kWave ? __ballot(lane + kWave < a.batch && t.row[lane + kWave] <= r) : 0ull;
    return upper ? 2 * kWave - 1 - __builtin_clzll(upper) : lower ? kWave - 1 - __builtin_clzll(lower) : 0;
}

// Row index of a query slot's (row, query head) in [M][n_heads].
__device__ __forceinline__ long slot_row(const SharedAttnDesc& a, const Work& w, int slot) {
    const int HG = a.heads * a.group;
    const int r = a.group == 1 ? slot : slot / a.group;
    return (long)(w.row0 + r) * HG + w.kvh * a.group + (slot - r * a.group);
}

// Fills the tables and the workgroup's work; false where it has no slot. A barrier for the whole workgroup.
template <int QT, int KT>
__device__ __forceinline__ bool find_work(const SharedAttnDesc& a, int tile, int kvh, int split, Tables& t, Work& w) {
    for (int i = threadIdx.x; i <= a.batch; i += kThreads) {
        t.row[i] = a.seg_start ? min(max(a.seg_start[i], 0), a.M) : i == 0 ? 0 : a.M;
        t.own[i] = a.fresh ? min(max(a.fresh_start[i], 0), a.fresh_rows) : 0;
    }
    __syncthreads();
    w.row0 = uniform(t.row[0]);
    w.slots = uniform(max(t.row[a.batch] - w.row0, 0)) * a.group;
    w.q0 = tile * QT;
    w.kvh = kvh;
    w.split = split;
    if (w.q0 >= w.slots) return false;
    w.first = uniform(request_of_all(a, t, w.row0 + w.q0 / a.group));
    w.last = max(uniform(request_of_all(a, t, w.row0 + (min(w.q0 + QT, w.slots) - 1) / a.group)), w.first);
    w.f0 = uniform(t.own[w.first]);
    w.f1 = max(uniform(t.own[w.last + 1]), w.f0);
    w.ntp = (a.T + KT - 1) / KT;
    const uint32_t nt = w.ntp + (w.f1 - w.f0 + KT - 1) / KT;    // below 2^24; times 32 ranges below 2^32
    w.t0 = uniform((int)(nt * split / a.nsplit));
    w.t1 = uniform((int)(nt * (split + 1) / a.nsplit));
    return true;
}

// KT low bits: those of the positions below n.
template <int KT>
__device__ __forceinline__ uint64_t below(int n) {
    return n >= KT ? (KT == 64 ? ~0ull : (1ull << (KT % 64)) - 1) : n <= 0 ? 0ull : (1ull << n) - 1;
}

// x where bit `at` of w is set, else -infinity, without a condition register per score.
__device__ __forceinline__ float seen_or_none(uint32_t w, int at, float x) {
    const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)w, at, 1);
    return __uint_as_float((__float_as_uint(x) & m) | (0xff800000u & ~m));
}

// Which keys of the tiles one slot sees.
template <int KT>
struct Sight {
    uint32_t at;                // byte offset of its request's hidden tokens in the table
    int lo, hi;                 // its request's own rows
    __device__ __forceinline__ void init(const SharedAttnDesc& a, const Tables& t, const Work& w, int slot) {
        const int s = min(slot, w.slots - 1);
        const int b = request_of(t, w.row0 + s / a.group, w.first, w.last + 1);
        at = (uint32_t)b * a.words * 8u;
        lo = t.own[b];
        hi = max(t.own[b + 1], lo);
    }
    // hidden ones among prefix tile t's keys, as loaded; `table`: the bits, without an entry where none is hidden
    __device__ __forceinline__ uint64_t fetch(__amdgpu_buffer_rsrc_t table, int t) const {
        if constexpr (KT == 64) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(table, (int)at + t * 8, 0, 0);
            return (uint64_t)v[1] << 32 | v[0];
        } else {
            return __builtin_amdgcn_raw_buffer_load_b32(table, (int)at + t * 4, 0, 0);
        }
    }
    __device__ __forceinline__ uint64_t prefix(const SharedAttnDesc& a, uint64_t hidden, int t) const {
        return ~hidden & below<KT>(a.T - t * KT);
    }
    // of the own tile of rows k0 on
    __device__ __forceinline__ uint64_t own(int k0) const { return below<KT>(hi - k0) & ~below<KT>(lo - k0); }
};

// The hidden tokens' words; reads past the last word, or without a table, are zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t hidden_table(const SharedAttnDesc& a) {
    return make_rsrc(a.bits, a.bits ? (uint32_t)a.batch * a.words * 8u : 0u);
}

// One slot's result over the keys [t0, t1) that it sees, by a wave: 64 keys at a time, a
// lane's key's score, then the lanes as columns of the weighted mean so far (not a sum: the mean of finite values is finite).
template <typename T, int KT>
__device__ __forceinline__ void recompute(const SharedAttnDesc& a, const Work& w, const Tables& t, int slot) {
    const int lane = threadIdx.x % kWave, hd = a.hd, dkv = a.heads * hd;
    Sight<64> sight;
    sight.init(a, t, w, slot);
    const long at = slot_row(a, w, slot);
    const T* const q = static_cast<const T*>(a.q) + at * hd;
    float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
    for (int part = 0; part < 2; ++part) {
        const T* const kv = static_cast<const T*>(part ? a.fresh : a.kv) + w.kvh * hd;
        const int k0 = part ? max(w.f0 + (w.t0 - w.ntp) * KT, sight.lo) : w.t0 * KT;
        const int k1 = part ? min(w.f0 + (w.t1 - w.ntp) * KT, sight.hi) : min(min(w.t1, w.ntp) * KT, a.T);
        for (int k = k0; k < k1; k += kWave) {
            const int key = k + lane;
            bool sees = key < k1;
            if (sees && !part && a.bits) sees = !((a.bits[sight.at / 8 + key / 64] >> (key % 64)) & 1);
            float s = -INFINITY;
            if (sees) {
                const T* const row = kv + (long)key * 2 * dkv;
                float dot = 0.f;
                for (int c = 0; c < hd; ++c) dot = fmaf(Elt<T>::to_f32(q[c]), Elt<T>::to_f32(row[c]), dot);
                s = dot * a.scale_log2;
            }
            const uint64_t seen = __ballot(sees);
            const uint64_t nan = __ballot(s != s);
            float up = fmaxf(m, wave_max(s));
            if (nan) up = __uint_as_float(0x7fc00000u);         // maxima drop NaN
            const float ref = up == -INFINITY ? 0.f : up;
            const float corr = m == -INFINITY ? 0.f : fast_exp2(m - ref);
            const float p = sees ? fast_exp2(s - ref) : 0.f;
            m = up;
            const float before = l * corr;
            l = before + wave_sum(p);
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            o[0] *= before * inv;
            o[1] *= before * inv;
            for (int j = 0; j < kWave; ++j) {
                if (!((seen >> j) & 1)) continue;
                const float pj = __shfl(p, j, kWave) * inv;
                const T* const row = kv + (long)(k + j) * 2 * dkv + dkv;
                if (lane < hd) o[0] = fmaf(pj, Elt<T>::to_f32(row[lane]), o[0]);
                if (lane + kWave < hd) o[1] = fmaf(pj, Elt<T>::to_f32(row[lane + kWave]), o[1]);
            }
        }
    }
    const long part = (long)w.split * a.M * a.heads * a.group + at;
    for (int i = 0; i < 2; ++i) {
        const int c = lane + i * kWave;
        if (c >= hd) continue;
        if (a.nsplit == 1) static_cast<T*>(a.o)[at * hd + c] = Elt<T>::from_f32(o[i]);
        else a.part_o[part * hd + c] = o[i];
    }
    if (a.nsplit > 1 && lane == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * part) = make_float2(m, l);
}

// The flagged slots of a tile again, the waves in turn; `bad` [QT / 32] in LDS, complete.
template <typename T, int QT, int KT>
__device__ __forceinline__ void recompute_bad(const SharedAttnDesc& a, const Work& w, const Tables& t, const uint32_t* bad, int wave) {
    for (int i = 0; i < (QT + 31) / 32; ++i) {
        const uint32_t b = uniform((int)bad[i]);
        if (!b) continue;
        for (int s = wave; s < 32; s += kThreads / kWave)
            if ((b >> s) & 1) recompute<T, KT>(a, w, t, w.q0 + i * 32 + s);
    }
}

// The four waves' sums of 16 slots, from slot `first` of the tile on, each relative to its own maximum (so
// [wave][slot][OLD] and sml [wave][slot]), to the output or the key range's part; slots without a finite result are flagged and left: the output may be the
// queries, which the second computation reads.
template <typename T, int HD, int OLD>
__device__ __forceinline__ void join_waves(const SharedAttnDesc& a, const Work& w, const float* so, const float2* sml, int tid,
                                           int first, uint32_t* bad) {
    const int s = tid / 16, slot = w.q0 + first + s;
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
    bool fine = finite(sum);
    const long row = slot_row(a, w, slot), part = (long)w.split * a.M * a.heads * a.group + row;
    constexpr int NC = (HD + 63) / 64;
    const int c0 = tid % 16 * 4;
    float o[NC][4];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = c0 + i * 64;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[i][r] = 0.f;
        if (c >= HD) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float4 x = *reinterpret_cast<const float4*>(so + (v * 16 + s) * OLD + c);
            o[i][0] += f[v] * x.x; o[i][1] += f[v] * x.y; o[i][2] += f[v] * x.z; o[i][3] += f[v] * x.w;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            fine = fine && finite(o[i][r]);
            o[i][r] *= inv;
        }
    }
    // of the 16 lanes that have the slot
    if (__ballot(!fine) >> (tid % kWave / 16 * 16) & 0xffff) {
        if (tid % 16 == 0) atomicOr(bad, 1u << (first + s));
        return;
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = c0 + i * 64;
        if (c >= HD) continue;
        if (a.nsplit == 1) store4<T>(static_cast<T*>(a.o) + row * HD + c, o[i]);
        else store4<float>(a.part_o + part * HD + c, o[i]);
    }
    if (a.nsplit > 1 && tid % 16 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * part) = make_float2(m, sum);
}

// Tiles of KT K rows and as many V rows by direct-to-LDS loads of NW waves, K and V apart.
template <int HD, int KT, int NW>
struct Tiles {
    static constexpr int ROWB = HD * 2, TILEB = KT * ROWB, PAD = 64;
    static constexpr int NQ = (TILEB + 1023) / 1024;        // 1 KB copies of the K or V rows, the last may be half of one
    static constexpr int IPW = (NQ + NW - 1) / NW;          // per wave, most
    static constexpr int PARTB = TILEB;
    static_assert(TILEB % 512 == 0, "tile copies");
    static constexpr bool SWZ = ROWB == 128 || ROWB == 256 || ROWB % 128 == 64;
    static constexpr uint32_t kAbsent = 0xfff00000u;
    uint32_t row_bytes, vk[IPW], vv[IPW];
    int rl[IPW];

    __device__ __forceinline__ void init(int heads, int kvh, int wave, int lane) {
        row_bytes = 4u * heads * HD;
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int pos = min(i * NW + wave, NQ - 1) * 1024 + lane * 16, r = pos / ROWB;
            rl[i] = r;
            const uint32_t row = (uint32_t)r * row_bytes + kvh * ROWB, c = pos % ROWB / 16;
            vk[i] = row + (c ^ k_swz<ROWB>(r)) * 16;
            vv[i] = row + row_bytes / 2 + (c ^ v_swz<ROWB>(r)) * 16;
        }
    }
    // K (or V) rows k0 on, of `end` in all, to LDS address `lds`; rows past the last read as zeros
    __device__ __forceinline__ void issue(u32x4_t rsrc, const uint32_t (&off)[IPW], int k0, int end, int wave, uint32_t lds) {
        const uint32_t base = (uint32_t)k0 * row_bytes;
        const bool whole = k0 + KT <= end;
#pragma unroll
        for (int i = 0; i < IPW; ++i) {
            const int q = i * NW + wave;
            if (NQ % NW != 0 && q >= NQ) continue;
            if (TILEB % 1024 != 0 && q == NQ - 1) {     // half a copy
                if (threadIdx.x % kWave < 32) dma_buf16(rsrc, whole || k0 + rl[i] < end ? off[i] + base : kAbsent, 0, lds + (uint32_t)q * 1024u);
            } else if (whole) {
                dma_buf16(rsrc, off[i], base, lds + (uint32_t)q * 1024u);
            } else {
                dma_buf16(rsrc, k0 + rl[i] < end ? off[i] + base : kAbsent, 0, lds + (uint32_t)q * 1024u);
            }
        }
    }
};

// The prefix tiles of 64 tokens that some request of the workgroup sees, 64 tiles at a time: every wave finds the same. A
// request that hides 30% of the tokens as one region skips as many tiles (453 us without hidden tokens, 397 with, above).
struct Live {
    static constexpr int kMost = 8;     // requests
    uint64_t seen;
    int base, to;
    bool some;      // whether tiles are left out at all
    __device__ __forceinline__ void look(const SharedAttnDesc& a, const Work& w, int lane) {
        const int t = base + lane;
        uint64_t v[kMost];      // all on their way at once
#pragma unroll
        for (int i = 0; i < kMost; ++i) v[i] = a.bits[(long)min(w.first + i, w.last) * a.words + min(t, a.words - 1)];
        uint64_t hidden = ~0ull;
#pragma unroll
        for (int i = 0; i < kMost; ++i) hidden &= v[i];
        seen = __ballot(t < to && hidden != ~0ull);
    }
    // of tiles [from, to); a few tiles, or those of many requests, are all taken
    __device__ __forceinline__ void init(const SharedAttnDesc& a, const Work& w, int lane, int from, int end) {
        base = from;
        to = end;
        some = a.bits && end - from >= 8 && w.last - w.first < kMost;
        if (some) look(a, w, lane);
    }
    // the first tile from t on, `to` where there is none
    __device__ __forceinline__ int next(const SharedAttnDesc& a, const Work& w, int lane, int t) {
        if (!some) return t;
        while (t < to) {
            if (t >= base + kWave) {
                base = t;
                look(a, w, lane);
            }
            const uint64_t m = seen >> (t - base);
            if (m) return t + __builtin_ctzll(m);
            t = base + kWave;
        }
        return to;
    }
};

template <int HD, int QT_>
struct Cfg {
    static constexpr int QT = QT_;
    static constexpr bool WIDE = QT == 128;             // waves have slots of their own and share the key tiles
    static constexpr int KT = WIDE ? 64 : 32;
    static constexpr int NQB = QT == 16 ? 1 : 2;        // 16-slot blocks per wave
    static constexpr int NW = WIDE ? 4 : 1;             // waves that load a tile
    using S = Tiles<HD, KT, NW>;
    static constexpr int NKS = KT / 16;
    static constexpr int NK32 = (HD + 31) / 32;
    static constexpr bool KTAIL = HD % 32 != 0;
    static constexpr bool SUM_IN_PAD = HD % 16 != 0;
    static constexpr int NREAL = (HD + 15) / 16;
    static constexpr int NHS = NREAL + (SUM_IN_PAD ? 0 : 1);
    static constexpr int OLD = HD + 4;
    static constexpr int STAGES = 2;
    static constexpr int V0 = STAGES * S::PARTB;            // a wave's (or the workgroup's) stages: K parts, then V parts, then zeros
    static constexpr int ZERO = 2 * STAGES * S::PARTB, RINGB = ZERO + S::PAD;
    static constexpr int TILES = (WIDE ? 1 : 4) * RINGB;
    static constexpr int JOIN = WIDE ? 4 * 32 * 2 * S::ROWB : (4 * 16 * OLD + 4 * 16 * 2) * 4;
    static constexpr int LDSB = ((TILES > JOIN ? TILES : JOIN) + 63) / 64 * 64;
};

constexpr int wide_per_cu(int hd) { return hd <= 32 ? 4 : hd <= 80 ? 3 : 2; }
constexpr int few_per_cu(int hd) { return hd <= 32 ? 4 : hd <= 48 ? 3 : hd <= 72 ? 2 : 1; }

// bf16. WIDE: 128 slots, 32 per wave; the four waves share 64-key tiles in two stages.
// Not WIDE: 16 or 32 slots, all of them in every wave, and every wave has 32-key tiles of its own (tile
// t0 + wave + 4 i) in two stages of its own, without a barrier; the four partial results are joined at the end.
// What bounds the wide form is each wave's softmax between its products (matrix cores busy 48% at head_dim 128, vector
// instructions as long): 8 requests of 1229 rows over 4096 tokens of 16 heads of 128 take 397 us (0.83 PFLOP/s of what is seen),
// 453 without hidden tokens (0.95), of 72 columns 309, of 64 258. Products of the next tile started under this one's softmax
// gained nothing (more registers, as many waits). Few slots are bound by a chain of loads, products and exponentials on
// few workgroups: 8 rows over 4096 tokens of 12 heads of 64 7.1 us, and the join 3.2.
template <int HD, int QT>
__global__ __launch_bounds__(kThreads, QT == 128 ? wide_per_cu(HD) : few_per_cu(HD)) void shared_bf16_kernel(SharedAttnDesc a, int qtiles) {
    using C = Cfg<HD, QT>;
    using S = typename C::S;
    constexpr bool WIDE = C::WIDE;
    constexpr int NQB = C::NQB, NKS = C::NKS, KT = C::KT;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[C::LDSB + 16];
    __shared__ Tables tables;
    __shared__ uint32_t bad[QT / 32 + 1];
    const uint32_t lds0 = lds_addr(smem);
    const uint32_t ones_rel = C::LDSB;                  // 8 bytes of bf16 ones (SUM_IN_PAD)
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave);
    const int grp = lane / 16, l16 = lane % 16;
    // WIDE: a head's slot tiles side by side, so that an XCD's L2 serves the head's rows to all of
    // them. Else a (tile, range) pair's heads side by side, which read neighbouring parts of the same rows.
    Work w;
    if constexpr (WIDE) {
        const int lb = xcd_logical_block(blockIdx.x, qtiles * a.nsplit * a.heads);
        if (!find_work<QT, KT>(a, lb % qtiles, lb / (qtiles * a.nsplit), lb / qtiles % a.nsplit, tables, w)) return;
    } else {
        const int i = blockIdx.x / kXcds, pair = i / a.heads * kXcds + blockIdx.x % kXcds;
        if (pair >= qtiles * a.nsplit) return;
        if (!find_work<QT, KT>(a, pair / a.nsplit, i % a.heads, pair % a.nsplit, tables, w)) return;
    }
    constexpr int step = WIDE ? 1 : 4;

    // constant LDS: zeros behind the rings, the ones block
    constexpr int RINGS = WIDE ? 1 : 4;
    if (tid < 4 * RINGS) *reinterpret_cast<uint4*>(smem + (tid / 4) * C::RINGB + C::ZERO + (tid % 4) * 16) = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 4 * RINGS) *reinterpret_cast<uint2*>(smem + C::LDSB) = make_uint2(0x3f803f80u, 0x3f803f80u);
    if (tid < QT / 32 + 1) bad[tid] = 0;

    // Q^T fragments (B operand), their sign that of the score scale
    bf16x8_t qf[NQB][C::NK32];
    Sight<KT> sight[NQB];
    const __amdgpu_buffer_rsrc_t table = hidden_table(a);
    const bf16_t* __restrict__ q = static_cast<const bf16_t*>(a.q);
    const int wq0 = w.q0 + (WIDE ? wave * 32 : 0);
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        const int slot = wq0 + qb * 16 + l16;
        const bf16_t* qp = q + slot_row(a, w, slot) * HD;
        sight[qb].init(a, tables, w, slot);
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
    // last QK step of a head_dim that is not a multiple of 32: lanes whose columns lie past the row read zeros
    static_assert(!C::KTAIL || !S::SWZ, "tail offsets");
    const bool in_row = (C::NK32 - 1) * 64 + grp * 16 < S::ROWB;
    const int rowA = 4 * grp + (l16 >> 2);
    const int fV = v_swz<S::ROWB>(rowA);
    uint32_t voffh[C::NREAL];
#pragma unroll
    for (int h = 0; h < C::NREAL; ++h) {
        const int hd = 16 * h + 4 * (l16 & 3);
        voffh[h] = rowA * S::ROWB + (((hd / 8) ^ fV) * 16) + (hd % 8) * 2;
    }
    const bool ones_lane = C::SUM_IN_PAD && (16 * (C::NREAL - 1) + 4 * (l16 & 3)) >= HD;

    f32x4_t oacc[NQB][C::NHS];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
        for (int h = 0; h < C::NHS; ++h) oacc[qb][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // scores are as multiplied, weights 2^(cs score + neg): neg is minus cs times the running maximum
    const float cs = fabsf(a.scale_log2), rescale_at = fminf(kRescaleLog2 / cs, 3.4e38f);    // finite for the smallest scales too
    float m_run[NQB], neg[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        m_run[qb] = -INFINITY;
        neg[qb] = 0.f;
    }
    const bf16x8_t onesf = __builtin_bit_cast(bf16x8_t, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
    constexpr uint64_t kAll = KT == 64 ? ~0ull : (1ull << (KT % 64)) - 1;

    const uint32_t ring = WIDE ? 0u : (uint32_t)(wave * C::RINGB);
    const uint32_t zero = ring + C::ZERO;
    // K fragment (16 keys, 32 columns) of the tile at `base`
    auto k_frag = [&](uint32_t base, int ks, int kc) {
        uint32_t at = base + koff[kc] + ks * 16 * S::ROWB;
        if (C::KTAIL && kc == C::NK32 - 1) at = in_row ? at : zero;
        return *reinterpret_cast<const bf16x8_t*>(smem + at);
    };
    auto qk = [&](uint32_t base, f32x4_t (&sacc)[NQB][NKS]) {
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int kc = 0; kc < C::NK32; ++kc) {
                const bf16x8_t kf = k_frag(base, ks, kc);
#pragma unroll
                for (int qb = 0; qb < NQB; ++qb) sacc[qb][ks] = mfma32(kf, qf[qb][kc], kc == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : sacc[qb][ks]);
            }
    };
    // scores of keys that a slot does not see become -infinity, whatever they were
    auto hide = [&](const uint64_t (&sees)[NQB], f32x4_t (&sacc)[NQB][NKS]) {
        bool all = true;
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) all = all && sees[qb] == kAll;
        if (__all(all)) return;
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            const uint64_t mine = sees[qb] >> (grp * 4);
            uint32_t half[2] = {(uint32_t)mine, (uint32_t)(mine >> 32)};
            asm volatile("" : "+v"(half[0]), "+v"(half[1]));    // what follows stays behind the branch
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                for (int r = 0; r < 4; ++r) sacc[qb][ks][r] = seen_or_none(half[ks / 2], ks % 2 * 16 + r, sacc[qb][ks][r]);
        }
    };
    // online softmax: running maxima and accumulators updated, a rescale only where a score exceeds its slot's
    // maximum by more than 2^8
    auto raise = [&](const f32x4_t (&sacc)[NQB][NKS]) {
        float mx[NQB];
        bool above = false;
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            mx[qb] = sacc[qb][0][0];
#pragma unroll
            for (int i = 1; i < 4 * NKS; ++i) mx[qb] = fmaxf(mx[qb], sacc[qb][i / 4][i % 4]);
            above = above || mx[qb] > m_run[qb] + rescale_at;
        }
        if (__any(above)) {
#pragma unroll
            for (int qb = 0; qb < NQB; ++qb) {
                const float up = fmaxf(m_run[qb], rows_max(mx[qb]));
                const float corr = m_run[qb] == -INFINITY ? 0.f : fast_exp2((m_run[qb] - up) * cs);
#pragma unroll
                for (int h = 0; h < C::NHS; ++h) oacc[qb][h] *= corr;
                m_run[qb] = up;
                // a maximum beyond float32 after scaling is infinite, and so its row NaN
                neg[qb] = up == -INFINITY ? 0.f : up * cs == INFINITY ? __uint_as_float(0x7fc00000u) : -up * cs;
            }
        }
    };
    auto weights = [&](f32x4_t (&sacc)[NQB][NKS]) {
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                for (int r = 0; r < 4; ++r) sacc[qb][ks][r] = fast_exp2(fmaf(sacc[qb][ks][r], cs, neg[qb]));
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
        for (int c = 0; c < KT / 32; ++c) {
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

    const bool active = wq0 < w.slots;
    __syncthreads();   // constant LDS
    f32x4_t sa[NQB][NKS];
    // Tiles [from, to) of one kind (tile 0 at row `base` of kv, which has `rows`): while a tile is multiplied the next one lands.
    auto run = [&](auto OWN, const void* kv, int base, int rows, int from, int to, int skip) __attribute__((always_inline)) {
        if constexpr (!WIDE) from += (wave - skip) & 3;     // the waves go on in turn from one kind to the next
        if (from >= to) return;     // the whole workgroup, or a wave that waits for no other
        Live live;
        auto after = [&](int t) {
            if constexpr (WIDE && !OWN) return live.next(a, w, lane, t);
            else return t;
        };
        if constexpr (WIDE && !OWN) {
            live.init(a, w, lane, from, to);
            from = after(from);
            if (from >= to) return;
        }
        const int lw = WIDE ? wave : 0;
        const u32x4_t rsrc = raw_rsrc(kv, (uint32_t)rows * 4u * a.heads * HD);
        S st;
        st.init(a.heads, w.kvh, lw, lane);
        auto issue = [&](int t, int n) {
            st.issue(rsrc, st.vk, base + t * KT, rows, lw, lds0 + ring + (n & 1) * S::PARTB);
            st.issue(rsrc, st.vv, base + t * KT, rows, lw, lds0 + ring + C::V0 + (n & 1) * S::PARTB);
        };
        uint64_t hidden[NQB];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) hidden[qb] = OWN ? 0ull : sight[qb].fetch(table, from);
        issue(from, 0);
        int n = 0;
        for (int t = from, then; t < to; t = then, ++n) {
            then = after(t + step);
            wait_all();   // tile t has landed, and this wave's reads of the parts refilled below are done
            if constexpr (WIDE) barrier_only();
            else asm volatile("" ::: "memory");
            uint64_t sees[NQB];
#pragma unroll
            for (int qb = 0; qb < NQB; ++qb) {
                sees[qb] = OWN ? sight[qb].own(base + t * KT) : sight[qb].prefix(a, hidden[qb], t);
                asm volatile("" : "+v"(sees[qb]));      // used before the next loads are under way
            }
            if (then < to) {
#pragma unroll
                for (int qb = 0; qb < NQB; ++qb)
                    if constexpr (!OWN) hidden[qb] = sight[qb].fetch(table, then);
                issue(then, n + 1);
            }
            if (WIDE && !active) continue;
            qk(ring + (n & 1) * S::PARTB, sa);
            hide(sees, sa);
            raise(sa);
            weights(sa);
            pv(ring + C::V0 + (n & 1) * S::PARTB, sa);
        }
        wait_all();
        if constexpr (WIDE) barrier_only();   // the parts may be written again
    };
    const int c0 = min(w.t0, w.ntp), c1 = min(w.t1, w.ntp);
    run(std::false_type{}, a.kv, 0, a.T, c0, c1, 0);
    if (w.f1 > w.f0) run(std::true_type{}, a.fresh, w.f0, w.f1, max(w.t0 - w.ntp, 0), max(w.t1 - w.ntp, 0), c1 - c0);

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
    const long range = (long)w.split * a.M * a.heads * a.group;
    __syncthreads();   // every wave is past its last read of the stages
    if constexpr (WIDE) {
        // through LDS: rows of a slot in 16-byte vectors, chunks swizzled by the slot where rows are a power of two
        constexpr int CH = HD / 8, CF = HD / 4;
        constexpr int SWM = (CH & (CH - 1)) == 0 ? (CH >= 16 ? 15 : CH - 1) : 0;
        constexpr int SWF = (CF & (CF - 1)) == 0 ? (CF >= 16 ? 15 : CF - 1) : 0;
        uint8_t* const so = smem + wave * 32 * S::ROWB * (a.nsplit == 1 ? 1 : 2);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            const float inv_l = l[qb] == 0.f ? 0.f : 1.0f / l[qb];
            const int rl = qb * 16 + l16;
            bool fine = finite(l[qb]);
#pragma unroll
            for (int h = 0; h < C::NHS; ++h) {
                const int cidx = h * 16 + grp * 4;
                if (cidx < HD) {
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        fine = fine && finite(oacc[qb][h][r]);
                        v[r] = oacc[qb][h][r] * inv_l;
                    }
                    if (a.nsplit == 1)
                        store4<bf16_t>(reinterpret_cast<bf16_t*>(so + rl * S::ROWB + (((cidx / 8) ^ (rl & SWM)) * 16) + (cidx % 8) * 2), v);
                    else
                        store4<float>(reinterpret_cast<float*>(so + rl * 2 * S::ROWB) + ((cidx / 4) ^ (rl & SWF)) * 4, v);
                }
            }
            const int slot = wq0 + rl;
            if (!fine && slot < w.slots) atomicOr(&bad[wave], 1u << rl);
            if (a.nsplit > 1 && fine && grp == 0 && slot < w.slots)
                *reinterpret_cast<float2*>(a.part_ml + 2 * (range + slot_row(a, w, slot))) = make_float2(m_run[qb] * cs, l[qb]);
        }
        __syncthreads();
        const uint32_t again = bad[wave];       // flagged slots are left: the output may be the queries, which the second computation reads
        if (a.nsplit == 1) {
            for (int k = lane; k < 32 * CH; k += kWave) {
                const int rl = k / CH, c = k % CH;
                if (wq0 + rl < w.slots && !(again >> rl & 1))
                    st16(static_cast<bf16_t*>(a.o) + slot_row(a, w, wq0 + rl) * HD + c * 8,
                         ld16(so + rl * S::ROWB + ((c ^ (rl & SWM)) * 16)));
            }
        } else {
            for (int k = lane; k < 32 * CF; k += kWave) {
                const int rl = k / CF, c = k % CF;
                if (wq0 + rl < w.slots && !(again >> rl & 1))
                    st16(a.part_o + (range + slot_row(a, w, wq0 + rl)) * HD + c * 4,
                         ld16(so + rl * 2 * S::ROWB + ((c ^ (rl & SWF)) * 16)));
            }
        }
    } else {
        // the four waves' sums, each relative to its own maximum, joined through LDS 16 slots at a time
        constexpr int OLD = C::OLD;
        float* const so = reinterpret_cast<float*>(smem);
        float2* const sml = reinterpret_cast<float2*>(so + 4 * 16 * OLD);
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
            join_waves<bf16_t, HD, OLD>(a, w, so, sml, tid, qb * 16, &bad[0]);
        }
    }
    __syncthreads();    // the flags are complete
    recompute_bad<bf16_t, QT, KT>(a, w, tables, bad, wave);
}

// float32: 16 or 32 query slots in every wave, 32-key tiles of its own per wave, staged through registers
// into padded rows, products on the float32 matrix instructions; joined at the end. 8 requests of 1024 rows over 4096 tokens
// of 8 heads of 64 take 785 us, 88 TFLOP/s of the 154 of a large product; 4 of 205 rows over 1024 tokens of 4 heads 27 us (32
// TFLOP/s: 208 workgroups, one wave per SIMD, matrix cores busy 37%; eight waves to a workgroup took 30, and more where there are many tiles).
template <int HD>
struct TilesF32 {
    static constexpr int KT = 32;
    static constexpr int CR = HD / 4;                   // 16-byte chunks per row
    static constexpr int NCH = 2 * KT * CR / kWave;     // chunks per lane
    static_assert(2 * KT * CR % kWave == 0, "whole chunks");
    // words per row: 4 P = 16 or 48 mod 64 keeps the four rows that a transposed V read takes in different banks
    static constexpr int P = HD + 4;
    static constexpr int WORDS = 2 * KT * P + 16;       // reads of a last block of eight columns go past the last row
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t row_bytes, col0;
    int lane, end;
    vec16 raw[NCH];
    __device__ __forceinline__ void init(const void* kv, int rows, int heads, int kvh, int lane_) {
        lane = lane_;
        row_bytes = 8u * heads * HD;
        col0 = kvh * HD * 4;
        rsrc = make_rsrc(kv, (uint32_t)rows * row_bytes);
        end = rows;
    }
    // rows past the last read as zeros
    __device__ __forceinline__ void issue(int k0) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int c = i * kWave + lane, r = c / CR, key = k0 + r % KT;
            const uint32_t o = key < end ? (uint32_t)key * row_bytes + (r >= KT ? row_bytes / 2 : 0u) + col0 + (c % CR) * 16 : 0xfff00000u;
            raw[i] = buf_ld16(rsrc, o, 0);
        }
    }
    __device__ __forceinline__ void store(float* smem) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int c = i * kWave + lane;
            st16(smem + (c / CR) * P + (c % CR) * 4, raw[i]);
        }
    }
};

// One staged tile serves NQB blocks of 16 slots.
template <int HD, int NQB>
__global__ __launch_bounds__(kThreads, 2) void shared_f32_kernel(SharedAttnDesc a, int qtiles) {
    using S = TilesF32<HD>;
    constexpr int KT = S::KT, P = S::P, NJ = (HD + 15) / 16, QT = 16 * NQB;
    constexpr int OLD = NJ * 16 + 4;
    constexpr int JOIN = 4 * 16 * OLD + 4 * 16 * 2;     // words of the waves' sums
    __shared__ __attribute__((aligned(16))) float smem[4 * S::WORDS > JOIN ? 4 * S::WORDS : JOIN];
    __shared__ Tables tables;
    __shared__ uint32_t bad[1];
    const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave), grp = lane / 16, l16 = lane % 16;
    const int i = blockIdx.x / kXcds, pair = i / a.heads * kXcds + blockIdx.x % kXcds;
    Work w;
    if (pair >= qtiles * a.nsplit) return;
    if (!find_work<QT, KT>(a, pair / a.nsplit, i % a.heads, pair % a.nsplit, tables, w)) return;
    if (tid == 0) bad[0] = 0;
    float* const sw = smem + wave * S::WORDS;
    if (lane < 16) sw[2 * KT * P + lane] = 0.f;

    // Q^T operand: slot l16 of a block, head_dim 16 j + 4 grp + e for the instruction (j, e)
    float qf[NQB][NJ][4];
    Sight<KT> sight[NQB];
    const __amdgpu_buffer_rsrc_t table = hidden_table(a);
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        const int slot = w.q0 + qb * 16 + l16;
        sight[qb].init(a, tables, w, slot);
        const float* const q = static_cast<const float*>(a.q) + slot_row(a, w, slot) * HD;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (slot < w.slots && j * 16 + grp * 4 < HD) load4<float>(q + j * 16 + grp * 4, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[qb][j][e] = v[e];
        }
    }
    f32x4_t oacc[NQB][NJ];
    float m_run[NQB], l_run[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
#pragma unroll
        for (int h = 0; h < NJ; ++h) oacc[qb][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m_run[qb] = -INFINITY;
        l_run[qb] = 0.f;
    }

    auto multiply = [&](const uint64_t (&sees)[NQB]) __attribute__((always_inline)) {
        // S^T: keys 16 ks + 4 grp + r of a slot, in the log2 domain
        f32x4_t acc[NQB][2];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) acc[qb][0] = acc[qb][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            float k[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
                if (HD % 16 == 0 || j + 1 < NJ || j * 16 + grp * 4 < HD) load4<float>(sw + (ks * 16 + l16) * P + j * 16 + grp * 4, k[ks]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                    for (int qb = 0; qb < NQB; ++qb) acc[qb][ks] = Elt<float>::mma(k[ks][e], qf[qb][j][e], acc[qb][ks]);
        }
        float sc[NQB][2][4];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
            float mx = -INFINITY;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sc[qb][ks][r] = seen_or_none((uint32_t)(sees[qb] >> (grp * 4)), ks * 16 + r, acc[qb][ks][r] * a.scale_log2);
                    mx = fmaxf(mx, sc[qb][ks][r]);
                }
            const float m_new = fmaxf(m_run[qb], rows_max(mx));
            const float ref = m_new == -INFINITY ? 0.f : m_new;
            const float corr = m_run[qb] == -INFINITY ? 0.f : fast_exp2(m_run[qb] - ref);
            m_run[qb] = m_new;
            l_run[qb] *= corr;
#pragma unroll
            for (int h = 0; h < NJ; ++h) oacc[qb][h] *= corr;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sc[qb][ks][r] = fast_exp2(sc[qb][ks][r] - ref);
                    l_run[qb] += sc[qb][ks][r];
                }
        }
        // O^T += V^T P^T; a last block of eight columns multiplies what lies behind the row too, into rows that are not used
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int h = 0; h < NJ; ++h) {
                    const float v = sw[(KT + ks * 16 + grp * 4 + r) * P + h * 16 + l16];
#pragma unroll
                    for (int qb = 0; qb < NQB; ++qb) oacc[qb][h] = Elt<float>::mma(v, sc[qb][ks][r], oacc[qb][h]);
                }
    };
    auto run = [&](auto OWN, const void* kv, int base, int rows, int from, int to, int skip) __attribute__((always_inline)) {
        from += (wave - skip) & 3;   // the waves go on in turn from one kind to the next
        if (from >= to) return;
        S st;
        st.init(kv, rows, a.heads, w.kvh, lane);
        uint64_t hidden[NQB], sees[NQB];
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) hidden[qb] = OWN ? 0ull : sight[qb].fetch(table, from);
        st.issue(base + from * KT);
        for (int t = from; t < to; t += 4) {
#pragma unroll
            for (int qb = 0; qb < NQB; ++qb) sees[qb] = OWN ? sight[qb].own(base + t * KT) : sight[qb].prefix(a, hidden[qb], t);
            asm volatile("" ::: "memory");      // LDS operations of a wave are done in order
            st.store(sw);
            asm volatile("" ::: "memory");
            if (t + 4 < to) {
#pragma unroll
                for (int qb = 0; qb < NQB; ++qb)
                    if constexpr (!OWN) hidden[qb] = sight[qb].fetch(table, t + 4);
                st.issue(base + (t + 4) * KT);
            }
            multiply(sees);
        }
    };
    const int c0 = min(w.t0, w.ntp), c1 = min(w.t1, w.ntp);
    run(std::false_type{}, a.kv, 0, a.T, c0, c1, 0);
    if (w.f1 > w.f0) run(std::true_type{}, a.fresh, w.f0, w.f1, max(w.t0 - w.ntp, 0), max(w.t1 - w.ntp, 0), c1 - c0);

    float* const so = smem;
    float2* const sml = reinterpret_cast<float2*>(so + 4 * 16 * OLD);
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
        const float l = rows_sum(l_run[qb]);
        __syncthreads();    // every wave is past its last read of the tiles, or of the block before
#pragma unroll
        for (int h = 0; h < NJ; ++h) {
            const float v[4] = {oacc[qb][h][0], oacc[qb][h][1], oacc[qb][h][2], oacc[qb][h][3]};
            store4<float>(so + (wave * 16 + l16) * OLD + h * 16 + grp * 4, v);
        }
        if (grp == 0) sml[wave * 16 + l16] = make_float2(m_run[qb], l);
        __syncthreads();
        join_waves<float, HD, OLD>(a, w, so, sml, tid, qb * 16, bad);
    }
    __syncthreads();    // the flags are complete
    recompute_bad<float, QT, KT>(a, w, tables, bad, wave);
}

// Join of the key ranges: range s has the weight l_s 2^(m_s - m); rows of no
// request are left alone, rows of no key get 0. One wave per (row, head): lane s
// holds range s's maximum and sum, then hd / 4 lanes take four columns each and as
// many groups of them as the wave holds take the ranges in turn. Bound by the parts' bytes: 574 rows of 16 heads of 72
// in 8 ranges 7.3 us (22 MB, 3 TB/s), 8 rows of 12 heads of 64 3.2 us, a launch.
template <typename T>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(SharedAttnDesc a) {
    const int HG = a.heads * a.group, hd = a.hd, lane = threadIdx.x % kWave;
    const int lo = a.seg_start ? min(max(a.seg_start[0], 0), a.M) : 0;
    const int hi = a.seg_start ? min(max(a.seg_start[a.batch], 0), a.M) : a.M;
    const long plane = (long)a.M * HG;
    const long sr = (long)lo * HG + (long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;   // (row, head)
    if (sr >= (long)hi * HG) return;
    const int CL = hd / 4, groups = kWave / CL, grp = lane / CL, col = lane % CL;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < a.nsplit) ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (lane * plane + sr));
    float m = wave_max(ml.x);
    if (__any(ml.x != ml.x)) m = __uint_as_float(0x7fc00000u);      // maxima drop NaN
    float f = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m) * ml.y;
    float L = wave_sum(f);
    const int down = -__builtin_amdgcn_frexp_expf(L);       // weights that sum to less than 1; 0 for 0 and NaN
    f = ldexpf(f, down);
    L = ldexpf(L, down);
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    const float* const po = a.part_o + sr * hd + col * 4;
    constexpr int kRounds = 8;      // rounds of loads on their way at once
    for (int s0 = 0; s0 < a.nsplit; s0 += kRounds * groups) {
        float4 p[kRounds];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int s = s0 + i * groups + grp;
            p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (grp < groups && s < a.nsplit) p[i] = *reinterpret_cast<const float4*>(po + s * plane * hd);
        }
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int s = s0 + i * groups + grp;
            const float fs = __shfl(f, min(s, kWave - 1), kWave);
            if (grp < groups && s < a.nsplit) {
                acc[0] += fs * p[i].x; acc[1] += fs * p[i].y; acc[2] += fs * p[i].z; acc[3] += fs * p[i].w;
            }
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

// One wave per word of 64 tokens: 32 requests of 4096 tokens 2.5 us, a launch.
__global__ __launch_bounds__(kThreads) void shared_bits_kernel(const uint8_t* __restrict__ mask, int batch, int T, int words, uint64_t* __restrict__ bits) {
    const int lane = threadIdx.x % kWave;
    const long i = (long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
    if (i >= (long)batch * words) return;
    const int b = (int)(i / words), t = (int)(i - (long)b * words) * 64 + lane;
    const uint64_t v = __ballot(t >= T || mask[(long)b * T + t] != 0);
    if (lane == 0) bits[i] = v;
}

int slot_tiles(const SharedAttnDesc& a, int tile) { return (int)(((long)a.M * a.group + tile - 1) / tile); }

template <int QT>
void launch_bf16(const SharedAttnDesc& a, hipStream_t s) {
    const int qtiles = slot_tiles(a, QT);
    const int pairs = qtiles * a.nsplit;
    const dim3 grid((unsigned)(QT == 128 ? pairs : (pairs + kXcds - 1) / kXcds * kXcds) * a.heads), block(kThreads);
    switch (a.hd) {
#define MS_HD(n) case n: hipLaunchKernelGGL((shared_bf16_kernel<n, QT>), grid, block, 0, s, a, qtiles); break;
        MS_HD(8) MS_HD(16) MS_HD(24) MS_HD(32) MS_HD(40) MS_HD(48) MS_HD(56) MS_HD(64)
        MS_HD(72) MS_HD(80) MS_HD(88) MS_HD(96) MS_HD(104) MS_HD(112) MS_HD(120) MS_HD(128)
#undef MS_HD
    }
}

template <int NQB>
void launch_f32(const SharedAttnDesc& a, hipStream_t s) {
    const int qtiles = slot_tiles(a, 16 * NQB);
    const int pairs = qtiles * a.nsplit;
    const dim3 grid((unsigned)(pairs + kXcds - 1) / kXcds * kXcds * a.heads), block(kThreads);
    switch (a.hd) {
#define MS_HD(n) case n: hipLaunchKernelGGL((shared_f32_kernel<n, NQB>), grid, block, 0, s, a, qtiles); break;
        MS_HD(8) MS_HD(16) MS_HD(24) MS_HD(32) MS_HD(40) MS_HD(48) MS_HD(56) MS_HD(64)
#undef MS_HD
    }
}

// Whether a split into n ranges stays below the 2^32 threads that end a launch.
bool ranges_fit(const SharedAttnDesc& a, int tile, int n) {
    constexpr long most = (1l << 32) / kThreads;
    return ((long)slot_tiles(a, tile) * n + kXcds) * a.heads < most &&
           (long)a.M * a.heads * a.group / (kThreads / kWave) + 1 < most;
}

}  // namespace

// Query slots per workgroup and key ranges: the pair with the least modelled time. A form whose workgroups take steps of
// `keys` keys takes, with k workgroups on the fullest of 256 CUs (at most as many as fit), in us
//   a + rounds (steps (s0 + s1 hd/64 + (s2 + s3 hd/64) k) + o0 + o1 hd/64)
// and more than one range r0 + r1 n MB + r2 MB more, MB the size of one range's parts. A tile's own rows are taken
// as its slots' rows and an eighth of all: the requests' number plays no part, so that a workspace is planned for the call's shapes.
// Fitted to 5949 measured times (237 shapes in bf16 and 234 in float32: 16 to 128 columns, 1 to 24 K/V heads, groups of 1 to 8, 64 to
// 11000 tokens, 1 to 5700 rows of 1 to 32 requests, every form, 1 to 48 ranges); among powers of two the chosen pair takes 1.02
// times the fastest on average, 1.40 times at most. In us at the best count of ranges, bf16, 16 / 32 / 128 slots: 8 requests over
// 4096 tokens of 16 heads of 64, one row each 11 / 13 / 17, 16 rows 21 / 19 / 24, 32 rows 31 / 25 / 30, 128 rows 94 / 54 / 50, 500 rows
// 390 / 237 / 133; float32, 16 / 32 slots: 1 request of 205 rows over 1024 tokens of 4 heads of 64 14.4 / 15.9, 4 of them 31.5 /
// 30.2, 3 of 137 to 661 rows over 1687 tokens of 26 heads 264 / 210.
void plan_shared_attention(int dtype, SharedAttnDesc& a) {
    a.tile = 16;
    a.nsplit = 1;
    if (a.M == 0) return;
    struct Form {
        int tile, keys;
        double a, s0, s1, s2, s3, o0, o1, r0, r1, r2;
    };
    static const Form bf16[] = {{16, 128, 2.98, 0.101, 0.237, 0.208, 0.201, 2.16, 0.345, 3.21, 0.85, 1.92},
                                {32, 128, 3.23, 0.044, 0.528, 0.378, 0.023, 2.96, 0.581, 2.92, 0.533, 2.83},
                                {128, 64, 5.25, 0.051, 0.356, 0.563, 0.0, 1.99, 1.21, 3.4, 0.248, 2.37}};
    static const Form f32[] = {{16, 128, 4.02, 0.0, 0.597, 0.258, 0.972, 1.085, 1.099, 3.08, 0.731, 0.607},
                               {32, 128, 4.19, 0.0, 0.99, 0.56, 1.378, 1.264, 1.244, 3.18, 1.06, 0.737}};
    const long slots = (long)a.M * a.group;
    const double h = a.hd / 64.0, mb = (double)slots * a.heads * (a.hd + 2) * 4e-6;
    double least = 1e30;
    for (int i = 0; i < (dtype == kBF16 ? 3 : 2); ++i) {
        const Form& f = dtype == kBF16 ? bf16[i] : f32[i];
        // few slots: not where a larger tile is full several times over
        if (dtype == kBF16 && f.tile < 128 && slots > 16 * f.tile + 16 * (f.tile - 16)) continue;
        const int most = dtype != kBF16 ? 2 : f.tile == 128 ? wide_per_cu(a.hd) : few_per_cu(a.hd);
        const long keys = a.T + std::min<long>(a.fresh_rows, a.fresh_rows / 8 + f.tile / a.group);
        const long steps = std::max(1l, (keys + f.keys - 1) / f.keys);
        for (int n = 1; n <= 32 && (n == 1 || (n <= (keys + 63) / 64 && ranges_fit(a, f.tile, n))); n *= 2) {
            const double groups = (double)slot_tiles(a, f.tile) * a.heads * n;
            const double k = std::min(std::ceil(groups / 256), (double)most), rounds = std::max(1.0, groups / (256.0 * most));
            double us = f.a + rounds * ((steps + n - 1) / n * (f.s0 + f.s1 * h + (f.s2 + f.s3 * h) * k) + f.o0 + f.o1 * h);
            if (n > 1) us += f.r0 + (f.r1 * n + f.r2) * mb;
            if (us < least) {
                least = us;
                a.tile = f.tile;
                a.nsplit = n;
            }
        }
    }
}

hipError_t launch_shared_bits(const uint8_t* mask, int batch, int T, uint64_t* bits, hipStream_t s) {
    const int words = (T + 63) / 64;
    const long n = (long)batch * words;
    const dim3 grid((unsigned)((n + kThreads / kWave - 1) / (kThreads / kWave))), block(kThreads);
    hipLaunchKernelGGL(shared_bits_kernel, grid, block, 0, s, mask, batch, T, words, bits);
    return hipGetLastError();
}

hipError_t launch_shared_attention(int dtype, const SharedAttnDesc& a, hipStream_t s) {
    if (a.M == 0) return hipSuccess;
    if (dtype == kBF16) {
        if (a.tile == 16) launch_bf16<16>(a, s);
        else if (a.tile == 32) launch_bf16<32>(a, s);
        else launch_bf16<128>(a, s);
    } else if (a.tile == 16) {
        launch_f32<1>(a, s);
    } else {
        launch_f32<2>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_shared_join(int dtype, const SharedAttnDesc& a, hipStream_t s) {
    if (a.M == 0 || a.nsplit == 1) return hipSuccess;
    const long n = (long)a.M * a.heads * a.group;
    const dim3 grid((unsigned)((n + kThreads / kWave - 1) / (kThreads / kWave))), block(kThreads);
    if (dtype == kBF16) hipLaunchKernelGGL(shared_join_kernel<bf16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(shared_join_kernel<float>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace ms
