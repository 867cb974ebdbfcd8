// Norms of queries and keys for each head, the position rotation and the K/V
// scatter, one pass over a projection's packed rows [Q heads | K heads | V heads]:
//   y = x / sqrt(mean(x^2) + eps) * gain,  (y_i, y_j) <- (y_i cos - y_j sin, y_j cos + y_i sin)
// for the pairs (i, j) of the rotated columns, (cos, sin) from the table's row of
// the packed row's position.
//
// Bound by the rows' bytes, in and out once. hd / VEC lanes of 16 bytes have a head,
// as many heads side by side as a wave holds, and walk over the row's heads: their
// columns stay the same, so the products of gains and (cos, sin) are formed once per row and
// live in registers. Sums of squares, norms and rotations are float32; the result is rounded once.
// 32768 rows of 16 Q, K and V heads of 72 (bf16) take 98 us, 4.7 TB/s where a copy of as much reaches 5.3; 24 + 8 + 8
// heads of 128 133 us (5.2 TB/s), of 12 heads of 64 65 us (4.8); float32, 8 heads of 64 81 us (5.1). One row of 24
// heads of 128 4.5 us, a launch and one chain of loads.
//
// Where the mean square with eps lies far out in float32 the head is scaled by the power of two that brings its largest
// element, or the root of eps, near 1, and eps by its square: exact but for what is 2^-126 of the largest. Far out is infinite,
// or below 2^-46: squares lose digits further down and the root's instruction takes a subnormal as 0, and a reciprocal root above 2^23
// would lift the last place of a subnormal product above 2^-126. A head whose root mean square is 1e-7 is there only with
// an eps as small. Looking for such heads costs 1 to 4% (95, 132, 62 and 81 us above without it); scaling them at the wave's end,
// out of the passes' way, took 101, 134, 69 and 81, one branch for four passes 100, 133, 66 and 81.
#include <algorithm>

#include "kernels.h"
#include "qk_norm_rope.h"

namespace ms {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// Pairs (2 p, 2 p + 1), in one lane; (p, p + rot / 2) where that is whole lanes away; or anywhere, through LDS.
enum { kPairs = 0, kLanes = 1, kAny = 2 };

template <typename T>
__device__ __forceinline__ void load_vec(const T* p, float* v) {
    if constexpr (sizeof(T) == 2) {
        const vec16 r = ld16(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    } else {
        load4<float>(p, v);
    }
}

template <typename T>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
    if constexpr (sizeof(T) == 2) {
        vec16 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        st16(p, o);
    } else {
        store4<float>(p, v);
    }
}

// One wave per (packed row, part of its heads).
template <typename T, int PAIRING>
__global__ __launch_bounds__(kThreads, 4) void qk_norm_rope_kernel(QkNormRopeDesc d) {
    constexpr int VEC = 16 / sizeof(T);
    constexpr int kAtOnce = PAIRING == kAny ? 2 : 4;        // passes whose rows are loaded before the first is used, as many as the registers hold
    __shared__ __attribute__((aligned(16))) uint8_t smem[PAIRING == kAny ? kWaves * kAtOnce * 1024 : 16];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int lph = d.hd / VEC, side = kWave / lph;         // lanes per head, heads side by side
    const int sub = min(lane / lph, side - 1), at = min(lane - sub * lph, lph - 1), col = at * VEC;     // lanes past the last head repeat its last
    const bool idle = lane >= side * lph;
    const int half = d.rot / 2;
    // passes over `side` heads of one kind: Q, K, V
    const int nq = (d.H + side - 1) / side, nk = (d.G + side - 1) / side, passes = nq + 2 * nk;
    const bool whole_heads = d.rot == d.hd;
    const float per = 1.0f / (float)d.hd;
    const bool in_rot = col < d.rot, all_in = col + VEC <= d.rot;
    // with kLanes, the columns that this lane's are turned with and the lane that holds them
    const int away = PAIRING == kLanes && in_rot ? (col < half ? half : -half) : 0;
    const int from = lane + away / VEC;
    auto partner = [&](int e) {         // the column that column col + e, below rot, is turned with
        const int c = col + e;
        return PAIRING == kPairs ? c ^ 1 : c < half ? c + half : c - half;
    };
    // gains of this lane's columns and of those they are turned with, as they lie
    vec16 ga[2], gb[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const T* const gain = static_cast<const T*>(k ? d.k_gain : d.q_gain);
        const uint32_t one = sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u;
        ga[k] = gb[k] = vec16{{one, one, one, one}};
        if (!gain) continue;
        ga[k] = ld16(gain + col);
        if constexpr (PAIRING == kLanes) {
            gb[k] = ld16(gain + col + away);
        } else {
            T x[VEC];
            __builtin_memcpy(x, &ga[k], 16);
            T y[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = PAIRING == kPairs ? x[e ^ 1] : gain[col + e < d.rot ? partner(e) : 0];
            __builtin_memcpy(&gb[k], y, 16);
        }
    }

    const long units = (long)d.M * d.parts;
    for (long unit = (long)blockIdx.x * kWaves + wave; unit < units; unit += (long)gridDim.x * kWaves) {
        const long m = d.parts == 1 ? unit : unit / d.parts;
        const int p0 = (int)(unit - m * d.parts);
        const T* const src = static_cast<const T*>(d.qkv) + m * d.ld;
        vec16 raw[kAtOnce];
        int kind[kAtOnce], head[kAtOnce];       // 0 Q, 1 K, 2 V, 3 past the last pass; this lane's head of that kind
        auto fetch = [&](int first) {
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int p = first + u * d.parts;
                kind[u] = p < nq ? 0 : p < nq + nk ? 1 : p < passes ? 2 : 3;
                head[u] = (kind[u] == 0 ? p : kind[u] == 1 ? p - nq : p - nq - nk) * side + sub;
                const int n = kind[u] == 0 ? d.H : d.G, before = kind[u] == 0 ? 0 : kind[u] == 1 ? d.H : d.H + d.G;
                raw[u] = ld16(src + (kind[u] == 3 ? 0 : before + min(head[u], n - 1)) * d.hd + col);   // past the last head: not written
            }
        };
        const int pos = d.pos ? d.pos[m] : (int)m;
        const int row = d.rows ? d.rows[m] : (int)m;
        fetch(p0);
        // y_c = (x_c fc + x_c' fs) / rms: gain and cos of column c, gain of the column c' that it is turned with and signed sin
        const bool turn = d.table && pos >= 0 && pos < d.n_pos;
        float cs[VEC], sn[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            cs[e] = 1.f;
            sn[e] = 0.f;
        }
        if (turn && in_rot) {
            const float* const t = d.table + (long)pos * half * 2;
            if (PAIRING == kPairs && all_in && half % 2 == 0) {
#pragma unroll
                for (int e = 0; e < VEC; e += 4) {
                    const float4 v = *reinterpret_cast<const float4*>(t + col + e);
                    cs[e] = cs[e + 1] = v.x;
                    sn[e] = -v.y;
                    sn[e + 1] = v.y;
                    cs[e + 2] = cs[e + 3] = v.z;
                    sn[e + 2] = -v.w;
                    sn[e + 3] = v.w;
                }
            } else if (PAIRING == kLanes) {
                const float* const p = t + (col < half ? col : col - half) * 2;
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const float4 v = *reinterpret_cast<const float4*>(p + 2 * e);
                    cs[e] = v.x;
                    sn[e] = col < half ? -v.y : v.y;
                    cs[e + 1] = v.z;
                    sn[e + 1] = col < half ? -v.w : v.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int c = col + e;
                    if (c >= d.rot) continue;
                    const bool first = PAIRING == kPairs ? (c & 1) == 0 : c < half;
                    const int pair = PAIRING == kPairs ? c >> 1 : first ? c : c - half;
                    const float2 v = *reinterpret_cast<const float2*>(t + pair * 2);
                    cs[e] = v.x;
                    sn[e] = first ? -v.y : v.y;
                }
            }
        }
        float fc[2][VEC], fs[2][VEC];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float x[VEC], y[VEC];
#pragma unroll
            for (int w = 0; w < 4; ++w) asm volatile("" : "+v"(ga[k].w[w]), "+v"(gb[k].w[w]));     // not unpacked before the loop
            load_vec<T>(reinterpret_cast<const T*>(&ga[k]), x);
            load_vec<T>(reinterpret_cast<const T*>(&gb[k]), y);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                fc[k][e] = x[e] * cs[e];
                fs[k][e] = y[e] * sn[e];
            }
        }
        const bool keep = row >= 0 && row < d.kv_rows;
        T* const q = static_cast<T*>(d.q) + m * d.H * d.hd;
        T* const kv = static_cast<T*>(d.kv) + (long)(keep ? row : 0) * 2 * d.G * d.hd;

        for (int first = p0;;) {
            if constexpr (PAIRING == kAny) {
                asm volatile("" ::: "memory");      // LDS operations of a wave are done in order
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (!idle) st16(smem + (wave * kAtOnce + u) * 1024 + lane * 16, raw[u]);     // a head's rows lie in order
                asm volatile("" ::: "memory");
            }
            float ss[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                float v[VEC];
                load_vec<T>(reinterpret_cast<const T*>(&raw[u]), v);
                ss[u] = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) ss[u] = fmaf(v[e], v[e], ss[u]);
#pragma unroll
                for (int w = 0; w < 4; ++w) asm volatile("" : "+v"(raw[u].w[w]));      // unpacked again below, not kept
            }
            for (int o = 1; o < lph; o <<= 1) {     // sums of what lies behind within the head; the first lane has them all
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const float t = __shfl_down(ss[u], o, kWave);
                    if (at + o < lph) ss[u] += t;
                }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) ss[u] = __shfl(ss[u], sub * lph, kWave);
            // 1 / sqrt(mean + eps) of the head times 2^down, that power of two the one near its largest element
            auto scaled_inv = [&](const vec16& r, int& down) {
                float x[VEC], big = sqrtf(d.eps), sum = 0.f;
                load_vec<T>(reinterpret_cast<const T*>(&r), x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) big = fmaxf(big, fabsf(x[e]));
                for (int o = 1; o < lph; o <<= 1) {
                    const float t = __shfl_down(big, o, kWave);
                    if (at + o < lph) big = fmaxf(big, t);
                }
                big = __shfl(big, sub * lph, kWave);
                down = -__builtin_amdgcn_frexp_expf(big);       // 0 for 0, infinities and NaN
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float t = ldexpf(x[e], down);
                    sum = fmaf(t, t, sum);
                }
                for (int o = 1; o < lph; o <<= 1) {
                    const float t = __shfl_down(sum, o, kWave);
                    if (at + o < lph) sum += t;
                }
                sum = __shfl(sum, sub * lph, kWave);
                return __builtin_amdgcn_rsqf(fmaf(sum, per, ldexpf(d.eps, 2 * down)));
            };
            auto turned = [&](int u, const float (&fc_)[VEC], const float (&fs_)[VEC], bool norm) {
                float inv = 1.0f;
                int down = 0;
                bool any = false;
                if (norm) {
                    const float mean = fmaf(ss[u], per, d.eps);
                    const bool far = !(mean >= 0x1p-46f && mean < INFINITY);
                    inv = __builtin_amdgcn_rsqf(mean);
                    any = __any(far);
                    if (any) {
                        const float scaled = scaled_inv(raw[u], down);
                        if (far) inv = scaled;
                        else down = 0;
                    }
                }
                float v[VEC], p[VEC], y[VEC];
                load_vec<T>(reinterpret_cast<const T*>(&raw[u]), v);
                if constexpr (PAIRING == kPairs) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) p[e] = v[e ^ 1];
                } else if constexpr (PAIRING == kLanes) {
                    vec16 o;
#pragma unroll
                    for (int k = 0; k < 4; ++k) o.w[k] = (uint32_t)__shfl((int)raw[u].w[k], from, kWave);
                    load_vec<T>(reinterpret_cast<const T*>(&o), p);
                } else {
                    const T* const x = reinterpret_cast<const T*>(smem + (wave * kAtOnce + u) * 1024) + sub * d.hd;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) p[e] = Elt<T>::to_f32(x[col + e < d.rot ? partner(e) : 0]);
                }
                if (any) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        v[e] = ldexpf(v[e], down);
                        p[e] = ldexpf(p[e], down);
                    }
                }
                if (turn && whole_heads) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) y[e] = fmaf(p[e], fs_[e], v[e] * fc_[e]) * inv;
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float x = v[e] * fc_[e];
                        y[e] = (turn && col + e < d.rot ? fmaf(p[e], fs_[e], x) : x) * inv;     // not 0 times an infinity
                    }
                }
                vec16 o;
                store_vec<T>(reinterpret_cast<T*>(&o), y);
                return o;
            };
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (kind[u] == 0) {
                    const vec16 y = turned(u, fc[0], fs[0], d.q_gain != nullptr);
                    if (!idle && head[u] < d.H) st16(q + head[u] * d.hd + col, y);
                } else if (kind[u] == 1) {
                    const vec16 y = turned(u, fc[1], fs[1], d.k_gain != nullptr);
                    if (!idle && head[u] < d.G && keep) st16(kv + head[u] * d.hd + col, y);
                } else if (kind[u] == 2) {
                    if (!idle && head[u] < d.G && keep) st16(kv + (d.G + head[u]) * d.hd + col, raw[u]);
                }
            }
            first += kAtOnce * d.parts;
            if (first >= passes) break;
            fetch(first);
        }
    }
}

template <typename T>
void launch(const QkNormRopeDesc& d, dim3 grid, hipStream_t s) {
    const dim3 block(kThreads);
    if (!d.halves) hipLaunchKernelGGL((qk_norm_rope_kernel<T, kPairs>), grid, block, 0, s, d);
    else if (d.rot / 2 % (16 / sizeof(T)) == 0) hipLaunchKernelGGL((qk_norm_rope_kernel<T, kLanes>), grid, block, 0, s, d);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<T, kAny>), grid, block, 0, s, d);
}

}  // namespace

hipError_t launch_qk_norm_rope(int dtype, const QkNormRopeDesc& desc, hipStream_t s) {
    if (desc.M == 0) return hipSuccess;
    QkNormRopeDesc d = desc;
    const int vec = dtype == kBF16 ? 8 : 4, side = kWave / (d.hd / vec);
    const int passes = (d.H + side - 1) / side + 2 * ((d.G + side - 1) / side);
    // few rows: their heads spread over more waves
    d.parts = (int)std::max(1l, std::min<long>(passes, 4096 / std::max(1, d.M)));
    // as many waves as the CUs hold take the rows in turn
    const dim3 grid((unsigned)std::min<long>(((long)d.M * d.parts + kWaves - 1) / kWaves, 256 * 4));
    if (dtype == kBF16) launch<bf16_t>(d, grid, s);
    else launch<float>(d, grid, s);
    return hipGetLastError();
}

}  // namespace ms
