// Norms of queries and keys for each head, the position rotation and the K/V
// scatter, one pass over a projection's packed rows [Q heads | K heads | V heads]:
//   y = x / sqrt(mean(x^2) + eps) * gain,  (y_i, y_j) <- (y_i cos - y_j sin, y_j cos + y_i sin)
// for the pairs (i, j) of the rotated columns, (cos, sin) from the table's row of
// the packed row's position.
//
// Bound by the rows' bytes, in and out once. hd / VEC lanes of 16 bytes have a head,
// as many heads side by side as a wave holds, and walk over the row's heads: their
// columns stay the same, so gains and (cos, sin) are loaded once per row and live in
// registers. Sums of squares, norms and rotations are float32; the result is rounded once.
#include <algorithm>

#include "kernels.h"
#include "qk_norm_rope.h"

namespace ms {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

enum { kPairs = 0, kHalves = 1 };

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
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(QkNormRopeDesc d) {
    constexpr int VEC = 16 / sizeof(T);
    const int lane = threadIdx.x % kWave;
    const long unit = (long)blockIdx.x * kWaves + threadIdx.x / kWave;
    const long m = unit / d.parts;
    if (m >= d.M) return;
    const int part = (int)(unit - m * d.parts);
    const int lph = d.hd / VEC, side = kWave / lph;         // lanes per head, heads side by side
    const int sub = lane / lph, at = lane - sub * lph, col = at * VEC;
    const int heads = d.H + 2 * d.G;
    const T* const src = static_cast<const T*>(d.qkv) + m * d.ld;

    float cs[VEC], sn[VEC];
    int other[VEC];         // column that each of this lane's columns is rotated with
    const int pos = d.pos ? d.pos[m] : (int)m;
    const bool turn = d.table && pos >= 0 && pos < d.n_pos;
    const int half = d.rot / 2;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const int c = col + e;
        const bool first = PAIRING == kPairs ? (c & 1) == 0 : c < half;
        const int pair = PAIRING == kPairs ? c >> 1 : first ? c : c - half;
        other[e] = PAIRING == kPairs ? c ^ 1 : first ? c + half : c - half;
        cs[e] = 1.f;
        sn[e] = 0.f;
        if (turn && c < d.rot) {
            const float2 t = *reinterpret_cast<const float2*>(d.table + ((long)pos * half + pair) * 2);
            cs[e] = t.x;
            sn[e] = first ? -t.y : t.y;
        } else {
            other[e] = c;
        }
    }
    const int row = d.rows ? d.rows[m] : (int)m;
    const bool keep = row >= 0 && row < d.kv_rows;
    T* const q = static_cast<T*>(d.q) + m * d.H * d.hd;
    T* const kv = static_cast<T*>(d.kv) + (long)(keep ? row : 0) * 2 * d.G * d.hd;
    // the heads of one pass share their lanes' columns; a head past the last is loaded as head 0 and not written
    for (int h0 = part * side; h0 < heads; h0 += d.parts * side) {
        const int h = h0 + sub;
        const bool mine = sub < side && h < heads;
        const bool is_q = h < d.H, is_v = h >= d.H + d.G;
        const T* const x = src + (mine ? h : 0) * d.hd;
        const int c0 = sub < side ? col : 0;
        const vec16 raw = ld16(x + c0);
        float v[VEC], y[VEC];
        load_vec<T>(reinterpret_cast<const T*>(&raw), v);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss = fmaf(v[e], v[e], ss);
        for (int o = 1; o < lph; o <<= 1) {     // sums of what lies behind within the head; the first lane has them all
            const float t = __shfl_down(ss, o, kWave);
            if (at + o < lph) ss += t;
        }
        ss = __shfl(ss, min(lane - at, kWave - 1), kWave);
        const T* const gain = static_cast<const T*>(is_q ? d.q_gain : d.k_gain);
        const float inv = gain ? 1.0f / sqrtf(ss / (float)d.hd + d.eps) : 1.0f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int oc = sub < side ? other[e] : 0;
            const float p = PAIRING == kPairs ? (oc == col + e ? v[e] : v[e ^ 1]) : Elt<T>::to_f32(x[oc]);
            const float ga = gain ? Elt<T>::to_f32(gain[c0 + e]) : 1.f, gb = gain ? Elt<T>::to_f32(gain[oc]) : 1.f;
            const float a = v[e] * inv * ga, b = p * inv * gb;
            y[e] = sn[e] == 0.f && oc == c0 + e ? a : fmaf(a, cs[e], b * sn[e]);
        }
        if (!mine) continue;
        if (is_q) {
            store_vec<T>(q + h * d.hd + col, y);
        } else if (keep) {
            T* const to = kv + (h - d.H) * d.hd + col;      // K heads, then V heads
            if (is_v) st16(to, raw);
            else store_vec<T>(to, y);
        }
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(int dtype, const QkNormRopeDesc& desc, hipStream_t s) {
    if (desc.M == 0) return hipSuccess;
    QkNormRopeDesc d = desc;
    const int vec = dtype == kBF16 ? 8 : 4, side = kWave / (d.hd / vec);
    const int passes = (d.H + 2 * d.G + side - 1) / side;
    // few rows: their heads spread over more waves
    d.parts = (int)std::max(1l, std::min<long>(passes, 2048 / std::max(1, d.M)));
    const dim3 grid((unsigned)(((long)d.M * d.parts + kWaves - 1) / kWaves)), block(kThreads);
    if (dtype == kBF16) {
        if (d.halves) hipLaunchKernelGGL((qk_norm_rope_kernel<bf16_t, kHalves>), grid, block, 0, s, d);
        else hipLaunchKernelGGL((qk_norm_rope_kernel<bf16_t, kPairs>), grid, block, 0, s, d);
    } else {
        if (d.halves) hipLaunchKernelGGL((qk_norm_rope_kernel<float, kHalves>), grid, block, 0, s, d);
        else hipLaunchKernelGGL((qk_norm_rope_kernel<float, kPairs>), grid, block, 0, s, d);
    }
    return hipGetLastError();
}

}  // namespace ms
