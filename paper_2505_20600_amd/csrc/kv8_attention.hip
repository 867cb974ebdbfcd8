// Attention over an 8-bit K/V cache: packed query rows of a batch over the
// listed cached tokens of their request (codes and scales) and its fresh K/V
// rows (the model's type), one softmax over both. A row without any key is 0.
#include <algorithm>

#include "kernels.h"
#include "kv8.h"

namespace ms {
namespace {

// One wave per (row, query head): lane = key of a 64-key tile for the scores,
// lane = column for the weighted sum.
template <typename T>
__global__ __launch_bounds__(kWave) void attend_row_kernel(Kv8AttnDesc a) {
    __shared__ float s_q[128], s_p[kWave], s_sc[kWave];
    __shared__ int s_row[kWave];
    const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y;
    const int hd = a.c.hd, H = a.c.heads, dkv = H * hd, d = dkv * a.group, g = head / a.group;
    int seg = 0;
    while (seg < a.nseg && !(row >= a.seg_start[seg] && row < a.seg_start[seg + 1])) ++seg;
    if (seg == a.nseg) return;
    const int b = a.seg_req ? a.seg_req[seg] : seg;
    Kv8Req r{nullptr, nullptr, nullptr, 0, 0, 0};
    if (b >= 0 && b < a.sel.batch) {
        r = kv8_request(a.c, a.sel, b);
        kv8_fresh(a, b, r);
    }
    for (int i = lane; i < hd; i += kWave) s_q[i] = Elt<T>::to_f32(static_cast<const T*>(a.q)[(long)row * d + head * hd + i]);
    __syncthreads();
    const T* const fresh = static_cast<const T*>(a.kv);
    float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
    const int total = r.nk + r.nf;
    for (int k0 = 0; k0 < total; k0 += kWave) {
        const int i = k0 + lane;
        const bool cached = i < r.nk;
        int t = -1;
        float sv = 0.f, z = -INFINITY;
        if (cached) {
            t = r.keys ? r.keys[i] : i;
            if (t < 0 || t >= a.c.T) t = -1;
        } else if (i < total) {
            t = a.f_rows ? a.f_rows[r.f0 + i - r.nk] : r.f0 + i - r.nk;
            if (t < 0 || t >= a.kv_rows) t = -1;
        }
        if (t >= 0) {
            float dot = 0.f;
            if (cached) {
                const uint8_t* sp = r.scales + (long)(t >> a.c.lblock) * 2 * H + g;
                sv = kv8_scale(sp[H]);
                const uint8_t* p = r.codes + (long)t * 2 * dkv + g * hd;
                const float sk = kv8_scale(sp[0]);
                for (int j = 0; j < hd; j += 2) {
                    const float2 v = kv8_to_f32x2<false>(*reinterpret_cast<const uint16_t*>(p + j), sk);
                    dot += s_q[j] * v.x + s_q[j + 1] * v.y;
                }
            } else {
                const T* p = fresh + (long)t * 2 * dkv + g * hd;
                for (int j = 0; j < hd; ++j) dot += s_q[j] * Elt<T>::to_f32(p[j]);
            }
            z = dot * a.scale_log2;
        }
        const float m_new = fmaxf(m, wave_max(z));
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float corr = m == -INFINITY ? 0.f : fast_exp2(m - ref);
        const float p = t >= 0 ? fast_exp2(z - ref) : 0.f;
        l = l * corr + wave_sum(p);
        m = m_new;
        __syncthreads();
        s_p[lane] = p;
        s_sc[lane] = sv;
        s_row[lane] = t;
        __syncthreads();
        for (int x = 0; x < 2; ++x) {
            const int col = lane + x * kWave;
            if (col >= hd) continue;
            float acc = o[x] * corr;
            for (int k = 0; k < kWave; ++k) {
                if (s_row[k] < 0) continue;
                float v;
                if (k0 + k < r.nk) {
                    v = kv8_to_f32x2<false>(r.codes[((long)s_row[k] * 2 + 1) * dkv + g * hd + col], s_sc[k]).x;
                } else {
                    v = Elt<T>::to_f32(fresh[((long)s_row[k] * 2 + 1) * dkv + g * hd + col]);
                }
                acc += s_p[k] * v;
            }
            o[x] = acc;
        }
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    for (int x = 0; x < 2; ++x) {
        const int col = lane + x * kWave;
        if (col < hd) static_cast<T*>(a.o)[(long)row * d + head * hd + col] = Elt<T>::from_f32(o[x] * inv);
    }
}

}  // namespace

int plan_kv8_attention(int dtype, int M, int nseg, int heads, int group, int hd, long keys) { return 1; }

hipError_t launch_kv8_attention(int dtype, const Kv8AttnDesc& a, hipStream_t s) {
    if (a.M == 0) return hipSuccess;
    const dim3 grid(a.M, a.c.heads * a.group), block(kWave);
    if (dtype == kBF16) hipLaunchKernelGGL(attend_row_kernel<bf16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(attend_row_kernel<float>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace ms
