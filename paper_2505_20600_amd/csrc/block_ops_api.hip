// Entry points of the 4-bit row products, the per-head norms with rotation, and
// the attention over a shared prefix: validation, then the launchers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/maskstep_ops.h"
#include "kernels.h"
#include "mx4.h"
#include "qk_norm_rope.h"
#include "shared_attention.h"
#include "step_internal.h"

namespace {

using ms::set_error;

constexpr int64_t kMaxRows = 1 << 26;

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool known_dtype(int32_t t) { return t == MS_FP32 || t == MS_BF16; }
int64_t element(int32_t t) { return t == MS_BF16 ? 2 : 4; }

ms_status check_rows(int32_t dtype, const void* x, int64_t rows, int32_t cols, int64_t ld, const void* codes, const void* scales) {
    if (!known_dtype(dtype)) return set_error(MS_EDTYPE, "unknown dtype %d", dtype);
    if (rows < 0 || rows > kMaxRows) return set_error(MS_ESHAPE, "rows %lld outside 0..2^26", (long long)rows);
    if (cols < 32 || cols % 32 || cols > (1 << 20)) return set_error(MS_ESHAPE, "cols %d must be a multiple of 32, 32..2^20", cols);
    if (ld < cols || ld > (1ll << 32) || ld * element(dtype) % 16)
        return set_error(MS_ESHAPE, "ld %lld must be at least cols %d, at most 2^32, and whole 16 bytes", (long long)ld, cols);
    if (rows > 0 && (!x || !codes || !scales)) return set_error(MS_EINVAL, "x, codes or scales is NULL");
    if (!aligned(x, 16) || !aligned(codes, 16)) return set_error(MS_EALIGN, "x or codes not 16-byte aligned");
    return MS_OK;
}

ms_status check_product(int32_t M, int32_t N, int32_t K) {
    if (M < 0 || M > kMaxRows) return set_error(MS_ESHAPE, "M %d outside 0..2^26", M);
    if (N < 4 || N % 4 || N > (1 << 20)) return set_error(MS_ESHAPE, "N %d must be a multiple of 4, 4..2^20", N);
    if (K < 32 || K % 32 || K > (1 << 20)) return set_error(MS_ESHAPE, "K %d must be a multiple of 32, 32..2^20", K);
    // then fewer than 2^21 tiles of 64 rows and columns or more, and at most 2^29 threads of the pass over a K split
    if ((int64_t)M * N > (1ll << 31)) return set_error(MS_ESHAPE, "M x N, %lld, above 2^31", (long long)M * N);
    return MS_OK;
}

ms_status check_attn(int32_t dtype, const ms_shared_attn* a, ms::SharedAttnDesc* d) {
    if (!a) return set_error(MS_EINVAL, "attention arguments are NULL");
    if (!known_dtype(dtype)) return set_error(MS_EDTYPE, "unknown dtype %d", dtype);
    if (a->rows < 0 || a->rows > kMaxRows) return set_error(MS_ESHAPE, "rows %d outside 0..2^26", a->rows);
    if (a->n_kv_heads < 1 || a->n_kv_heads > 1024) return set_error(MS_ESHAPE, "n_kv_heads %d outside 1..1024", a->n_kv_heads);
    if (a->n_heads < 1 || a->n_heads % a->n_kv_heads || a->n_heads > 1024)
        return set_error(MS_ESHAPE, "n_heads %d must be a multiple of n_kv_heads %d, at most 1024", a->n_heads, a->n_kv_heads);
    if (a->head_dim < 8 || a->head_dim % 8 || a->head_dim > (dtype == MS_BF16 ? 128 : 64))
        return set_error(MS_ESHAPE, "head_dim %d must be a multiple of 8, at most 128 (bf16) or 64 (fp32)", a->head_dim);
    // at most one workgroup per 16 of them, 2^23 of 256 threads: a launch takes fewer than 2^32 threads
    if ((int64_t)a->rows * a->n_heads > (1 << 27)) return set_error(MS_ESHAPE, "rows x n_heads above 2^27");
    if (a->batch < 1 || a->batch > ms::kSharedMaxBatch)
        return set_error(MS_ESHAPE, "batch %d outside 1..%d", a->batch, ms::kSharedMaxBatch);
    if (a->tokens < 0 || a->tokens > (1 << 20)) return set_error(MS_ESHAPE, "tokens %d outside 0..2^20", a->tokens);
    const int64_t row = 2ll * a->n_kv_heads * a->head_dim * element(dtype), most = (1ll << 32) - (1 << 20);
    if (a->tokens * row >= most) return set_error(MS_ESHAPE, "tokens %d: the prefix's rows must stay below 4095 MiB", a->tokens);
    if (!a->seg_start && a->batch > 1) return set_error(MS_EINVAL, "a batch of more than one needs seg_start");
    if (a->rows > 0 && (!a->q || !a->out)) return set_error(MS_EINVAL, "q or out is NULL");
    if (a->tokens > 0 && !a->kv) return set_error(MS_EINVAL, "kv is NULL");
    if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->kv, 16) || !aligned(a->fresh, 16))
        return set_error(MS_EALIGN, "q, out, kv or fresh not 16-byte aligned");
    if (!aligned(a->bits, 8)) return set_error(MS_EALIGN, "bits not 8-byte aligned");
    if (!aligned(a->seg_start, 4) || !aligned(a->fresh_start, 4)) return set_error(MS_EALIGN, "an int32 table is not 4-byte aligned");
    if (!std::isfinite(a->scale)) return set_error(MS_EINVAL, "scale must be finite");
    if (a->fresh) {
        if (!a->fresh_start) return set_error(MS_EINVAL, "own rows need fresh_start");
        if (a->fresh_rows < 0 || a->fresh_rows > (1 << 28) || a->fresh_rows * row >= most)
            return set_error(MS_ESHAPE, "fresh_rows %lld: the rows must stay below 4095 MiB", (long long)a->fresh_rows);
    }
    const bool own = a->fresh && a->fresh_rows > 0;
    d->q = a->q;
    d->o = a->out;
    d->kv = a->kv;
    d->bits = a->tokens > 0 ? a->bits : nullptr;
    d->seg_start = a->seg_start;
    d->fresh = own ? a->fresh : nullptr;
    d->fresh_start = own ? a->fresh_start : nullptr;
    d->fresh_rows = own ? (int)a->fresh_rows : 0;
    d->batch = a->batch;
    d->T = a->tokens;
    d->words = (a->tokens + 63) / 64;
    d->M = a->rows;
    d->heads = a->n_kv_heads;
    d->group = a->n_heads / a->n_kv_heads;
    d->hd = a->head_dim;
    d->scale_log2 = (float)(1.4426950408889634 * (a->scale != 0.f ? (double)a->scale : 1.0 / std::sqrt((double)a->head_dim)));
    if (!std::isfinite(d->scale_log2)) return set_error(MS_EINVAL, "scale too large");
    d->tile = 16;
    d->nsplit = 1;
    d->part_o = d->part_ml = nullptr;
    return MS_OK;
}

// Float32 words of partial results per key range.
size_t range_floats(const ms::SharedAttnDesc& d) { return (size_t)d.M * d.heads * d.group * (d.hd + 2); }

// The form and the key ranges of a call with rows, its parts within ws_bytes.
void plan_attn(int32_t dtype, ms::SharedAttnDesc& d, size_t ws_bytes) {
    ms::plan_shared_attention(dtype, d);
    d.nsplit = std::max(1, std::min(d.nsplit, (int)std::min<size_t>(ws_bytes / (range_floats(d) * sizeof(float)), 1024)));
}

}  // namespace

extern "C" {

ms_status ms_mx4_quantize(int32_t dtype, const void* x, int64_t rows, int32_t cols, int64_t ld, void* codes, void* scales,
                          void* stream) {
    ms_status st = check_rows(dtype, x, rows, cols, ld, codes, scales);
    if (st != MS_OK) return st;
    hipError_t e = ms::launch_mx4_quantize(dtype, x, rows, cols, ld, static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales),
                                           static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "quantize launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

ms_status ms_mx4_dequantize(int32_t dtype, const void* codes, const void* scales, int64_t rows, int32_t cols, void* x,
                            int64_t ld, void* stream) {
    ms_status st = check_rows(dtype, x, rows, cols, ld, codes, scales);
    if (st != MS_OK) return st;
    hipError_t e = ms::launch_mx4_dequantize(dtype, static_cast<const uint8_t*>(codes), static_cast<const uint8_t*>(scales), rows,
                                             cols, x, ld, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "dequantize launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

size_t ms_mx4_linear_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (check_product(M, N, K) != MS_OK) return 0;
    ms::clear_error();
    ms::Mx4LinearDesc d{};
    d.g.M = M;
    d.g.N = N;
    d.g.K = K;
    ms::plan_mx4_linear(d, ~(size_t)0);
    return d.g.ksplit > 1 ? (size_t)d.g.ksplit * M * N * sizeof(float) : 0;
}

ms_status ms_mx4_linear(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* a_codes, const void* a_scales,
                        const void* w_codes, const void* w_scales, const void* bias, const void* resid, void* out,
                        int32_t epilogue, void* d_ws, size_t ws_bytes, void* stream) {
    if (!known_dtype(dtype)) return set_error(MS_EDTYPE, "unknown dtype %d", dtype);
    ms_status st = check_product(M, N, K);
    if (st != MS_OK) return st;
    if (epilogue < MS_EPI_BIAS || epilogue > MS_EPI_BIAS_GELU) return set_error(MS_EINVAL, "unknown epilogue %d", epilogue);
    if (!w_codes || !w_scales || !bias) return set_error(MS_EINVAL, "w_codes, w_scales or bias is NULL");
    if (M > 0 && (!a_codes || !a_scales || !out || (epilogue == MS_EPI_BIAS_RESID && !resid)))
        return set_error(MS_EINVAL, "a_codes, a_scales, out or resid is NULL");
    for (const void* p : {a_codes, w_codes, bias, resid, static_cast<const void*>(out), static_cast<const void*>(d_ws)})
        if (!aligned(p, 16)) return set_error(MS_EALIGN, "codes, bias, resid, out or workspace not 16-byte aligned");
    if (M == 0) return ms::clear_error();
    ms::Mx4LinearDesc d{};
    d.a = static_cast<const uint8_t*>(a_codes);
    d.as = static_cast<const uint8_t*>(a_scales);
    d.w = static_cast<const uint8_t*>(w_codes);
    d.ws = static_cast<const uint8_t*>(w_scales);
    d.g.bias = bias;
    d.g.R = resid;
    d.g.C = out;
    d.g.M = M;
    d.g.N = d.g.ldr = d.g.ldc = N;
    d.g.K = K;
    d.g.epilogue = epilogue == MS_EPI_BIAS ? ms::kEpiBias : epilogue == MS_EPI_BIAS_RESID ? ms::kEpiBiasResid : ms::kEpiBiasGelu;
    d.g.part = static_cast<float*>(d_ws);
    ms::plan_mx4_linear(d, d_ws ? ws_bytes / sizeof(float) : 0);
    hipError_t e = ms::launch_mx4_linear(dtype, d, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "product launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

ms_status ms_mx4_linear_plan(int32_t M, int32_t N, int32_t K, size_t ws_bytes, int32_t* tile, int32_t* ranges) {
    if (!tile || !ranges) return set_error(MS_EINVAL, "tile or ranges is NULL");
    ms_status st = check_product(M, N, K);
    if (st != MS_OK) return st;
    ms::Mx4LinearDesc d{};
    d.g.M = M;
    d.g.N = N;
    d.g.K = K;
    ms::plan_mx4_linear(d, ws_bytes / sizeof(float));
    *tile = d.form == ms::kMx4Rows ? 16 : d.form == ms::kMx4Tile64 ? 64 : d.form == ms::kMx4Tile128 ? 128 : 256;
    *ranges = d.g.ksplit;
    return ms::clear_error();
}

ms_status ms_qk_norm_rope(const ms_qk_norm_rope_args* a, void* stream) {
    if (!a) return set_error(MS_EINVAL, "arguments are NULL");
    if (!known_dtype(a->dtype)) return set_error(MS_EDTYPE, "unknown dtype %d", a->dtype);
    if (a->rows < 0 || a->rows > kMaxRows) return set_error(MS_ESHAPE, "rows %d outside 0..2^26", a->rows);
    if (a->n_heads < 1 || a->n_heads > 1024 || a->n_kv_heads < 1 || a->n_kv_heads > 1024)
        return set_error(MS_ESHAPE, "n_heads %d or n_kv_heads %d outside 1..1024", a->n_heads, a->n_kv_heads);
    if (a->head_dim < 8 || a->head_dim % 8 || a->head_dim > 128)
        return set_error(MS_ESHAPE, "head_dim %d must be a multiple of 8, at most 128", a->head_dim);
    const int64_t cols = (int64_t)(a->n_heads + 2 * a->n_kv_heads) * a->head_dim;
    if (a->ld < cols || a->ld > (1ll << 32) || a->ld * element(a->dtype) % 16)
        return set_error(MS_ESHAPE, "ld %lld must be at least the %lld columns of the heads, at most 2^32, and whole 16 bytes",
                         (long long)a->ld, (long long)cols);
    if (a->kv_rows < 0 || a->kv_rows > (1ll << 31)) return set_error(MS_ESHAPE, "kv_rows outside 0..2^31");
    if (a->table) {
        if (a->rot < 2 || a->rot % 2 || a->rot > a->head_dim)
            return set_error(MS_ESHAPE, "rot %d must be even, 2..head_dim", a->rot);
        if (a->n_pos < 0 || a->n_pos > (1 << 30)) return set_error(MS_ESHAPE, "n_pos %d outside 0..2^30", a->n_pos);
    }
    if (a->pairing != MS_ROPE_PAIRS && a->pairing != MS_ROPE_HALVES) return set_error(MS_EINVAL, "unknown pairing %d", a->pairing);
    if (!(a->eps >= 0.f) || !std::isfinite(a->eps)) return set_error(MS_EINVAL, "eps must be finite and not negative");
    if (a->rows > 0 && (!a->qkv || !a->q || (a->kv_rows > 0 && !a->kv))) return set_error(MS_EINVAL, "qkv, q or kv is NULL");
    if (!aligned(a->qkv, 16) || !aligned(a->q, 16) || !aligned(a->kv, 16) || !aligned(a->q_gain, 16) || !aligned(a->k_gain, 16) ||
        !aligned(a->table, 16))
        return set_error(MS_EALIGN, "qkv, q, kv, a gain or the table not 16-byte aligned");
    if (!aligned(a->pos, 4) || !aligned(a->dst_rows, 4)) return set_error(MS_EALIGN, "an int32 table is not 4-byte aligned");
    ms::QkNormRopeDesc d{a->qkv, a->q, a->kv, a->q_gain, a->k_gain, a->table, a->pos, a->dst_rows, (long)a->ld, (long)a->kv_rows,
                         a->rows, a->n_heads, a->n_kv_heads, a->head_dim, a->table ? a->rot : 0, a->n_pos,
                         a->pairing == MS_ROPE_HALVES, a->eps, 1};
    hipError_t e = ms::launch_qk_norm_rope(a->dtype, d, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "norm and rotation launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

ms_status ms_shared_bits(const void* mask, int32_t batch, int32_t tokens, uint64_t* bits, void* stream) {
    if (!mask || !bits) return set_error(MS_EINVAL, "mask or bits is NULL");
    if (batch < 1 || batch > ms::kSharedMaxBatch) return set_error(MS_ESHAPE, "batch %d outside 1..%d", batch, ms::kSharedMaxBatch);
    if (tokens < 1 || tokens > (1 << 20)) return set_error(MS_ESHAPE, "tokens %d outside 1..2^20", tokens);
    if (!aligned(bits, 8)) return set_error(MS_EALIGN, "bits not 8-byte aligned");
    hipError_t e = ms::launch_shared_bits(static_cast<const uint8_t*>(mask), batch, tokens, bits, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "bits launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

size_t ms_shared_attention_workspace_bytes(int32_t dtype, const ms_shared_attn* a) {
    ms::SharedAttnDesc d;
    if (check_attn(dtype, a, &d) != MS_OK) return 0;
    ms::clear_error();
    ms::plan_shared_attention(dtype, d);
    return d.nsplit > 1 ? d.nsplit * range_floats(d) * sizeof(float) : 0;
}

ms_status ms_shared_attention_plan(int32_t dtype, const ms_shared_attn* a, size_t ws_bytes, int32_t* tile, int32_t* ranges) {
    if (!tile || !ranges) return set_error(MS_EINVAL, "tile or ranges is NULL");
    ms::SharedAttnDesc d;
    ms_status st = check_attn(dtype, a, &d);
    if (st != MS_OK) return st;
    if (d.M > 0) plan_attn(dtype, d, ws_bytes);
    *tile = d.tile;
    *ranges = d.nsplit;
    return ms::clear_error();
}

ms_status ms_shared_attention(int32_t dtype, const ms_shared_attn* a, void* d_ws, size_t ws_bytes, void* stream) {
    ms::SharedAttnDesc d;
    ms_status st = check_attn(dtype, a, &d);
    if (st != MS_OK) return st;
    if (!aligned(d_ws, 16)) return set_error(MS_EALIGN, "workspace not 16-byte aligned");
    if (d.M == 0) return ms::clear_error();
    plan_attn(dtype, d, d_ws ? ws_bytes : 0);
    if (d.nsplit > 1) {
        d.part_o = static_cast<float*>(d_ws);
        d.part_ml = d.part_o + (size_t)d.nsplit * d.M * d.heads * d.group * d.hd;
    }
    hipError_t e = ms::launch_shared_attention(dtype, d, static_cast<hipStream_t>(stream));
    if (e == hipSuccess) e = ms::launch_shared_join(dtype, d, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "attention launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

}  // extern "C"
