// Entry points of the 8-bit K/V cache: validation, then the launchers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/maskstep_ops.h"
#include "kernels.h"
#include "kv8.h"
#include "step_internal.h"

namespace {

constexpr int kMaxTokens = 1 << 20;

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

ms_status check_cache(const ms_kv8_cache* c, ms::Kv8Cache* out) {
    using ms::set_error;
    if (!c) return set_error(MS_EINVAL, "cache description is NULL");
    if (c->dtype != MS_FP32 && c->dtype != MS_BF16) return set_error(MS_EDTYPE, "unknown dtype %d", c->dtype);
    if (c->n_caches < 1 || c->n_caches > kMaxTokens) return set_error(MS_ESHAPE, "n_caches %d outside 1..2^20", c->n_caches);
    if (c->tokens < 1 || c->tokens > kMaxTokens) return set_error(MS_ESHAPE, "tokens %d outside 1..2^20", c->tokens);
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return set_error(MS_ESHAPE, "n_kv_heads %d outside 1..1024", c->n_kv_heads);
    if (c->head_dim < 8 || c->head_dim % 8 || c->head_dim > (c->dtype == MS_BF16 ? 128 : 64))
        return set_error(MS_ESHAPE, "head_dim %d must be a multiple of 8, at most 128 (bf16) or 64 (fp32)", c->head_dim);
    if (c->block < 1 || c->block > 128 || (c->block & (c->block - 1)))
        return set_error(MS_ESHAPE, "block %d must be a power of two, 1..128", c->block);
    if (2ll * c->tokens * c->n_kv_heads * c->head_dim >= (1ll << 32) - (1 << 20))
        return set_error(MS_ESHAPE, "one cache's codes (tokens x 2 x n_kv_heads x head_dim bytes) must stay below 4095 MiB");
    if (!c->codes || !c->scales) return set_error(MS_EINVAL, "codes or scales is NULL");
    if (!aligned(c->codes, 16)) return set_error(MS_EALIGN, "codes not 16-byte aligned");
    out->codes = static_cast<uint8_t*>(c->codes);
    out->scales = static_cast<uint8_t*>(c->scales);
    out->n_caches = out->n_scales = c->n_caches;
    out->T = c->tokens;
    out->heads = c->n_kv_heads;
    out->hd = c->head_dim;
    out->lblock = 0;
    while ((1 << out->lblock) < c->block) ++out->lblock;
    out->blocks = (c->tokens + c->block - 1) / c->block;
    return MS_OK;
}

ms_status check_select(const ms_kv8_cache* c, const ms_kv8_select* sel, ms::Kv8Select* out) {
    using ms::set_error;
    if (!sel) return set_error(MS_EINVAL, "selection is NULL");
    if (sel->batch < 1 || sel->batch > ms::kKv8MaxSegments)
        return set_error(MS_ESHAPE, "batch %d outside 1..%d", sel->batch, ms::kKv8MaxSegments);
    if (!sel->cache_of && sel->batch > c->n_caches)
        return set_error(MS_ESHAPE, "batch %d above n_caches %d needs cache_of", sel->batch, c->n_caches);
    if (sel->keys && (sel->ld_keys < 0 || sel->ld_keys > kMaxTokens))
        return set_error(MS_ESHAPE, "ld_keys %d outside 0..2^20", sel->ld_keys);
    if (!aligned(sel->cache_of, 4) || !aligned(sel->keys, 4) || !aligned(sel->n_keys, 4))
        return set_error(MS_EALIGN, "an int32 table is not 4-byte aligned");
    out->codes_of = out->scales_of = sel->cache_of;
    out->keys = sel->keys;
    out->n_keys = sel->n_keys;
    out->ld_keys = sel->keys ? sel->ld_keys : c->tokens;
    out->batch = sel->batch;
    return MS_OK;
}

ms_status check_attn(const ms_kv8_cache* c, const ms_kv8_select* sel, const ms_kv8_attn* a, ms::Kv8AttnDesc* d) {
    using ms::set_error;
    ms_status st = check_cache(c, &d->c);
    if (st != MS_OK) return st;
    st = check_select(c, sel, &d->sel);
    if (st != MS_OK) return st;
    if (!a) return set_error(MS_EINVAL, "attention arguments are NULL");
    if (a->rows < 0 || a->rows > (1 << 26)) return set_error(MS_ESHAPE, "rows %d outside 0..2^26", a->rows);
    if (a->n_heads < 1 || a->n_heads % c->n_kv_heads || a->n_heads > 1024)
        return set_error(MS_ESHAPE, "n_heads %d must be a multiple of n_kv_heads %d, at most 1024", a->n_heads, c->n_kv_heads);
    // at most one workgroup per 16 of them, 2^23 of 256 threads: a launch takes fewer than 2^32 threads
    if ((int64_t)a->rows * a->n_heads > (1 << 27)) return set_error(MS_ESHAPE, "rows x n_heads above 2^27");
    if (a->n_seg < 1 || a->n_seg > ms::kKv8MaxSegments)
        return set_error(MS_ESHAPE, "n_seg %d outside 1..%d", a->n_seg, ms::kKv8MaxSegments);
    if (!a->seg_req && a->n_seg > sel->batch) return set_error(MS_ESHAPE, "n_seg %d above batch %d needs seg_req", a->n_seg, sel->batch);
    if (!a->seg_start || (a->rows > 0 && (!a->q || !a->out))) return set_error(MS_EINVAL, "q, out or seg_start is NULL");
    if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->fresh, 16))
        return set_error(MS_EALIGN, "q, out or fresh not 16-byte aligned");
    if (!aligned(a->seg_start, 4) || !aligned(a->seg_req, 4) || !aligned(a->fresh_list, 4) || !aligned(a->fresh_start, 4))
        return set_error(MS_EALIGN, "an int32 table is not 4-byte aligned");
    if (!std::isfinite(a->scale)) return set_error(MS_EINVAL, "scale must be finite");
    long entries = 0;
    if (a->fresh) {
        if (!a->fresh_start) return set_error(MS_EINVAL, "fresh rows need fresh_start");
        const int64_t row = 2ll * c->n_kv_heads * c->head_dim * (c->dtype == MS_BF16 ? 2 : 4);
        if (a->fresh_rows < 0 || a->fresh_rows > (1 << 28) || a->fresh_rows * row >= (1ll << 32) - (1 << 20))
            return set_error(MS_ESHAPE, "fresh_rows %lld: the rows must stay below 4095 MiB", (long long)a->fresh_rows);
        entries = a->fresh_list ? a->fresh_entries : a->fresh_rows;
        if (entries < 0 || entries > (1 << 28)) return set_error(MS_ESHAPE, "fresh rows or entries outside 0..2^28");
    }
    d->q = a->q;
    d->o = a->out;
    d->seg_start = a->seg_start;
    d->seg_req = a->seg_req;
    d->nseg = a->n_seg;
    d->M = a->rows;
    d->group = a->n_heads / c->n_kv_heads;
    d->kv = a->fresh && a->fresh_rows > 0 ? a->fresh : nullptr;
    d->f_rows = a->fresh_list;
    d->f_start = a->fresh_start;
    d->f_end = a->fresh_start ? a->fresh_start + 1 : nullptr;
    d->kv_rows = a->fresh ? a->fresh_rows : 0;
    d->f_list = (int)entries;
    d->scale_log2 = (float)(1.4426950408889634 * (a->scale != 0.f ? (double)a->scale : 1.0 / std::sqrt((double)c->head_dim)));
    if (!std::isfinite(d->scale_log2)) return set_error(MS_EINVAL, "scale too large");
    d->tile = 16;
    d->nsplit = 1;
    d->part_o = d->part_ml = nullptr;
    return MS_OK;
}

// Float32 words of partial results per key range.
size_t range_floats(const ms::Kv8AttnDesc& d) {
    return (size_t)d.M * d.c.heads * d.group * (d.c.hd + 2);
}

void plan(int dtype, ms::Kv8AttnDesc& d) {
    // the fresh rows: about as many for each request
    ms::plan_kv8_attention(dtype, d, d.sel.ld_keys + d.f_list / d.sel.batch);
}

}  // namespace

extern "C" {

ms_status ms_kv8_keys(const void* mask, int32_t batch, int32_t tokens, int32_t* keys, int32_t ld_keys, int32_t* n_keys,
                      void* stream) {
    using ms::set_error;
    if (!mask || !keys || !n_keys) return set_error(MS_EINVAL, "mask, keys or n_keys is NULL");
    if (batch < 1 || batch > ms::kKv8MaxSegments) return set_error(MS_ESHAPE, "batch %d outside 1..%d", batch, ms::kKv8MaxSegments);
    if (tokens < 1 || tokens > kMaxTokens) return set_error(MS_ESHAPE, "tokens %d outside 1..2^20", tokens);
    if (ld_keys < tokens || ld_keys > kMaxTokens) return set_error(MS_ESHAPE, "ld_keys %d outside tokens..2^20", ld_keys);
    if (!aligned(keys, 4) || !aligned(n_keys, 4)) return set_error(MS_EALIGN, "an int32 table is not 4-byte aligned");
    hipError_t e = ms::launch_kv8_keys(static_cast<const uint8_t*>(mask), batch, tokens, keys, ld_keys, n_keys,
                                       static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "key list launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

ms_status ms_kv8_quantize(const ms_kv8_cache* c, const void* kv, int64_t kv_rows, int64_t row_stride,
                          const int32_t* src_row, void* stream) {
    using ms::set_error;
    ms::Kv8Cache k;
    ms_status st = check_cache(c, &k);
    if (st != MS_OK) return st;
    if (!kv) return set_error(MS_EINVAL, "kv is NULL");
    if (!aligned(kv, 16)) return set_error(MS_EALIGN, "kv not 16-byte aligned");
    if (!aligned(src_row, 4)) return set_error(MS_EALIGN, "an int32 table is not 4-byte aligned");
    if (kv_rows < 1 || kv_rows > (1ll << 40)) return set_error(MS_ESHAPE, "kv_rows outside 1..2^40");
    if (!src_row && (row_stride < c->tokens || row_stride > kv_rows ||
                     (int64_t)(c->n_caches - 1) * row_stride + c->tokens > kv_rows))
        return set_error(MS_ESHAPE, "row_stride %lld: need at least tokens, and %d caches of it within %lld rows",
                         (long long)row_stride, c->n_caches, (long long)kv_rows);
    if (!ms::kv8_quantize_fits(c->dtype, k))
        return set_error(MS_ESHAPE, "%d caches of %d tokens of %d heads are too many for one call", c->n_caches, c->tokens,
                         c->n_kv_heads);
    hipError_t e = ms::launch_kv8_quantize(c->dtype, k, kv, row_stride, src_row, kv_rows, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "quantize launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

ms_status ms_kv8_dequantize(const ms_kv8_cache* c, const ms_kv8_select* sel, void* kv, int64_t row_stride, void* stream) {
    using ms::set_error;
    ms::Kv8Cache k;
    ms_status st = check_cache(c, &k);
    if (st != MS_OK) return st;
    ms::Kv8Select s;
    st = check_select(c, sel, &s);
    if (st != MS_OK) return st;
    if (!kv) return set_error(MS_EINVAL, "kv is NULL");
    if (!aligned(kv, 16)) return set_error(MS_EALIGN, "kv not 16-byte aligned");
    if (row_stride < c->tokens || row_stride > (1ll << 40)) return set_error(MS_ESHAPE, "row_stride outside tokens..2^40");
    hipError_t e = ms::launch_kv8_dequantize(c->dtype, k, s, kv, row_stride, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "dequantize launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

size_t ms_kv8_attention_workspace_bytes(const ms_kv8_cache* c, const ms_kv8_select* sel, const ms_kv8_attn* a) {
    ms::Kv8AttnDesc d;
    if (check_attn(c, sel, a, &d) != MS_OK) return 0;
    ms::clear_error();
    plan(c->dtype, d);
    return d.nsplit > 1 ? d.nsplit * range_floats(d) * sizeof(float) : 0;
}

ms_status ms_kv8_attention(const ms_kv8_cache* c, const ms_kv8_select* sel, const ms_kv8_attn* a, void* d_ws,
                           size_t ws_bytes, void* stream) {
    using ms::set_error;
    ms::Kv8AttnDesc d;
    ms_status st = check_attn(c, sel, a, &d);
    if (st != MS_OK) return st;
    if (!aligned(d_ws, 16)) return set_error(MS_EALIGN, "workspace not 16-byte aligned");
    if (d.M == 0) return ms::clear_error();
    const size_t one = range_floats(d) * sizeof(float);
    plan(c->dtype, d);
    d.nsplit = std::max(1, std::min(d.nsplit, d_ws ? (int)std::min<size_t>(ws_bytes / one, 1024) : 1));
    if (d.nsplit > 1) {
        d.part_o = static_cast<float*>(d_ws);
        d.part_ml = d.part_o + (size_t)d.nsplit * d.M * d.c.heads * d.group * d.c.hd;
    }
    hipError_t e = ms::launch_kv8_attention(c->dtype, d, static_cast<hipStream_t>(stream));
    if (e == hipSuccess) e = ms::launch_kv8_join(c->dtype, d, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(MS_EHIP, "attention launch: %s", hipGetErrorString(e));
    return ms::clear_error();
}

}  // extern "C"
