/*
 * maskstep operator entry points: the block's row GEMM as a standalone call,
 * for kernel-level parity tests and tuning, and the K/V cache in 8 bits
 * (writing it, reading it back, attention over it). The step API in
 * maskstep.h uses the same kernels.
 *
 * Table 1 of InstGenIE (arXiv 2505.20600) counts the projections XW and the
 * feed-forward (XW1)W2 as the work that shrinks with the masked-row count;
 * these are the row GEMMs computed here.
 */
#ifndef MASKSTEP_OPS_H
#define MASKSTEP_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "maskstep.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MS_EPI_BIAS = 0,        /* out = A W^T + bias */
    MS_EPI_BIAS_RESID = 1,  /* out = A W^T + bias + resid */
    MS_EPI_BIAS_GELU = 2    /* out = GELU(A W^T + bias), x (1 + erf(x / sqrt 2)) / 2 to 3.3e-7 */
} ms_epilogue;

/* out[M][N] = epilogue(A[M][K] W[N][K]^T + bias[N] (+ resid[M][N])), row-major,
 * element type `dtype` (ms_dtype), float32 accumulation, device pointers,
 * 16-byte aligned. K must be a multiple of 64 (bf16) or 32 (fp32) and N of 4.
 * tile_m x tile_n selects the output tile (256x256, 256x192, 192x192, 256x128,
 * 128x128, 128x64, 64x128 or 64x64; float32: 64x64; 0 x 0 = the planner's
 * choice) and
 * ksplit the number of K-range splits (0 = planner's choice; > 1 needs
 * ksplit * M * N * 4 bytes of device workspace in d_ws, NULL otherwise).
 * Asynchronous on `stream`; errors as in maskstep.h, nothing enqueued on error. */
ms_status ms_linear(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* A, const void* W,
                    const void* bias, const void* resid, void* out, int32_t epilogue,
                    int32_t tile_m, int32_t tile_n, int32_t ksplit, void* d_ws, size_t ws_bytes,
                    void* stream);

/* ------------------------------------------------------------------------
 * K/V cache in 8 bits.
 *
 * codes   uint8 [n_caches][tokens][2][n_kv_heads][head_dim], e4m3: sign, four
 *         exponent bits (bias 7), three mantissa bits, largest 448, no
 *         infinities, NaN 0x7f / 0xff. The K row of a token, then its V row.
 * scales  uint8 [n_caches][ceil(tokens / block)][2][n_kv_heads], exponent
 *         bytes b of powers of two 2^(b - 127), one per block of `block`
 *         consecutive tokens, K or V, and head (255 stands for NaN).
 * value = code * scale, exact in bf16 and float32 from 2^-126 up to the type's
 * largest value; one beyond that (code 256 at the scale 2^120, to which the
 * largest bf16 and float32 values round, stands for 2^128) is read as infinite.
 *
 * Element type `dtype` is that of the K/V rows written or read, of the queries
 * and of the output. Pointers are device pointers, 16-byte aligned but for
 * scales (any) and the int32 tables (4 bytes). Calls are asynchronous on
 * `stream`, which belongs to the calling thread's current device, as the
 * buffers do; they allocate nothing and may be captured; errors as in
 * maskstep.h, nothing enqueued on error. Two calls in flight at once must not
 * share a buffer that one of them writes (outputs, workspace).
 *
 * Table entries are read on the device and bounded there: a cache number, token
 * number or row outside its range stands for no key (or no new row), a count
 * is limited to its list, and row ranges to the packed rows. Tables may name a token more
 * than once (attention then counts it as often) and several requests may name
 * one cache.
 *
 * Limits: n_caches 1..2^20; tokens 1..2^20; block a power of two, 1..128;
 * head_dim a multiple of 8, <= 128 (float32: <= 64); n_kv_heads 1..1024; one
 * cache's codes below 4095 MiB; batch and n_seg 1..128; rows x n_heads at
 * most 2^27; one ms_kv8_quantize below 2^28 pieces of at most 1 KiB of a K or V
 * row (whole heads), tokens counted up to whole blocks of at least 16. */
typedef struct {
    int32_t dtype;          /* ms_dtype */
    int32_t n_caches, tokens, n_kv_heads, head_dim, block;
    void* codes;            /* written by ms_kv8_quantize only */
    void* scales;
} ms_kv8_cache;

/* Which cached tokens the requests of a batch read. */
typedef struct {
    int32_t batch;
    int32_t ld_keys;            /* row length of keys; not used when keys is NULL */
    const int32_t* cache_of;    /* [batch] cache number of each request; NULL: request b has cache b (batch <= n_caches) */
    const int32_t* keys;        /* [batch][ld_keys] token numbers; NULL: tokens 0, 1, ... in order */
    const int32_t* n_keys;      /* [batch] how many of them; NULL: all ld_keys, or every token */
} ms_kv8_select;

/* The unmasked tokens of every request, ascending: mask uint8 [batch][tokens]
 * (nonzero = masked, as for mask_step_init) -> keys [batch][ld_keys], n_keys
 * [batch]. ld_keys >= tokens. Entries past a request's count are not written. */
ms_status ms_kv8_keys(const void* mask, int32_t batch, int32_t tokens, int32_t* keys, int32_t ld_keys, int32_t* n_keys,
                      void* stream);

/* K/V rows kv [kv_rows][2][n_kv_heads][head_dim] into every cache of `c`.
 * src_row NULL: token t of cache s is row s * row_stride + t, every token is
 * written (row_stride >= tokens, (n_caches - 1) * row_stride + tokens <=
 * kv_rows). src_row [n_caches][tokens]: token t of cache s becomes row
 * src_row[s][t] where that is a row of kv, and keeps its value elsewhere; a
 * block without a new row is not touched, one with some takes a new scale from
 * all its values, and its kept codes are written for that scale (a kept value
 * changes only where it falls below the new scale's smallest normal code,
 * 2^-6 scale, or an earlier such rounding shows).
 *
 * Scale of a block: the smallest power of two s >= 2^-126 with max |x| <= 448 s
 * over the finite x; 1 if they are all zero. code = x / s rounded to nearest
 * even. NaN and infinities become NaN. */
ms_status ms_kv8_quantize(const ms_kv8_cache* c, const void* kv, int64_t kv_rows, int64_t row_stride,
                          const int32_t* src_row, void* stream);

/* The listed tokens' values: kv[b * row_stride + t] for every listed token t of
 * request b, kv rows as above (row_stride >= tokens). Rows of other tokens are
 * left as they are. */
ms_status ms_kv8_dequantize(const ms_kv8_cache* c, const ms_kv8_select* sel, void* kv, int64_t row_stride, void* stream);

/* Attention of packed query rows over the listed cached tokens of their request
 * and its fresh K/V rows, one softmax over both:
 *   out[m][h] = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q[m][h].k_j),
 * K/V head h / (n_heads / n_kv_heads). A row without any key gives zeros, and so
 * does one whose scores are all -infinity (scores are float32, and one beyond
 * its range is infinite; one of +infinity makes its row NaN). Rows outside
 * [seg_start[0], seg_start[n_seg]) are left as they are. A NaN in a query or in a key or value that is listed makes its
 * rows NaN; tokens that are not listed have no effect whatever they hold.
 * Scores, maxima, sums and the parts of key ranges are float32. bf16 rounds
 * twice: the weights w_j relative to the running maximum, the matrix cores'
 * operand (numerator and denominator take the same rounded ones: 2^-8 of each,
 * at most 2^-8 sum w |v - out| / sum w of the result), and the output. */
typedef struct {
    const void* q;              /* [rows][n_heads][head_dim] */
    void* out;                  /* the same; may be q */
    int32_t rows, n_heads;
    int32_t n_seg;
    const int32_t* seg_start;   /* [n_seg + 1] first packed row of each segment, ascending */
    const int32_t* seg_req;     /* [n_seg] request of each segment; NULL: segment s is request s (n_seg <= batch) */
    const void* fresh;          /* [fresh_rows][2][n_kv_heads][head_dim]; NULL: cached tokens only */
    int64_t fresh_rows;
    const int32_t* fresh_list;  /* [fresh_entries] rows of `fresh`; NULL: entry i is row i (fresh_entries = fresh_rows) */
    int32_t fresh_entries;
    const int32_t* fresh_start; /* [batch + 1] first list entry of each request, ascending */
    float scale;                /* of the scores; 0: 1 / sqrt(head_dim) */
} ms_kv8_attn;

/* Bytes of workspace with which ms_kv8_attention may split the keys of each
 * request as it sees fit (0 when it would not; 0 with the error set on invalid
 * arguments, else the error is cleared). seg_start and the other tables are not read. */
size_t ms_kv8_attention_workspace_bytes(const ms_kv8_cache* c, const ms_kv8_select* sel, const ms_kv8_attn* a);

/* With less workspace than that (or none) it splits into fewer ranges; the
 * order of summation then differs, and with it the last bits. */
ms_status ms_kv8_attention(const ms_kv8_cache* c, const ms_kv8_select* sel, const ms_kv8_attn* a, void* d_ws,
                           size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MASKSTEP_OPS_H */
