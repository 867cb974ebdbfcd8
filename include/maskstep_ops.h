/*
 * maskstep operator entry points: the block's row GEMM as a standalone call,
 * for kernel-level parity tests and tuning, and the K/V cache in 8 bits
 * (writing it, reading it back, attention over it); the step API in
 * maskstep.h uses the same kernels. Then three operators for blocks of other
 * designs: row products of microscaled 4-bit operands, the norms of queries and
 * keys for each head with the position rotation and the K/V scatter, and attention
 * of a batch over one shared prefix.
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

/* ------------------------------------------------------------------------
 * Row products of microscaled 4-bit operands.
 *
 * A row of K elements, K a multiple of 32:
 * codes   uint8 [K / 2], e2m1, element 2i in the low half of byte i: sign, two
 *         exponent bits, one mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their
 *         negatives.
 * scales  uint8 [K / 32], exponent bytes b of powers of two 2^(b - 127), one per
 *         32 consecutive elements; 255 makes them NaN.
 * Rows lie behind each other without gaps. Element type `dtype` is that of the rows
 * read or written in full. Pointers are device pointers, 16-byte aligned but for
 * scales (any). Calls are asynchronous on `stream`, which belongs to the calling
 * thread's current device, as the buffers do; they allocate nothing and may be
 * captured; errors as in maskstep.h, nothing enqueued on error. Inputs and outputs
 * must not overlap (but resid, which may be out), and two calls in flight at once must
 * not share a buffer that one of them writes.
 *
 * Limits: rows, M 0..2^26; cols, N, K at most 2^20; N a multiple of 4; M x N at most 2^31. */

/* Rows x [rows][cols], `ld` elements apart (ld >= cols, whole 16 bytes), into codes
 * and scales. Scale of 32 elements: the smallest power of two s with max |x| <= 7 s,
 * between 2^-126 and 2^125; 1 if they are all zero. code = x / s rounded to nearest
 * even, above 6 to 6. An infinity or NaN among them: codes 0, scale byte 255. */
ms_status ms_mx4_quantize(int32_t dtype, const void* x, int64_t rows, int32_t cols, int64_t ld, void* codes, void* scales,
                          void* stream);

/* The values of such rows, exact but where a code times a scale byte below 1 or
 * above 252 (which ms_mx4_quantize does not write) leaves the type. Elements between rows are left as they are. */
ms_status ms_mx4_dequantize(int32_t dtype, const void* codes, const void* scales, int64_t rows, int32_t cols, void* x,
                            int64_t ld, void* stream);

/* Bytes of workspace with which ms_mx4_linear may split K as it sees fit (0 when it would not; 0 with the
 * error set on invalid sizes, else the error is cleared). */
size_t ms_mx4_linear_workspace_bytes(int32_t M, int32_t N, int32_t K);

/* What ms_mx4_linear launches for these sizes with ws_bytes of workspace (for parity tests and tuning): a workgroup's
 * outputs are tile x tile (16, 64, 128 or 256), K is split into `ranges`. */
ms_status ms_mx4_linear_plan(int32_t M, int32_t N, int32_t K, size_t ws_bytes, int32_t* tile, int32_t* ranges);

/* out[M][N] = epilogue(A W^T + bias[N] (+ resid[M][N])), A [M][K] and W [N][K] codes and scales, float32 sums, one
 * rounding to `dtype` (that of bias, resid and out). A NaN scale makes its row (of A) or column (of W) NaN. With less
 * workspace than the above (or none) K is split into fewer ranges; the order of summation then differs. */
ms_status ms_mx4_linear(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* a_codes, const void* a_scales,
                        const void* w_codes, const void* w_scales, const void* bias, const void* resid, void* out,
                        int32_t epilogue, void* d_ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Norms of queries and keys for each head, position rotation, K/V scatter, in one
 * pass over a projection's packed rows [n_heads Q | n_kv_heads K | n_kv_heads V]
 * heads of head_dim:
 *   y = x / sqrt(mean(x^2) + eps) * gain        (Q and K heads; the mean over the head)
 *   (y_i, y_j) <- (y_i cos - y_j sin, y_j cos + y_i sin)   (the first `rot` columns)
 * with the pairs (i, j) = (2p, 2p + 1) or (p, p + rot / 2) and cos, sin =
 * table[pos[m]][p]. Q goes to q[m], K and V of packed row m to kv[dst_rows[m]]. Float32
 * within, one rounding; V is copied. The norm holds for heads of any finite size, also where float32
 * does not hold their squares; a head of zeros is 0, with eps = 0 NaN. Conventions as above; a row of kv must not
 * be named twice in one call, and the outputs must not overlap the inputs.
 * Limits: rows 0..2^26; heads 1..1024 each; head_dim a multiple of 8, <= 128; ld whole 16 bytes. */
enum { MS_ROPE_PAIRS = 0, MS_ROPE_HALVES = 1 };
typedef struct {
    int32_t dtype;              /* of qkv, the gains, q and kv */
    int32_t rows, n_heads, n_kv_heads, head_dim;
    const void* qkv;            /* [rows] rows of (n_heads + 2 n_kv_heads) x head_dim elements, ld apart */
    int64_t ld;
    const void *q_gain, *k_gain;/* [head_dim]; NULL: that kind is not normalised */
    float eps;
    const float* table;         /* [n_pos][rot / 2][2] cos, sin; NULL: no rotation */
    int32_t n_pos, rot, pairing;
    const int32_t* pos;         /* [rows]; NULL: m. A position outside 0..n_pos - 1: the row is not rotated */
    void* q;                    /* [rows][n_heads][head_dim] */
    void* kv;                   /* [kv_rows][2][n_kv_heads][head_dim] */
    int64_t kv_rows;
    const int32_t* dst_rows;    /* [rows] rows of kv; NULL: m. Outside 0..kv_rows - 1: K and V are not written */
} ms_qk_norm_rope_args;
ms_status ms_qk_norm_rope(const ms_qk_norm_rope_args* a, void* stream);

/* ------------------------------------------------------------------------
 * Attention of a batch over one shared prefix: the requests edit one template (or
 * follow one prompt, a row at a time), whose K/V rows are read and multiplied once for all of
 * them; each request hides prefix tokens of its own (those it recomputes) and brings K/V
 * rows of its own, one softmax over both:
 *   out[m][h] = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q[m][h].k_j),
 * j over the prefix tokens that row m's request b does not hide, then its own rows
 * [fresh_start[b], fresh_start[b + 1]); K/V head h / (n_heads / n_kv_heads). There is no order
 * among own rows: a row sees all of its request's, so that several rows of a causal continuation
 * in one call would see later ones. A row
 * without any key gives zeros, and so does one whose scores are all -infinity
 * (scores are float32, q[m][h].k_j before the scale too, and one beyond its range is infinite; one of +infinity makes its
 * row NaN). What a row does not see has no effect on it whatever it holds; a NaN in a
 * query or in a key or value that it sees makes it NaN. Finite values give a finite result, up
 * to the type's largest (less float32's rounding), whatever the weights sum to. Rows outside [seg_start[0],
 * seg_start[batch]) are left as they are.
 * Scores, maxima, sums and the parts of key ranges are float32. bf16 rounds twice: the
 * weights w_j relative to the running maximum, the matrix cores' operand (numerator
 * and denominator take the same rounded ones: 2^-8 of each, at most 2^-8 sum w |v - out|
 * / sum w of the result), and the output.
 *
 * Table entries are read on the device and bounded there (row and own-row starts to their
 * buffers). Conventions as above; out may be q. Pointers 16-byte aligned but for bits (8
 * bytes) and the int32 tables (4).
 * Limits: batch 1..128; tokens 0..2^20; head_dim a multiple of 8, <= 128 (float32: <= 64);
 * heads 1..1024; the prefix and the own rows below 4095 MiB each; rows x n_heads at most 2^27. */
typedef struct {
    const void* q;              /* [rows][n_heads][head_dim] */
    void* out;                  /* the same; may be q */
    int32_t rows, n_heads, n_kv_heads, head_dim;
    const void* kv;             /* prefix [tokens][2][n_kv_heads][head_dim] */
    int32_t tokens, batch;
    const uint64_t* bits;       /* [batch][ceil(tokens / 64)], bit t % 64 of word t / 64 set: token t is hidden; NULL: none is */
    const int32_t* seg_start;   /* [batch + 1] first packed row of each request, ascending; NULL: one request, every row */
    const void* fresh;          /* [fresh_rows][2][n_kv_heads][head_dim]; NULL: prefix only */
    int64_t fresh_rows;
    const int32_t* fresh_start; /* [batch + 1] first own row of each request, ascending */
    float scale;                /* of the scores; 0: 1 / sqrt(head_dim) */
} ms_shared_attn;

/* The hidden tokens of every request as bits: mask uint8 [batch][tokens] (nonzero = hidden, as the masked
 * tokens of mask_step_init) -> bits [batch][ceil(tokens / 64)]. */
ms_status ms_shared_bits(const void* mask, int32_t batch, int32_t tokens, uint64_t* bits, void* stream);

/* Bytes of workspace with which ms_shared_attention may split the keys as it sees fit (0 when it would not; 0 with the error set on
 * invalid arguments, else the error is cleared). The tables are not read. */
size_t ms_shared_attention_workspace_bytes(int32_t dtype, const ms_shared_attn* a);

/* What ms_shared_attention launches for such arguments with ws_bytes of workspace (for parity tests and tuning): `tile` query
 * slots (a row and a query head of one K/V head) per workgroup (16, 32, or in bf16 128), the keys in `ranges`. The tables are not read. */
ms_status ms_shared_attention_plan(int32_t dtype, const ms_shared_attn* a, size_t ws_bytes, int32_t* tile, int32_t* ranges);

/* With less workspace than that (or none) it splits into fewer ranges; the order of summation
 * then differs, and with it the last bits. */
ms_status ms_shared_attention(int32_t dtype, const ms_shared_attn* a, void* d_ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MASKSTEP_OPS_H */
