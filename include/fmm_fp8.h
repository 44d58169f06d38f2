/*
 * fmm_fp8.h - the 8-bit floating-point layer of the B200 (sm_100a) library of fmm.h: activations and weights in e4m3 with
 * an fp32 scale for each block of 128, their product, its gradients, and all three for tokens that are sorted by expert.
 *
 * e4m3 form of a matrix: codes (one byte a number, e4m3 without infinities) and scales (fp32), one for each block.  A number is
 * code * scale.  The blocks of the three forms (the last ones of a row or column being as short as they come):
 *     rows     128 consecutive columns of a row      scales[b][i]: block b of row i           ceil(cols / 128) x rows
 *     columns  128 consecutive rows of a column      scales[b][j]: block b of column j        rows / 128 x cols
 *     tiles    128 rows x 128 columns                scales[a][b], dense                      ceil(rows / 128) x ceil(cols / 128)
 * With a = max(max |x| over the block, 1e-12):
 *     FMM_FP8_SCALE_AMAX_DIV_448   scale = fl(a / 448),                         code = e4m3(fl(x * fl(448 / a)))
 *     FMM_FP8_SCALE_POW2           scale = 2^e, e = ceil(log2(fl(a / 448))),    code = e4m3(x * 2^-e)
 * all in fp32, e4m3() to the nearest number, ties to even, at most 448.  A block that holds an infinity or a NaN gets NaN as its scale.
 *
 * A product contracts over the axis along which the blocks of its operands run: forward and input gradient take rows and
 * tiles, the weight gradient takes columns on both sides.
 *
 * Groups (experts).  `groups` > 0 with `offsets` (dev, groups + 1 numbers): rows offsets[g] .. offsets[g + 1] - 1 of the tokens
 * belong to group g.  They are read on the device, so a call needs no synchronisation: one that is below its predecessor or
 * negative counts as its predecessor (or 0), one beyond the rows as the rows.  Rows of no group take no part and are not written.  At most
 * FMM_FP8_MAX_GROUPS.  groups == 0: one group of all rows, offsets is not used.
 *     In the form along the columns every group begins on a multiple of 128 rows, in the order of the groups, and the rest of its last
 *     block is zeros; fmm_fp8_column_rows says how many rows that takes at most.  Rows behind the last block in use are neither written nor read.
 *
 * General rules
 *   - Status codes, "dev" pointers and streams as in fmm.h: nothing throws, aborts or traps the device, nothing is
 *     allocated or synchronised, work is only enqueued on `cuda_stream`, on the current device.  Calls may be captured
 *     into CUDA graphs.  Results do not depend on the run: no floating-point atomics, every sum in a fixed order.
 *   - Matrices are row-major; `ld*` is the distance between rows in elements, at least the number of columns.  Inputs and outputs in
 *     fp32, bf16 and fp16 may have any alignment that their type allows (16-byte aligned rows are fastest).  Codes have 16-byte
 *     aligned rows (ld a multiple of 16), scales of rows and columns too (ld a multiple of 4), unless the call says that they are `loose`: then these may
 *     lie as fp32 numbers do, rows any distance apart, and products load them without TMA.  Nothing is written behind the last column of a row,
 *     and nothing read but what shares an aligned 16-byte vector with an element of the row.
 *   - Rows, columns and groups may be 0: then nothing is read, and what an empty sum gives is written.  M, N, K and column rows are below
 *     2^31 - 16384 (FMM_ERR_SHAPE).
 *   - An output may not overlap an input or another output.
 */
#ifndef FMM_FP8_H
#define FMM_FP8_H

#include "fmm_int8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FMM_FP8_SCALE_AMAX_DIV_448 = 0, FMM_FP8_SCALE_POW2 = 1 } fmm_fp8_scale_t;
#define FMM_FP8_MAX_GROUPS 1024

/* Rows of the form along the columns of `rows` tokens in `groups` groups: the multiple of 128 that holds any distribution of them. */
fmm_status_t fmm_fp8_column_rows(int64_t rows, int64_t groups, int64_t* column_rows);

/* Forms of x (dev, rows x cols of `type`) along its rows, along its columns, or both from one pass over x.
 *   codes (rows x cols), scales (ceil(cols / 128) x rows, lds apart): form along the rows; codes NULL: not wanted.
 *   column_codes (fmm_fp8_column_rows x cols), column_scales (a row for each 128 of those): along the columns; NULL: not wanted.
 *   loose != 0: both kinds of scales as any fp32 numbers. */
typedef struct {
    fmm_type_t type;
    fmm_fp8_scale_t scale_mode;
    int64_t rows, cols;
    const void* x;          int64_t ldx;
    int64_t groups;         const int32_t* offsets;
    uint8_t* codes;         int64_t ldc;
    float* scales;          int64_t lds;
    uint8_t* column_codes;  int64_t ldcc;
    float* column_scales;   int64_t ldcs;
    int64_t loose;
} fmm_fp8_quantize_t;
fmm_status_t fmm_fp8_quantize(const fmm_fp8_quantize_t* p, void* cuda_stream);

/* Form in tiles of `count` matrices x (dev, rows x cols of `type`, step_x elements apart): codes (step_c apart) and scales (dense, one matrix
 * behind the other). */
typedef struct {
    fmm_type_t type;
    fmm_fp8_scale_t scale_mode;
    int64_t count, rows, cols;
    const void* x;          int64_t ldx, step_x;
    uint8_t* codes;         int64_t ldc, step_c;
    float* scales;
} fmm_fp8_quantize_weight_t;
fmm_status_t fmm_fp8_quantize_weight(const fmm_fp8_quantize_weight_t* p, void* cuda_stream);

/* The product and its gradients.  With the numbers that codes and scales stand for, g being the group of token i:
 *     fmm_fp8_matmul       out[i][j]    (+)= sum_k a[i][k] b_g[j][k] + bias_g[j]    a: M x K along its rows,   b_g: N x K in tiles, out M x N
 *     fmm_fp8_grad_input   out[i][k]    (+)= sum_j a[i][j] b_g[j][k]                a: M x N (dy), its rows,   b_g: N x K in tiles, out M x K
 *     fmm_fp8_grad_weight  out_g[j][k]  (+)= sum_i a[i][j] b[i][k]                  a: M x N (dy) and b: M x K along their columns, out_g N x K
 *   M: tokens; grad_weight: rows of the form along the columns, a multiple of 128 (FMM_ERR_SHAPE).  tokens: of a grouped grad_weight only, the number of
 *   tokens (from 1 to M, else FMM_ERR_SHAPE), to which offsets are cut as elsewhere; 0: it is not known, and with offsets beyond it nothing is read outside of the
 *   M rows, but the gradients of groups that end there are not specified.
 *   a, lda, a_scales, lda_scales; b, ldb, b_scales as the forms have them, ldb_scales: of grad_weight's b only.  loose != 0: scales along rows and
 *   columns as any fp32 numbers.  step_b: codes from one group's weight to the next (a multiple of 16), whose scales are dense.  bias: groups x N of `type`, dense, or NULL (gradients: NULL).
 *   out: of `type`; step_out: elements from one group's weight gradient to the next.  accumulate != 0 adds to what it holds; without, a group
 *   without rows has 0 as its weight gradient.
 *   Arithmetic: the products of a block of 128 are summed by the tensor cores in fp32, the blocks' sums, times their two scales, in fp32 registers,
 *   rounded to nearest; the result is rounded once.  The two scales are multiplied first, in fp32 (grad_weight: the sum times b's scale, then a's), so that
 *   scales whose product is beyond fp32 give infinities or NaN. */
typedef struct {
    fmm_type_t type;
    int accumulate;
    int64_t M, N, K;
    int64_t groups;         const int32_t* offsets;
    const uint8_t* a;       int64_t lda;
    const float* a_scales;  int64_t lda_scales;
    const uint8_t* b;       int64_t ldb, step_b;
    const float* b_scales;  int64_t ldb_scales;
    const void* bias;
    void* out;              int64_t ldo, step_out;
    int64_t loose, tokens;
} fmm_fp8_product_t;
fmm_status_t fmm_fp8_matmul(const fmm_fp8_product_t* p, void* cuda_stream);
fmm_status_t fmm_fp8_grad_input(const fmm_fp8_product_t* p, void* cuda_stream);
fmm_status_t fmm_fp8_grad_weight(const fmm_fp8_product_t* p, void* cuda_stream);

/* How products are multiplied, for tests and measurements: from now on every call of the calling host thread takes tiles of so many columns: 256
 * (pairs of CTAs, 256 rows), 128, 64 (fmm_fp8_matmul only) or 8 (the kernel for few tokens, fmm_fp8_matmul only); others get FMM_ERR_SHAPE.  shares: CTAs
 * that share the contraction of a tile, 1 to 4 (1 for 256 and 8).  columns 0: the library chooses again. */
fmm_status_t fmm_fp8_force_tile(int columns, int shares);

/* Status of these kernels on the current device, and its self-test, as fmm_int8_status and fmm_int8_selftest_bounded_wait. */
fmm_status_t fmm_fp8_status(int* code);
fmm_status_t fmm_fp8_status_clear(void);
fmm_status_t fmm_fp8_selftest_bounded_wait(int64_t limit_ns, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FMM_FP8_H */
