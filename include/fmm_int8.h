/*
 * fmm_int8.h - the 8-bit integer layer of the B200 (sm_100a) library of fmm.h: activations and weights in 8-bit
 * integers with fp32 scales, their product, the root-mean-square norm in front of it, and the gradients of both from
 * what is held in 8 bits.
 *
 * 8-bit form of a matrix X (rows x cols): codes (int8) and scales (fp32), one scale per row (block == 0) or per block
 * of `block` (32 or 128) consecutive columns of a row, the last block of a row being as short as it comes.  An element
 * stands for code * scale.  With a = max(max |x| over the block, 1e-12):
 *     FMM_INT8_SCALE_AMAX_DIV_127   scale = fl(a / 127),                      code = round(fl(x * fl(127 / a)))
 *     FMM_INT8_SCALE_POW2           scale = 2^e, e = ceil(log2(fl(a / 127))), code = round(x * 2^-e)
 * all in fp32, round() to the nearest integer, ties to even; |code| <= 127.  Values of power-of-two scales are exact in
 * bf16.  A block that holds an infinity or a NaN gets NaN as its scale.
 *
 * General rules
 *   - Status codes, "dev" pointers and streams as in fmm.h: nothing throws, aborts or traps the device, nothing is
 *     allocated or synchronised, work is only enqueued on `cuda_stream`, on the current device.  Calls may be captured
 *     into CUDA graphs.  Results do not depend on the run: no floating-point atomics, every sum in a fixed order.
 *   - Matrices are row-major; `ld*` is the distance between rows in elements, at least the number of columns.  Any
 *     alignment that their type allows is accepted where nothing else is said (16-byte aligned rows are read and
 *     written fastest).  Nothing is written behind the last column of a row, and nothing read but what shares an
 *     aligned 16-byte vector with an element of the row.
 *   - Rows and columns may be 0: then nothing is read, and what an empty sum gives is written.  They are below
 *     2^31 - 16384 (FMM_ERR_SHAPE).
 *   - An output may not overlap an input or another output, except where it is said.
 *   - workspace: dev, 256-byte aligned, caller-owned; calls that share one must be stream-ordered.
 */
#ifndef FMM_INT8_H
#define FMM_INT8_H

#include "fmm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { FMM_INT8_SCALE_AMAX_DIV_127 = 0, FMM_INT8_SCALE_POW2 = 1 } fmm_int8_scale_t;
typedef enum { FMM_TYPE_F32 = 0, FMM_TYPE_BF16 = 1, FMM_TYPE_F16 = 2 } fmm_type_t;

/* 8-bit form of x (dev, rows x cols of `type`): codes (dev, rows x cols) and scales (dev, rows if block == 0, else
 * rows x ceil(cols / block), dense). */
typedef struct {
    fmm_type_t type;
    int block;
    fmm_int8_scale_t scale_mode;
    int64_t rows, cols;
    const void* x;        int64_t ldx;
    int8_t* codes;        int64_t ldc;
    float* scales;
} fmm_int8_quantize_t;
fmm_status_t fmm_int8_quantize(const fmm_int8_quantize_t* p, void* cuda_stream);

/* x = code * scale, taken in fp32 and rounded once to `type` (dev, rows x cols); codes and scales as above. */
typedef struct {
    fmm_type_t type;
    int block;
    int64_t rows, cols;
    const int8_t* codes;  int64_t ldc;
    const float* scales;
    void* x;              int64_t ldx;
} fmm_int8_dequantize_t;
fmm_status_t fmm_int8_dequantize(const fmm_int8_dequantize_t* p, void* cuda_stream);

/* Residual's addition, root-mean-square norm and 8-bit output, row by row:
 *     h = fl(x + residual)  (x itself where residual is NULL);  rstd = fl32(1 / sqrt(sum h^2 / cols + eps)), in fp64;
 *     codes, scales (one per row) = 8-bit form of fl(fl(h * rstd) * gain);
 *     checkpoint, checkpoint_scales = 8-bit form of h in blocks of checkpoint_block, FMM_INT8_SCALE_AMAX_DIV_127.
 *   x, residual, gain (cols), hidden: of `type`.  residual == NULL: no addition; hidden is then not written and may be
 *   NULL.  hidden receives h rounded to `type`; it may be the same matrix as x or as residual (same pointer and
 *   distance between rows).  rstd (rows) may be NULL.  checkpoint_block 0: no checkpoint, checkpoint and
 *   checkpoint_scales are not used.  eps finite, >= 0.  Of rows without columns nothing is written. */
typedef struct {
    fmm_type_t type;
    fmm_int8_scale_t scale_mode;
    int checkpoint_block;
    int64_t rows, cols;
    double eps;
    const void* x;        int64_t ldx;
    const void* residual; int64_t ldr;
    const void* gain;
    void* hidden;         int64_t ldh;
    int8_t* codes;        int64_t ldc;
    float* scales;
    float* rstd;
    int8_t* checkpoint;   int64_t ldk;
    float* checkpoint_scales;
} fmm_int8_rms_norm_t;
fmm_status_t fmm_int8_rms_norm(const fmm_int8_rms_norm_t* p, void* cuda_stream);

/* Gradients of that norm, the rounding to 8 bits counting as the identity (straight through).  With
 * xhat = checkpoint value * rstd and c = mean over the row of (dy * gain * xhat):
 *     dx = rstd * (dy * gain - xhat * c) + dresidual;     dgain = sum over the rows of dy * xhat   (fp32)
 *   dy, gain, dresidual (NULL: none), dx: of `type`.  dx, the gradient of x and of residual alike, may be the same
 *   matrix as dy or as dresidual.  block: 32 or 128, or 0 for one checkpoint scale per row. */
typedef struct {
    fmm_type_t type;
    int block;
    int64_t rows, cols;
    const void* dy;        int64_t ldy;
    const int8_t* checkpoint; int64_t ldk;
    const float* checkpoint_scales;
    const float* rstd;
    const void* gain;
    const void* dresidual; int64_t ldr;
    void* dx;              int64_t ldx;
    float* dgain;
} fmm_int8_rms_norm_backward_t;
fmm_status_t fmm_int8_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes);
fmm_status_t fmm_int8_rms_norm_backward(const fmm_int8_rms_norm_backward_t* p, void* workspace, size_t workspace_bytes,
                                        void* cuda_stream);

/* C = (A B^T) scaled by row and column, plus a bias: C[i][j] = acc * a_scales[i] * b_scales[j] + bias[j], the sum acc of
 * the products of codes being exact, the rest in fp32, rounded once to `type`.
 *   a dev, M x K codes (tokens); b dev, N x K codes (a weight, one row per output channel); c dev, M x N; bias dev, N of
 *   `type`, or NULL.  a and b 16-byte aligned, lda and ldb multiples of 16 (FMM_ERR_INVALID_ARG; the codes that
 *   fmm_int8_quantize and fmm_int8_rms_norm write may have any such ld); K <= 131071, so that no sum leaves 32 bits
 *   (FMM_ERR_SHAPE). */
typedef struct {
    fmm_type_t type;
    int64_t M, N, K;
    const int8_t* a;      int64_t lda;
    const float* a_scales;
    const int8_t* b;      int64_t ldb;
    const float* b_scales;
    const void* bias;
    void* c;              int64_t ldc;
} fmm_int8_matmul_t;
fmm_status_t fmm_int8_matmul(const fmm_int8_matmul_t* p, void* cuda_stream);

/* Gradients of that product for dy (dev, M x N of `type`, FMM_TYPE_BF16 or FMM_TYPE_F16), from what is held in 8 bits; products
 * are summed in fp32.
 *     fmm_int8_grad_weight: out[j][k] (+)= sum_i dy[i][j] * (codes[i][k] * scales[i])      codes M x K, out N x K
 *     fmm_int8_grad_input:  out[i][k] (+)= sum_j dy[i][j] * (codes[j][k] * scales[j])      codes N x K, out M x K
 *   out: dev, of out_type, FMM_TYPE_F32 or dy's type; accumulate != 0 adds to what it holds.
 *   Values.  code * scale is a number of fp32.  The tensor cores take 16-bit numbers, so a value is multiplied in parts of dy's type:
 *     out_type FMM_TYPE_F32   bf16: three parts, nothing is lost; fp16: two, 2^-21 of the value (or 2^-32 of the largest scale)
 *     out_type that of dy     two parts: bf16 2^-15, fp16 as above; but fmm_int8_grad_input of bf16 takes the codes, which are exact, and
 *                             dy * scale in half precision: 2^-11 of it, or 2^-39 of the largest in its row (out's rounding: 2^-8)
 *   Where the scales of 64 consecutive rows (the first a multiple of 64) are powers of two, one part is the value and the others are left
 *   out: with FMM_INT8_SCALE_POW2 a gradient takes a third (FMM_TYPE_F32, bf16) or half of the time.  fp16 parts carry a power of two
 *   for the whole matrix, so that values beyond fp16's range, as 64 * 1024 for an activation of 65504, do not leave it.
 *   rounded != 0: one part in any case, the value rounded once to dy's type (2^-8 of it for bf16, 2^-11 for fp16).
 *   An infinity or NaN, of dy or of a scale, reaches what it is a term of, as in the product of the values.  (A dy * scale beyond fp32 counts
 *   as infinite in the bf16 input gradient.)
 *   The workspace holds the values' parts and, where its rows are not 16-byte aligned or it is scaled, a copy of dy (FMM_ERR_SHAPE
 *   where that could be 2^46 bytes or more); its size is asked for with the same arguments (of which the matrices' own addresses but dy's
 *   do not matter). */
typedef struct {
    fmm_type_t type, out_type;
    int accumulate, rounded;
    int64_t M, N, K;
    const void* dy;       int64_t ldy;
    const int8_t* codes;  int64_t ldc;
    const float* scales;
    void* out;            int64_t ldo;
} fmm_int8_grad_t;
fmm_status_t fmm_int8_grad_weight_workspace_bytes(const fmm_int8_grad_t* p, size_t* bytes);
fmm_status_t fmm_int8_grad_input_workspace_bytes(const fmm_int8_grad_t* p, size_t* bytes);
fmm_status_t fmm_int8_grad_weight(const fmm_int8_grad_t* p, void* workspace, size_t workspace_bytes, void* cuda_stream);
fmm_status_t fmm_int8_grad_input(const fmm_int8_grad_t* p, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* How a product or gradient is multiplied, for tests and measurements. */
typedef struct {
    int kernel;                  /* 1: persistent CTA pairs (columns 256, k_shares 1); 2: a cluster of k_shares CTAs a tile;
                                    3: few tokens (products of up to eight; columns 8, k_shares 1) */
    int columns;                 /* cluster: of a tile: products 16, 32, 64, 128; gradients 64, 128 */
    int k_shares;                /* cluster: CTAs that share the contraction, 1 to 8, each a stage (128 codes, 64 numbers) at least */
} fmm_int8_product_shape_t;
typedef enum { FMM_INT8_MATMUL = 0, FMM_INT8_GRAD_WEIGHT = 1, FMM_INT8_GRAD_INPUT = 2 } fmm_int8_product_t;
/* The shape that a call of this size takes on the current device (M, N, K > 0, as the call has them; out_type: of its output). */
fmm_status_t fmm_int8_product_shape(fmm_int8_product_t which, int64_t M, int64_t N, int64_t K, fmm_type_t out_type, fmm_int8_product_shape_t* shape);
/* From now on every call of the calling host thread takes `shape` instead of the one that the library expects to be fastest; NULL: the
 * library chooses again.  FMM_ERR_INVALID_ARG for a shape that does not exist; a call that cannot be multiplied that way (more tokens
 * than few, more shares than stages, columns that its kind does not have) returns FMM_ERR_SHAPE. */
fmm_status_t fmm_int8_force_product_shape(const fmm_int8_product_shape_t* shape);

/* Status of the product kernels on the current device, read after cudaDeviceSynchronize: *code == 0, or the location of
 * the first bounded device-side wait that gave up (FMM_ERR_DEVICE_TIMEOUT; the results of that call are invalid).
 * Debug build (fmm_debug_build): also the first store outside the ranges that a launch was given. */
fmm_status_t fmm_int8_status(int* code);
fmm_status_t fmm_int8_status_clear(void);
/* Self-test of that status: enqueues a one-warp kernel that waits, with the products' bounded-wait routine, on a barrier that nothing
 * signals; after limit_ns (1 .. 2e9) it gives up and records location 901.  Look up the status once before capturing this. */
fmm_status_t fmm_int8_selftest_bounded_wait(int64_t limit_ns, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* FMM_INT8_H */
