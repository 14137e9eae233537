/*
 * mvue_layer.h -- the rest of a layer's own arithmetic beside the pruned products of mvue.h: layer normalisation and its
 * backward pass, the dense products (the forward product, and the backward product where the gradient is not pruned) in
 * 8-bit floating point with block scales, and the quantiser that feeds them.
 *
 * The rules of mvue_train.h hold: device pointers, caller-owned buffers, work enqueued on `stream`, argument errors found on
 * the host before anything is launched, tensors aligned to their element type unless a call says more.
 *
 * And the Muon step, for the weights that are matrices: it takes the dW of the update products as mvue_adamw_step does.
 */
#ifndef MVUE_LAYER_H_
#define MVUE_LAYER_H_

#include "mvue_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------------------------------------------
 * Layer normalisation
 * --------------------------------------------------------------------------------------------------------------- */

/* For each row of x [rows, cols]:
 *   mean = sum x / cols;  rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps);  y_c = (x_c - mean) rstd gamma_c + beta_c
 *  x, y       MVUE_F32 or MVUE_BF16 (the same); ldx, ldy >= cols.  y may be x.
 *  gamma, beta   [cols], MVUE_F32 or MVUE_BF16 (affine_dtype), either may be NULL (ones, zeros).
 *  mean, rstd [rows] float outputs for the backward pass, either may be NULL.
 * Arithmetic in binary32; the output is rounded once.  Its range is the row's, too: where the sum of squares about the mean overflows (elements
 * about 2^64 / sqrt(cols) from it) rstd is 0 and y beta, where the sum of the elements does y may be NaN; squares below 2^-149 count as nothing
 * beside eps.  rows = 0: nothing.  cols >= 1. */
MVUE_API int mvue_layer_norm(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* gamma, const void* beta,
                             int affine_dtype, float eps, void* y, int64_t ldy, float* mean, float* rstd, void* stream);

/* Its backward pass, from x and the forward pass's mean and rstd; xh = (x - mean) rstd, sums over a row's columns:
 *   dx_c = rstd (gamma_c dy_c - sum(gamma dy) / cols - xh_c sum(gamma dy xh) / cols)
 *   dgamma_c = sum over rows of dy_c xh_c;  dbeta_c = sum over rows of dy_c
 *  dgamma, dbeta   [cols] float, either may be NULL; rows = 0 sets them to zero.
 *  workspace  mvue_layer_norm_workspace_bytes(rows, cols) bytes, 16-byte aligned; contents scratch.  None is needed without
 *             dgamma and dbeta.
 * dx may be dy or x (and is what mvue_prune takes as the neural gradient of the layer below).  Equal inputs give equal bits. */
MVUE_API int mvue_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int dtype, int64_t rows, int64_t cols,
                                      const float* mean, const float* rstd, const void* gamma, int affine_dtype, void* dx, int64_t lddx,
                                      float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream);
MVUE_API int mvue_layer_norm_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes);   /* bytes: HOST */

/* ---------------------------------------------------------------------------------------------------------------
 * 8-bit floating point with block scales
 * --------------------------------------------------------------------------------------------------------------- */

/* Elements along the reduction axis of a product that share a scale (and, in a weight, along the other axis too). */
#define MVUE_SCALE_BLOCK 128

/* Codes of x [rows, cols] (MVUE_F32 or MVUE_BF16, ldx >= cols) as 8-bit floats of four exponent and three mantissa bits (e4m3:
 * largest 448, no infinities, 0x7F and 0xFF are NaN), one scale for each block of block_rows x 128 elements (block_rows 1 or 128;
 * blocks at the right and lower edges may be short):
 *   scale = 2^(e - 127), e the least byte >= 1 for which the block's largest finite magnitude is at most 448 scale
 *   code = e4m3(x / scale), to the nearest, ties to even
 * Elements that are infinite or NaN get a NaN code and do not count for the scale.
 *  codes      [rows, cols] bytes, ldq >= cols (the products want codes 16-byte aligned and ldq a multiple of 16).
 *  scales     exponent bytes e: [ceil(cols / 128), rows] for block_rows = 1 (a block's rows are neighbours),
 *             [ceil(rows / 128), ceil(cols / 128)] for block_rows = 128.
 * options: MVUE_OPT_STOCHASTIC_ROUNDING rounds without bias: with z = |x| / scale cut (to the nearest) to a multiple of 2^-20 of the
 * distance of the two codes around it, the larger code is taken where the fraction of that distance plus r 2^-16 reaches one, and the
 * expectation is z.  r: elements 8j .. 8j + 7 of row i take the eight halves (low first) of the words of Philox4x32-10 with counter
 * (lo32(u), hi32(u), 3, 0), u = i ceil(cols / 8) + j, under the key `seed` (pass another one each step).  Other bits: MVUE_ERR_OPTION.
 * rows = 0 or cols = 0: nothing. */
MVUE_API int mvue_quantize_e4m3(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int block_rows, unsigned options,
                                uint64_t seed, void* codes, int64_t ldq, void* scales, void* stream);

/* Products of such codes, each multiplied by its scale, summed in binary32 on the tensor cores and rounded once to the output type:
 *   forward    C[tokens x out] = x W^T     x [tokens, in] with one scale per 1 x 128, W [out, in] with one per 128 x 128
 *   backward   C[tokens x in]  = g W       g [tokens, out] with one scale per 1 x 128, the same W and scales
 *  x, g, W    e4m3 codes, 16-byte aligned, leading dimensions multiples of 16 bytes (MVUE_ERR_ALIGN); any extents.
 *  scales     as mvue_quantize_e4m3 leaves them; the byte 255 stands for NaN.
 *  C          MVUE_F32 or MVUE_BF16, ldc >= its columns; 32-byte aligned rows take the wide stores.
 *  dev_status optional device int, receives MVUE_ERR_DEVICE_TIMEOUT if a bounded wait expires (the tiles of C that it was for are NaN then);
 *             otherwise left untouched.
 * tokens = 0: nothing.  Equal inputs give equal bits.  The tensor core cuts off what an addition has below the sum's last place: sums of one
 * sign over 150,000 terms come out 5e-5 too small, over 2^20 terms 1.5e-3; up to 65,000 nothing is seen. */
MVUE_API int mvue_scaled_forward_gemm(const void* x, const void* x_scales, int64_t tokens, int64_t in, int64_t ldx, const void* W,
                                      const void* W_scales, int64_t out, int64_t ldW, void* C, int c_dtype, int64_t ldc, int* dev_status,
                                      void* stream);
MVUE_API int mvue_scaled_backward_gemm(const void* g, const void* g_scales, int64_t tokens, int64_t out, int64_t ldg, const void* W,
                                       const void* W_scales, int64_t in, int64_t ldW, void* C, int c_dtype, int64_t ldc, int* dev_status,
                                       void* stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Muon
 * --------------------------------------------------------------------------------------------------------------- */

/* The polynomial 3.4445 s - 4.7750 s^3 + 2.0315 s^5 applied ns_steps times (1 .. 16) to the singular values of x / (||x|| + 1e-7),
 * ||x|| the root of the sum of squares: five steps bring those above a hundredth or so between 0.7 and 1.2 and leave the
 * singular vectors as they are.
 *   X = x / (||x|| + 1e-7);  ns_steps times:  A = X X^T,  X = 3.4445 X + (-4.7750 A + 2.0315 A A) X
 * (X^T X where rows > cols).  Products of binary16 values with binary32 sums, the first term with the others (3.4445 I - 4.7750 A + 2.0315 A A
 * is one matrix); in all steps but the last two the first term is taken from 22 bits of X.  Against exact arithmetic, five steps:
 * 1e-3 to 3e-3 of the result's norm from sixteen rows and columns on, whatever the spectrum.  Below, the result hangs on a few singular values, and
 * one may lie where the polynomials are steep: 2e-3 to 3e-3 as a rule, but up to 7e-3 with eight rows or columns, 1e-2 with four, 2e-2 with two.
 * A matrix with an element that is not finite becomes NaN throughout.
 *  x          [batch, rows, cols], MVUE_F32 or MVUE_BF16, ldx >= cols, x_stride elements between matrices.
 *  out        the same, MVUE_F32 or MVUE_BF16; matrices do not overlap.  It may be x, with x's type, ldx and x_stride.
 *  workspace  mvue_orthogonalize_workspace_bytes(batch, rows, cols) bytes, 256-byte aligned; contents scratch.
 *  dev_status optional device int, receives MVUE_ERR_DEVICE_TIMEOUT if a bounded wait expires (matrices it was for are NaN then); otherwise
 *             left untouched.
 * min(rows, cols) <= 2^17, max(rows, cols) <= 2^20 (MVUE_ERR_SHAPE): sums of more terms would be further off than that.  An empty extent:
 * nothing.  Equal calls give equal bits; how the sums of X X^T are split depends on how many matrices of the same extents a call has, so a
 * matrix of 1024 columns or more (rows, where it has more) may differ by roundings between a call of its own and one with others. */
MVUE_API int mvue_orthogonalize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ldx, int64_t x_stride, int ns_steps,
                                void* out, int out_dtype, int64_t ldo, int64_t out_stride, void* workspace, size_t workspace_bytes,
                                int* dev_status, void* stream);
MVUE_API int mvue_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, size_t* bytes);   /* bytes: HOST */

/* One matrix of the step: rows x cols, contiguous.
 *  param      MVUE_F32 or MVUE_BF16 (param_dtype), updated in place.
 *  master     optional float copy of a bf16 param, as in mvue_adamw_tensor.
 *  grad       MVUE_F32 or MVUE_BF16 (grad_dtype), read only.
 *  momentum   float, updated in place.
 * Buffers of one call must not overlap. */
typedef struct {
    void* param;
    void* master;
    const void* grad;
    void* momentum;
    int64_t rows, cols;
    int32_t param_dtype;
    int32_t grad_dtype;
} mvue_muon_tensor;

typedef enum {
    MVUE_MUON_SCALE_RMS = 0,      /* 0.2 sqrt(max(rows, cols)): the update is as large as AdamW's */
    MVUE_MUON_SCALE_SHAPE = 1     /* sqrt(max(1, rows / cols)) */
} mvue_muon_scale;

#define MVUE_OPT_NESTEROV 16u

/* The step:
 *   g' = g * grad_scale (* *dev_grad_scale);  M' = momentum M + (1 - momentum) g'
 *   U = M', or with MVUE_OPT_NESTEROV momentum M' + (1 - momentum) g'
 *   param' = param (1 - lr weight_decay) - lr scale orthogonalize(U)          (scale: scale_rule)
 * Arithmetic in binary32 outside the products.  options: MVUE_OPT_NESTEROV; MVUE_OPT_STOCHASTIC_ROUNDING rounds a bf16 param without
 * master stochastically, with the random numbers of mvue_adamw_step (matrices of a call numbered through in order, each padded to a
 * multiple of 256 elements).  Other bits: MVUE_ERR_OPTION. */
typedef struct {
    double lr, momentum, weight_decay, grad_scale;
    const float* dev_grad_scale;
    uint64_t seed;
    int32_t ns_steps;
    int32_t scale_rule;
    uint32_t options;
} mvue_muon_config;

/* tensors: HOST array of `count` entries (0, and empty matrices, are accepted); it may be freed on return.  Matrices of equal extents go
 * through the products together, up to 64 and 2^27 elements at a time; extents and bits as in mvue_orthogonalize.  workspace:
 * mvue_muon_workspace_bytes(tensors, count) bytes (only the extents are looked at), 256-byte aligned; contents scratch.  Errors as mvue_adamw_step's, MVUE_ERR_WORKSPACE beside them. */
MVUE_API int mvue_muon_step(const mvue_muon_tensor* tensors, int64_t count, const mvue_muon_config* config, void* workspace,
                            size_t workspace_bytes, int* dev_status, void* stream);
MVUE_API int mvue_muon_workspace_bytes(const mvue_muon_tensor* tensors, int64_t count, size_t* bytes);   /* bytes: HOST */

#ifdef __cplusplus
}
#endif
#endif /* MVUE_LAYER_H_ */
