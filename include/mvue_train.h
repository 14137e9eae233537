/*
 * mvue_train.h -- what a training step needs around the pruned products of mvue.h:
 * the AdamW step over many tensors that takes the dW the update products leave, group
 * normalisation with an activation on channels-last maps (its backward pass hands the
 * neural gradient to mvue_prune), and embedding lookup with its gradient (which takes the
 * dh of the last backward product).
 *
 * The general rules of mvue.h hold (device pointers, caller-owned buffers, work enqueued on `stream`, argument
 * errors found on the host before anything is launched), with these differences: empty extents are accepted where a
 * call says so, and tensors need no more than the alignment of their element type -- 32-byte aligned buffers and
 * leading dimensions take the wide loads, others are slower.
 */
#ifndef MVUE_TRAIN_H_
#define MVUE_TRAIN_H_

#include "mvue.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------------------------------------------
 * AdamW over many tensors
 * --------------------------------------------------------------------------------------------------------------- */

/* Elements that share one scale of the 8-bit states. */
#define MVUE_ADAMW_BLOCK 256

/* One tensor of the step: numel elements, contiguous (any order of dimensions that is the same in all its buffers).
 *  param      MVUE_F32 or MVUE_BF16 (param_dtype), updated in place.
 *  master     optional float copy of a bf16 param: the step reads and updates the copy, and param receives it rounded
 *             to the nearest bf16 (param itself is not read).  NULL otherwise; an MVUE_F32 param takes none.
 *  grad       MVUE_F32 or MVUE_BF16 (grad_dtype), read only.
 *  exp_avg, exp_avg_sq   state_bits = 32: float m and v.
 *             state_bits = 8: one byte per element, 8-bit floats of four exponent and three mantissa bits (e4m3) of m
 *             and of sqrt(v), in units of exp_avg_scale / exp_avg_sq_scale: one float for each MVUE_ADAMW_BLOCK
 *             consecutive elements (the last block of a tensor may be short).  All zero bytes and scales = zero state.
 * Buffers of one call must not overlap. */
typedef struct {
    void* param;
    void* master;
    const void* grad;
    void* exp_avg;
    void* exp_avg_sq;
    void* exp_avg_scale;
    void* exp_avg_sq_scale;
    int64_t numel;
    int32_t param_dtype;
    int32_t grad_dtype;
} mvue_adamw_tensor;

/* The step (step = t >= 1), in binary32; constants are formed in double on the host:
 *   g' = g * grad_scale (* *dev_grad_scale)
 *   m' = beta1 m + (1 - beta1) g'
 *   v' = beta2 v + ((1 - beta2) g') g'
 *   param' = param (1 - lr weight_decay) - (lr / (1 - beta1^t)) * (m' / (sqrt(v') / sqrt(1 - beta2^t) + eps))
 * m' and v' with each operation rounded on its own; the root and the quotient within 2 units in the last place (with 8-bit states
 * a root below 2^-63 may count as 0 where it is lost beside eps), the product by the decay fused with the sum.  (|g'| above 2^63 overflows v'.)
 * grad_scale: HOST value, 1 for none; dev_grad_scale: optional DEVICE float (a clipping factor or a loss scale's
 * inverse that the host does not know), read when the step runs.
 * state_bits: 32 or 8.  With 8 bits the new m and sqrt(v) of a block are divided by the block's new scale
 * top / 448 (top the largest magnitude; the new scale is top * fl(1/448), the factor 448 * fl(1/top), a magnitude
 * is capped at 448) and rounded to a neighbouring code at random so that the code's expectation is the value: an
 * average that moves by a thousandth per step, less than a hundredth of the distance of two codes, would otherwise never move.
 * (The magnitude in steps of its binade, of 2^-9 below 2^-6, plus the random number, in binary32, is cut to whole steps.)
 * sqrt(v') is the root rounded to the nearest binary32 number here.  A non-zero v keeps a code of at least the smallest.
 * Blocks whose largest |m| is below 2^-110 store zeros; a non-finite value makes its block's scale NaN.
 * options: MVUE_OPT_STOCHASTIC_ROUNDING: a bf16 param without master is rounded to bf16 stochastically (as the
 * survivors of mvue_prune_opts) instead of to the nearest -- updates below half a unit in the last place then count in
 * the mean.  Other bits: MVUE_ERR_OPTION.
 * The random bits: the tensors of a call, each padded to a multiple of MVUE_ADAMW_BLOCK elements, are numbered through
 * in order; elements 8u .. 8u + 7 take the eight halves (low first) of the words of Philox4x32-10 with counter
 * (lo32(u), hi32(u), 2, 0) under the key `seed` (pass another one each step).  The param takes the 16 bits as they are, the two
 * states the same bits with their bytes exchanged.  Equal inputs and seed give equal bits. */
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;
    double grad_scale;
    const float* dev_grad_scale;
    uint64_t seed;
    int32_t state_bits;
    uint32_t options;
} mvue_adamw_config;

/* tensors: HOST array of `count` entries (count = 0 and numel = 0 are accepted and do nothing); it may be freed on
 * return.  Errors: MVUE_ERR_NULL, MVUE_ERR_DTYPE (a dtype, a master beside an MVUE_F32 param, state_bits),
 * MVUE_ERR_SHAPE (negative count or numel, step < 1, more than 2^31 - 1 tiles of 2048 elements), MVUE_ERR_ALIGN
 * (a pointer not aligned to its element), MVUE_ERR_OPTION (an unknown bit; a beta outside [0, 1)). */
MVUE_API int mvue_adamw_step(const mvue_adamw_tensor* tensors, int64_t count, const mvue_adamw_config* config, void* stream);

/* ---------------------------------------------------------------------------------------------------------------
 * Embedding
 * --------------------------------------------------------------------------------------------------------------- */

/* out[t] = scale * W[ids[t]] for t < tokens (tokens = 0: nothing).
 *  ids      device integers of id_bits = 32 or 64 bits.  An id outside [0, vocab) gives a row of zeros and writes
 *           MVUE_ERR_INDEX to *dev_status (optional device int, otherwise left untouched).
 *  W        [vocab x cols], MVUE_F32 or MVUE_BF16, ldW >= cols;  out [tokens x cols], MVUE_F32 or MVUE_BF16, ldout >= cols.
 * The product is formed in binary32 and rounded once.  Rows whose base, cols and leading dimension are multiples of eight
 * elements (16 bytes of bf16, 32 of fp32) are moved in pieces of eight, others in pairs or element by element. */
MVUE_API int mvue_embedding(const void* ids, int id_bits, int64_t tokens, const void* W, int w_dtype, int64_t vocab, int64_t cols,
                            int64_t ldW, float scale, void* out, int out_dtype, int64_t ldout, int* dev_status, void* stream);

/* The lookup's gradient: dW[v] (+)= scale * sum of dy[t] over the tokens with ids[t] = v, for all v < vocab; rows that no
 * token names are zero (accumulate != 0: dW is added to, MVUE_F32 only, and rows that no token names are not touched).
 *  dy       [tokens x cols], MVUE_F32 or MVUE_BF16;  dW [vocab x cols], MVUE_F32 or MVUE_BF16.
 *  padding_idx   tokens with this id add nothing (a negative one: none does so).  Ids outside [0, vocab) add nothing and
 *           write MVUE_ERR_INDEX to *dev_status (optional).
 *  workspace     mvue_embedding_grad_workspace_bytes(tokens, cols) bytes, 32-byte aligned; contents scratch.
 * Sums are formed in binary32: the list sorted by id is cut into runs of 4 to 32 tokens (by the number of tokens), a run's
 * rows are added in token order and an id's runs in a fixed order: equal inputs give equal bits.  tokens = 0 gives zeros. */
MVUE_API int mvue_embedding_grad(const void* ids, int id_bits, int64_t tokens, const void* dy, int dy_dtype, int64_t cols, int64_t lddy,
                                 float scale, int64_t padding_idx, void* dW, int dW_dtype, int64_t vocab, int64_t lddW, int accumulate,
                                 void* workspace, size_t workspace_bytes, int* dev_status, void* stream);
MVUE_API int mvue_embedding_grad_workspace_bytes(int64_t tokens, int64_t cols, size_t* bytes);   /* bytes: HOST */

/* ---------------------------------------------------------------------------------------------------------------
 * Group normalisation with an activation, channels last
 * --------------------------------------------------------------------------------------------------------------- */

/* GELU: z times the normal distribution function of z (not its tanh approximation). */
typedef enum { MVUE_ACT_NONE = 0, MVUE_ACT_RELU = 1, MVUE_ACT_SILU = 2, MVUE_ACT_GELU = 3 } mvue_act;

/* x [n, s, c] (s positions of c channels; c a multiple of groups, cg = c / groups), over each group of cg neighbouring
 * channels of a sample:
 *   mean = sum x / (s cg);  rstd = 1 / sqrt(sum (x - mean)^2 / (s cg) + eps)
 *   z = (x - mean) rstd gamma_c + beta_c;  y = act(z)
 *  x, y       MVUE_F32 or MVUE_BF16 (the same); ldx, ldy >= c: elements between positions; a sample has s of them.
 *             y may be x.
 *  gamma, beta   [c], MVUE_F32 or MVUE_BF16 (affine_dtype), either may be NULL (ones, zeros).
 *  mean, rstd [n, groups] float outputs for the backward pass, either may be NULL.
 *  workspace  mvue_group_norm_workspace_bytes(n, s, c, groups) bytes, 16-byte aligned; contents scratch.  A call that
 *             gives mean and rstd and whose samples stay in shared memory (x and y aligned for wide accesses, whole groups
 *             that fit eight thread blocks) uses none and accepts NULL; others return MVUE_ERR_WORKSPACE without it.
 *  dev_status optional device int, receives MVUE_ERR_DEVICE_TIMEOUT if a bounded wait between the blocks of a cluster expires;
 *             otherwise left untouched.  What depended on the wait is NaN then: y, mean and rstd of the samples concerned, or dx
 *             in the backward pass.
 * Arithmetic in binary32; the output is rounded once.  n = 0: nothing.  s >= 1. */
MVUE_API int mvue_group_norm_act(const void* x, int dtype, int64_t n, int64_t s, int64_t c, int64_t ldx, int groups, const void* gamma,
                                 const void* beta, int affine_dtype, float eps, int act, void* y, int64_t ldy, float* mean, float* rstd,
                                 void* workspace, size_t workspace_bytes, int* dev_status, void* stream);

/* Its backward pass, z formed again from x and the forward pass's mean and rstd:
 *   dz = dy act'(z);  dbeta_c = sum dz;  dgamma_c = sum dz xh, xh = (x - mean) rstd   (over n and s)
 *   dx = rstd (gamma_c dz - mean over the group of gamma dz - xh * mean over the group of gamma dz xh)
 * (the derivative of ReLU at 0 is 0).  dgamma, dbeta: [c] float, either may be NULL; n = 0 sets them to zero.  dx is what
 * mvue_prune takes as the neural gradient of the layer below.  dx may be dy.  Equal inputs give equal bits. */
MVUE_API int mvue_group_norm_act_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int dtype, int64_t n, int64_t s,
                                          int64_t c, int groups, const float* mean, const float* rstd, const void* gamma,
                                          const void* beta, int affine_dtype, int act, void* dx, int64_t lddx, float* dgamma,
                                          float* dbeta, void* workspace, size_t workspace_bytes, int* dev_status, void* stream);
MVUE_API int mvue_group_norm_workspace_bytes(int64_t n, int64_t s, int64_t c, int groups, size_t* bytes);   /* bytes: HOST */

/* Self-test of that bounded wait.  One forward launch (dy = NULL) or one backward launch, without affine and activation and
 * with eps = 1, on contiguous tensors whose samples stay in the shared memory of two or more thread blocks (else
 * MVUE_ERR_SHAPE), in which the blocks send one another nothing: every wait gives up after `polls` polls
 * (1 <= polls <= 65536, else MVUE_ERR_SHAPE; each takes about 4 us) and the blocks leave the ordinary way.
 * MVUE_ERR_DEVICE_TIMEOUT is written to *dev_status (required) and NaN to the outputs.  Nothing is in flight, nothing
 * traps or faults, and the next call must be correct.  The other arguments are those of the two calls above. */
MVUE_API int mvue_selftest_group_norm_timeout(int polls, const void* x, const void* dy, int dtype, int64_t n, int64_t s, int64_t c,
                                              int groups, float* mean, float* rstd, void* out, void* workspace,
                                              size_t workspace_bytes, int* dev_status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MVUE_TRAIN_H_ */
