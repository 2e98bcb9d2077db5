/*
 * clq_block.h -- C ABI of the operators around the 8-bit linears of a transformer block
 * (libclq.so, AMD Instinct MI355X, gfx950): RMS norm with the residual's addition, its result in
 * 16 or 32 bits or rotated and in 8 bits; rotary positions with several axes; the 8-bit linear with
 * activation, gate and residual in its epilogue.
 *
 * Conventions are those of clq.h: device pointers, caller-owned buffers, checks on the host before
 * anything is enqueued, no synchronisation, no allocation, CLQ_ERR_* statuses.  clq_type is that of
 * clq_mx4.h.  Arithmetic is fp32, each output rounded once.
 *   - Shapes: 1 <= M, N < 2^31; K as each entry point says.  Row strides are in elements, at least
 *     the row length and multiples of 8.
 *   - Matrices and codes are 16-byte aligned; scales, positions and perm 4-byte; freqs 8-byte; bias
 *     2-byte.
 *   - Samples: a matrix with one row for each of `samples` equal runs of the M rows (M % samples == 0);
 *     row r of M belongs to sample r / (M / samples).
 *   - An output may be an input itself (same address, stride and type: in place) where the entry point
 *     says so, and must not overlap what the call reads otherwise.
 */
#ifndef CLQ_BLOCK_H
#define CLQ_BLOCK_H

#include "clq_mx4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- RMS norm ------------------------------------------------------------------------
 *   s = X + R,   n = s / sqrt(mean(s^2) + eps) * W[sample]
 *   X        fp16, bf16 or fp32 [M][K], row stride ldx.
 *   R        the residual stream, fp16, bf16 or fp32 [M][K], row stride ldr; NULL: none (then sum is
 *            NULL too).
 *   W        fp16, bf16 or fp32 [samples][K], contiguous; NULL: ones (samples 1).
 *   eps      finite, 2^-126 at least.
 *   sum      out, s rounded to R's type, row stride ld_sum; may be R, in place.  The norm is that of s
 *            before this rounding.
 * A row that holds a NaN or an infinity gives NaN where s / infinity is one and, in the 8-bit form, a
 * NaN scale.  Squares are summed in fp32: a row whose sum of them reaches 2^128 (a root mean square of
 * 2^64 / sqrt(K), 2^61 at K = 64 and 2^57 at K = 16384) counts as infinitely large: zeros, in the 8-bit form
 * codes with a scale of 0, or a NaN one where its rotation passes fp32's range too.  In the 8-bit form rows
 * whose rotated s W stays under 2^-119 are zeros. */

/* Y = n in fp16, bf16 or fp32, row stride ldy; may be X, in place.  8 <= K <= 16384, K % 8 == 0. */
clq_status clq_rms_norm(const void *X, clq_type x_type, int64_t ldx, const void *R, clq_type r_type, int64_t ldr,
                        const void *W, clq_type w_type, int64_t samples, float eps, int64_t M, int64_t K, void *Y,
                        clq_type y_type, int64_t ldy, void *sum, int64_t ld_sum, hipStream_t stream);

/* n rotated and quantized as clq_rotate_quant_act8 does: x~ = FWHT_block(gather(n, perm)),
 * x_scale = max|x~| / 127, codes rne(127 x~ / max|x~|).  n is not rounded in between.
 *   64 <= K <= 16384, K % 64 == 0; block 32, 64 or 128, dividing K; perm int32 [K] or NULL.
 *   Xq8      out, clq_act8_bytes(M, K) bytes; x_scale out, fp32 [M]. */
clq_status clq_rms_norm_act8(const void *X, clq_type x_type, int64_t ldx, const void *R, clq_type r_type, int64_t ldr,
                             const void *W, clq_type w_type, int64_t samples, float eps, const int32_t *perm,
                             int64_t M, int64_t K, int32_t block, void *Xq8, float *x_scale, void *sum, int64_t ld_sum,
                             hipStream_t stream);

/* clq_rotate_quant_act8 of fp16, bf16 or fp32 activations (the results of an activating linear, say, that
 * were not rounded to 16 bits): the same codes and scales for finite fp16 values.  A NaN in a row, and an
 * infinity with its opposite or another in one block, give a NaN scale, a lone infinity an infinite one; rows
 * whose rotation stays under 2^-119 are zeros.  Shapes as above. */
clq_status clq_quantize_act8(const void *X, clq_type x_type, int64_t ldx, const int32_t *perm, int64_t M, int64_t K,
                             int32_t block, void *Xq8, float *x_scale, hipStream_t stream);

/* The values that 8-bit codes and their scales stand for (still rotated): out [M][K] of `type`, row
 * stride ldo.  64 <= K <= 32768, K % 64 == 0. */
clq_status clq_dequantize_act8(const void *Xq8, const float *x_scale, int64_t M, int64_t K, clq_type type, void *out,
                               int64_t ldo, hipStream_t stream);

/* ---- rotary positions -------------------------------------------------------------------
 * Turns pairs of a head's first 2 P columns, P = pair_ends[axes - 1]: pair i by the angle
 *   positions[row % tokens][axis(i)] * freqs[i],
 * axis(i) the first axis a with i < pair_ends[a]:
 *   (a, b) -> (a cos - b sin, b cos + a sin).
 *   X        fp16 or bf16 [M][heads][D], strides ldx (row) and lhx (head), multiples of 8; D % 8 == 0,
 *            D <= 256, heads <= 2^20.  Heads may be columns of a wider row (queries and keys of one projection).
 *   positions  int32 or fp32 [tokens][axes] (position_type: 0 int32, 1 fp32), M % tokens == 0.
 *   freqs    fp64 [P], radians a position.  Angles are formed and reduced in fp64.
 *   pair_ends  host int32 [axes], 1 <= axes <= 4, ascending, the last a multiple of 4, 2 P <= D.
 *   interleaved  1: pair i is columns 2i, 2i + 1; 0: columns i, i + P.
 *   inverse  1: by the opposite angle (the transpose).
 *   W        NULL, or fp16, bf16 or fp32 weights of an RMS norm of each head (all D columns) ahead of the
 *            turn, [D] (weight_heads 1) or [heads][D] (weight_heads = heads), contiguous; eps as for the norm, and
 *            so its limit: a head whose squares add up to 2^128 is zeros.
 *   Y        out, X's type, strides ldy and lhy, no value of it in two places of the head's rows; may be X,
 *            in place. */
clq_status clq_rope_axes(const void *X, clq_type type, int64_t ldx, int64_t lhx, const void *positions,
                         int32_t position_type, int64_t tokens, const double *freqs, const int32_t *pair_ends,
                         int32_t axes, int32_t interleaved, int32_t inverse, const void *W, clq_type w_type,
                         int64_t weight_heads, float eps, int64_t M, int64_t heads, int64_t D, void *Y, int64_t ldy,
                         int64_t lhy, hipStream_t stream);

/* ---- 8-bit linear with epilogue ----------------------------------------------------------
 *   Y = R + gate[sample] * act(dequant(Xq8 . Wq^T) + bias)
 * on the operands of clq_a8_linear (wbits 4 or 8, 64 <= K <= 32768, K % 64 == 0; fewer than 2^24 tiles of
 * 256 tokens x 128 channels).
 *   bias     fp16 or bf16 [N], or NULL.
 *   act      CLQ_ACT_NONE, CLQ_ACT_GELU (tanh form) or CLQ_ACT_SILU; ARG for CLQ_ACT_SWIGLU.
 *   gate     fp16, bf16 or fp32 [samples][N], contiguous, or NULL (samples 1).
 *   R        the residual stream, of the output's type [M][N], row stride ldr >= N (any), or NULL.
 *   Y        out, fp16, bf16 or fp32, row stride ldy; may be R, in place. */
#define CLQ_ACT_SILU 3 /* h / (1 + exp(-h)) */
clq_status clq_a8_linear_act(const void *Xq8, const float *x_scale, const void *Wq, const float *w_scale,
                             int32_t wbits, const void *bias, clq_type bias_type, int32_t act, const void *gate,
                             clq_type gate_type, int64_t samples, const void *R, int64_t ldr, int64_t M, int64_t N,
                             int64_t K, clq_type type, void *Y, int64_t ldy, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CLQ_BLOCK_H */
