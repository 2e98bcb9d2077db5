/*
 * clq_mx4.h -- C ABI of the microscaled 4-bit (MX4) operators of libclq.so and of
 * the expert layer built on them, for AMD Instinct MI355X (gfx950).
 *
 * MX4 keeps 4-bit floating-point codes (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives) with one power-of-two scale for every 32 consecutive values of a row:
 *
 *   e = max(floor(log2(max|x|)) - 2, -126),   code = rne(x / 2^e), at most 6,
 *
 * and the scale stored as the byte e + 127.  The quantizer rotates a row by the
 * block-Hadamard matrix first (block 32, 64 or 128; 0: no rotation), with an optional
 * gather vector, as clq_rotate_quant_act does; weights absorb the rotation and its
 * 1 / block.  A group whose rotated values hold an infinity or a NaN gets the scale byte
 * 255 and stands for NaN, so that every output it enters is a NaN.
 *
 * Conventions are those of clq.h: device pointers, caller-owned buffers, checks on the
 * host before anything is enqueued, no synchronisation, CLQ_ERR_* statuses.  Values
 * are fp16 or bf16 (clq_type), results fp32 too; sums are fp32.
 *   - Shapes: 1 <= M, N, T; 64 <= K <= 32768 with K % 64 == 0 and K % block == 0;
 *     1 <= experts <= 512; rows of a matrix (experts * padded rows) below 2^31;
 *     products of fewer than 2^24 tiles of 256 rows x 128 channels.  Row strides
 *     are in elements, at least the row length and multiples of 8 (logits: any).
 *   - Matrix and code pointers are 16-byte aligned, scales 16-byte aligned, bias 2-byte,
 *     int32 and float tables 4-byte aligned.
 *   - perm must be a permutation of 0..K-1 and activations and weights quantized with the
 *     same block and perm.  These are not checked (activations may also come gathered
 *     already, and are then quantized without perm).
 *   - An output must not overlap the matrices that the call reads (the Python binding
 *     refuses it).
 */
#ifndef CLQ_MX4_H
#define CLQ_MX4_H

#include "clq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CLQ_F16 = 0, CLQ_BF16 = 1, CLQ_F32 = 2 } clq_type;
typedef enum {
    CLQ_ACT_NONE = 0,
    CLQ_ACT_GELU = 1,    /* the tanh form: h / (1 + exp(-2 sqrt(2/pi) (h + 0.044715 h^3))) */
    CLQ_ACT_SWIGLU = 2   /* silu(g) * u, g and u the first and second half of the channels */
} clq_act;
typedef enum { CLQ_SOFTMAX = 0, CLQ_SIGMOID = 1 } clq_score;

/* ---- MX4 matrices --------------------------------------------------------------- */

/* Bytes of the codes and of the scales of `rows` rows of K values, in opaque layouts
 * (weights = 1: of a weight matrix, rows padded to a multiple of 64; 0: of activations,
 * padded to 32).  0 if the shape is out of range.  An expert layer's weights are that
 * many bytes for each expert, one after the other. */
size_t clq_mx4_code_bytes(int64_t rows, int64_t K, int32_t weights);
size_t clq_mx4_scale_bytes(int64_t rows, int64_t K, int32_t weights);

/* Rotates and quantizes activations.
 *   X       fp16 or bf16 [M][K], row stride ldx.
 *   perm    int32 [K] gather vector, or NULL.
 *   codes, scales   out, clq_mx4_code_bytes / _scale_bytes (M, K, 0) bytes; padding rows
 *           are zeros.
 * x~ = FWHT_block(gather(x, perm)) in fp32, stage order h = 1, 2, ..., block / 2. */
clq_status clq_mx4_quantize(const void *X, clq_type type, int64_t ldx, const int32_t *perm, int64_t M, int64_t K,
                            int32_t block, void *codes, void *scales, hipStream_t stream);

/* Rotates and quantizes weights: W fp16 or bf16 [experts][N][K], contiguous.  The
 * quantized values are those of FWHT_block(gather(w, perm)) / block.
 *   gated   1: the first N / 2 rows are gates, the others their partners (N % 64 == 0);
 *           their output channels are interleaved for CLQ_ACT_SWIGLU.
 *   codes, scales   out, experts times the bytes of one N x K weight matrix. */
clq_status clq_mx4_quantize_weights(const void *W, clq_type type, const int32_t *perm, int64_t experts, int64_t N,
                                    int64_t K, int32_t block, int32_t gated, void *codes, void *scales,
                                    hipStream_t stream);

/* Lays out weights that are MX4 already: row-major codes uint8 [experts][N][K/2] (byte j
 * holds codes 2j, low half, and 2j + 1) and scale bytes uint8 [experts][N][K/32]. */
clq_status clq_mx4_pack_weights(const void *row_codes, const void *row_scales, int64_t experts, int64_t N, int64_t K,
                                int32_t gated, void *codes, void *scales, hipStream_t stream);

/* The values that codes and scales stand for: out [matrices][rows][K] of `type` (fp16 rounds
 * and overflows to infinity; bf16 and fp32 are exact), row stride ldo; weights, gated: how
 * the matrix was quantized (activations: 0, 0, one matrix). */
clq_status clq_mx4_dequantize(const void *codes, const void *scales, int32_t weights, int32_t gated, int64_t matrices,
                              int64_t rows, int64_t K, clq_type type, void *out, int64_t ldo, hipStream_t stream);

/* Y = X . W^T + bias, summed in fp32 and rounded once to `type` (fp16, bf16, or fp32: not rounded).
 *   bias    fp16 or bf16 [N] (bias_type), or NULL.
 *   Y       out, [M][N], row stride ldy. */
clq_status clq_mx4_linear(const void *Xq, const void *Xs, const void *Wq, const void *Ws, const void *bias,
                          clq_type bias_type, int64_t M, int64_t N, int64_t K, clq_type type, void *Y, int64_t ldy,
                          hipStream_t stream);

/* The same with the result activated, rotated and quantized again, as the next product's
 * input: act(X . W^T + bias) in fp32, then as clq_mx4_quantize with `block`, without a rounding
 * in between.  N % 64 == 0; CLQ_ACT_SWIGLU takes gated weights with N % 128 == 0, writes N / 2
 * columns and takes block 0, 32 or 64.
 *   codes, scales   out, clq_mx4_code_bytes / _scale_bytes (M, columns, 0) bytes. */
clq_status clq_mx4_linear_mx4(const void *Xq, const void *Xs, const void *Wq, const void *Ws, const void *bias,
                              clq_type bias_type, int64_t M, int64_t N, int64_t K, clq_act act, int32_t block,
                              void *codes, void *scales, hipStream_t stream);

/* ---- expert layer ---------------------------------------------------------------- */

/* Routes tokens to experts.
 *   logits  [T][experts] of `type` (fp32 too), row stride ld.
 *   top_k   1 .. 32 experts for a token.
 *   score   softmax or sigmoid of the logits, in fp32.
 *   bias    fp32 [experts] added to the scores for the ranking alone, or NULL.
 *   groups  1 .. 64, dividing experts: a group counts the sum of its two best ranks, and
 *           only the experts of the top_groups best groups can be chosen (top_k of them at
 *           least).  1: no groups.
 *   renormalize   1: a token's weights are divided by their sum (weights that sum to 0 stay 0).
 *   scale   factor of the weights.
 *   ids     out, int32 [T][top_k], best first, ties to the lower index.  Experts rank by score
 *           + bias, or by the logits themselves without a bias and groups.
 *   weights out, fp32 [T][top_k].
 * A token whose logits are all -infinity gets the experts 0 .. top_k - 1 under softmax, with
 * weights 0; one with a NaN among its logits gets NaN weights and valid experts. */
clq_status clq_expert_route(const void *logits, clq_type type, int64_t ld, int64_t T, int64_t experts, int32_t top_k,
                            clq_score score, const float *bias, int32_t groups, int32_t top_groups,
                            int32_t renormalize, float scale, int32_t *ids, float *weights, hipStream_t stream);

/* Rows that a plan of T x top_k assignments to `experts` experts can need (0 if out of range):
 * every expert's rows start on a multiple of 32. */
int64_t clq_expert_plan_rows(int64_t T, int64_t top_k, int64_t experts);
/* int32 entries of a plan's tables, and bytes of the workspace it is made in (0: none). */
int64_t clq_expert_plan_ints(int64_t experts);
size_t clq_expert_plan_workspace_bytes(int64_t T, int64_t top_k, int64_t experts);

/* Sorts assignments by expert, stable in the order of tokens and slots.
 *   ids     int32 [T][top_k]; entries outside 0 .. experts - 1 belong to no expert here (a
 *           dropped token, another process's expert) and get no row.
 *   tables  out, int32 [clq_expert_plan_ints]: rows of each expert, then opaque.
 *   rows    out, int32 [T][top_k]: the row of each assignment, -1 for none.  Expert e's rows
 *           start at 32 * sum over e' < e of ceil(rows of e' / 32).
 *   source  out, int32 [clq_expert_plan_rows]: the token of each row in use, -1 on padding.
 *   workspace   clq_expert_plan_workspace_bytes, no initial contents needed; NULL if that is 0. */
clq_status clq_expert_plan(const int32_t *ids, int64_t T, int64_t top_k, int64_t experts, int32_t *tables,
                           int32_t *rows, int32_t *source, void *workspace, size_t workspace_bytes,
                           hipStream_t stream);

/* clq_mx4_quantize of tokens into a plan's rows: row r is token source[r].
 *   codes, scales   out, of clq_expert_plan_rows rows; rows past the plan's last are not
 *                   written. */
clq_status clq_mx4_dispatch(const void *X, clq_type type, int64_t ldx, const int32_t *perm, int64_t T, int64_t top_k,
                            int64_t experts, int64_t K, int32_t block, const int32_t *tables, const int32_t *source,
                            void *codes, void *scales, hipStream_t stream);

/* clq_mx4_linear and clq_mx4_linear_mx4 with each row multiplied by its expert's weights:
 * Wq, Ws of `experts` matrices, bias [experts][N], rows and tables of a plan of T x top_k
 * assignments.  Rows past the plan's last are not written; padding rows hold the result for an
 * input of zeros. */
clq_status clq_mx4_experts(const void *Xq, const void *Xs, const int32_t *tables, int64_t T, int64_t top_k,
                           int64_t experts, const void *Wq, const void *Ws, const void *bias, clq_type bias_type,
                           int64_t N, int64_t K, clq_type type, void *Y, int64_t ldy, hipStream_t stream);
clq_status clq_mx4_experts_mx4(const void *Xq, const void *Xs, const int32_t *tables, int64_t T, int64_t top_k,
                               int64_t experts, const void *Wq, const void *Ws, const void *bias, clq_type bias_type,
                               int64_t N, int64_t K, clq_act act, int32_t block, void *codes, void *scales,
                               hipStream_t stream);

/* out[t] = sum over j of weights[t][j] * Y[rows[t][j]], in the order of the slots, in fp32,
 * rounded once; rows of -1 add nothing.  Y [plan rows][N] of `type`, out [T][N] of `out_type`,
 * row strides ldy and ldo. */
clq_status clq_expert_combine(const void *Y, clq_type type, int64_t ldy, const int32_t *rows, const float *weights,
                              int64_t T, int64_t top_k, int64_t experts, int64_t N, void *out, clq_type out_type,
                              int64_t ldo, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* CLQ_MX4_H */
