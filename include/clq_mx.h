/*
 * clq_mx.h - microscaled 4-bit floating point in libclq: quantization, the
 * product, routing to experts and the experts' products, for one GB300
 * (sm_103a).
 *
 * The INT4 path of clq.h runs on 8-bit tensor-core operands, because sm_103a
 * has no integer tcgen05 MMA.  E2M1 codes with a scale for each block of a
 * row are what its tensor cores multiply natively, at twice that rate, and the
 * block scales follow outliers that a scale per token cannot; the swap and
 * the block Hadamard rotation of clq.h go in front of them as before.
 *
 * Conventions are clq.h's (status codes, device pointers owned by the caller,
 * no allocation, no synchronization, asynchronous on `stream`, arguments
 * checked on the host before anything is launched, device-side faults in the
 * status word of clq_get_device_status, the rule on `perm` excepted: these
 * calls read it only after the work enqueued before them).
 *
 * CODES.  E2M1: sign bit 3; 0, 1, .., 7 of the other bits are 0, 0.5, 1, 1.5,
 * 2, 3, 4, 6.  A row of K codes is K / 2 bytes, code 2j in the low nibble of
 * byte j; rows are contiguous.  K % 32 == 0, 32 <= K <= 16384; fewer than 2^30
 * rows.
 * SCALES.  One byte a block of `block` codes of a row:
 *   CLQ_MX_BLOCK32  blocks of 32, E8M0 bytes: 2^(byte - 127), 0xFF is NaN;
 *   CLQ_MX_BLOCK16  blocks of 16, E4M3 bytes (not negative), and an fp32
 *                   scale for each row besides.
 * They lie as the tensor cores take them: the scale of row 128 i + 32 j + r
 * (j < 4, r < 32), block 4 c + q (q < 4) is byte
 * (i C + c) 512 + 16 r + 4 j + q, C = ceil(K / block / 4); clq_mx_scale_bytes
 * gives the array's size.  Bytes of rows past the last are never used; those
 * of blocks past the last (block 4 c + q >= K / block) are 0.
 * VALUES.  code * scale (* row scale).
 * QUANTIZATION of a row v of fp32 values, amax over absolute values:
 *   BLOCK32  scale = 2^e, e = ceil(log2(amax_block / 6)) (at least -127, so
 *            nothing saturates), code = rn(v * 2^-e); a block with an infinity
 *            or a NaN has scale NaN (and codes 0).
 *   BLOCK16  s_row = max(amax_row * r, 2^-100), r = 1 / 2688 in fp32 (2688 = 6 *
 *            448, the largest code times the largest scale), scale =
 *            e4m3_rn(amax_block / (6 s_row)), code = rn(v * (1 / (scale s_row))), 0 where scale
 *            is 0; a row with an infinity or a NaN has s_row NaN (codes and
 *            scales 0).
 *   rn rounds to the nearest E2M1 value, ties to the even code, |.| > 6 to 6.
 * Every step, the swap and the rotation among them, is one IEEE fp32 operation in the
 * order written, but for an activation (see clq_mx_act); a value that is exactly 0 has
 * code 0 (not 8, its negative).
 * VERSION.  clq_version counts the functions of clq.h alone; a library has those of this
 * header if it has clq_mx_scale_bytes.
 */
#ifndef CLQ_MX_H
#define CLQ_MX_H

#include "clq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t clq_mx_format;
#define CLQ_MX_BLOCK32 0
#define CLQ_MX_BLOCK16 1

#define CLQ_F32 2 /* logits of clq_mx_route only */

/* What is applied to a row before the swap and the rotation, in fp32: for every finite 16-bit
 * input within 2^-21 |x| of the exact value (SWIGLU: 2^-21 |g u|, where that is a finite fp32
 * number), wherever an activation is taken, so that a code may differ from the exact one's where
 * a value lies that close to the middle of two, and so may the scale of a block (or a row). */
typedef int32_t clq_mx_act;
#define CLQ_MX_ACT_NONE 0
#define CLQ_MX_ACT_GELU 1   /* 0.5 x (1 + erf(x / sqrt 2))                     */
#define CLQ_MX_ACT_SWIGLU 2 /* g / (1 + exp(-g)) u; the row holds 2K values,   */
                            /* 8 of g, 8 of u, 8 of g, ..                      */

/* Bytes of the scale array of `rows` x K codes (0 for bad arguments). */
size_t clq_mx_scale_bytes(int32_t rows, int32_t K, clq_mx_format fmt);

/*
 * Rows -> codes and scales.  X: device [M][ldx] of `dtype` (fp16 / bf16), K
 * values a row (2K for SWIGLU).  perm: device int32 [K] or NULL (no swap); b: order
 * of the block Hadamard rotation, a power of two <= 256 with K % b == 0; 1: none.
 * The rotation is unnormalized, as in clq.h, its stages in ascending order.  codes:
 * device [rows][K / 2]; scales: device, clq_mx_scale_bytes; row_scale: device
 * fp32 [rows], BLOCK16 only (NULL else).  out_rows NULL: rows = M and row i is
 * written to row i.  Else: device int32 [M][k], row i goes to the k rows
 * out_rows[i][..] (negative: nowhere) of `rows` rows; an index >= rows is not
 * written and reported as CLQ_ERR_DEVICE_INDEX, as is one of perm outside [0, K).
 * X, codes and scales 16-byte aligned, ldx % 8 == 0.
 */
clq_status clq_mx_quantize(const void* X, clq_dtype dtype, int32_t M, int32_t K, int32_t ldx,
                           const int32_t* perm, int32_t b, clq_mx_act act, clq_mx_format fmt,
                           uint8_t* codes, uint8_t* scales, float* row_scale,
                           const int32_t* out_rows, int32_t k, int32_t rows, void* stream);

/* Codes and scales -> their values, rounded to `dtype`: out device [M][K]. */
clq_status clq_mx_dequantize(const uint8_t* codes, const uint8_t* scales, const float* row_scale,
                             int32_t M, int32_t K, clq_mx_format fmt, clq_dtype dtype, void* out,
                             void* stream);

/*
 * Y[i][n] = out_dtype(sum_k x[i][k] w[n][k] / b + bias[n]), x and w the values of
 * two code arrays of one format, accumulated in fp32 (products of codes and scales
 * are exact; BLOCK16's row scales and 1 / b are multiplied with one another first, in
 * fp32, and the sum with that).  Xq / Xs / s_x: codes, scales and (BLOCK16) row scales of M rows; Wq /
 * Ws / s_w: of N; bias: device [N] of `dtype` or NULL; Y: device [M][N], 16-byte
 * aligned.  Codes and scales 16-byte, row scales 4-byte aligned.
 */
clq_status clq_mx_linear(const uint8_t* Xq, const uint8_t* Xs, const float* s_x,
                         const uint8_t* Wq, const uint8_t* Ws, const float* s_w, const void* bias,
                         int32_t M, int32_t N, int32_t K, int32_t b, clq_mx_format fmt,
                         clq_dtype dtype, void* Y, void* stream);

/*
 * Routing of T tokens to k of E experts.  logits: device [T][ld] of `dtype` (fp16,
 * bf16 or CLQ_F32), 1 <= E <= 512, 1 <= k <= min(E, 32).  All in fp32:
 *   scoring 0: p = softmax(logits); 1: p = 1 / (1 + exp(-logit));
 *   c = p + balance (device fp32 [E] or NULL);
 *   groups > 1 (E % groups == 0): of the groups of E / groups neighbours the
 *   top_groups with the largest sum of their group_top (1 or 2) largest c stay, ties to
 *   the lowest; a masked expert's c counts as -infinity there, so that a group with one
 *   among its group_top largest comes last;
 *   the k largest c, ties to the lowest index; weight = p, divided by the sum of the
 *   k if `renormalize`, times `scale`.
 * The softmax sums by halves (element i + element i + n / 2, n the power of two >= E,
 * missing ones 0, and so on), so its scores have one value.  A logit of
 * -infinity or NaN masks its expert, as does a c of those; an infinity counts as the
 * largest finite value.  Places for which no expert is left hold expert -1 with weight 0.
 * experts: device int32 [T][k]; weights: device fp32 [T][k].
 */
clq_status clq_mx_route(const void* logits, int32_t dtype, int32_t T, int32_t E, int32_t ld,
                        const float* balance, int32_t k, int32_t scoring, int32_t groups,
                        int32_t top_groups, int32_t group_top, int32_t renormalize, float scale,
                        int32_t* experts, float* weights, void* stream);

/*
 * Where the rows of a routing go: each expert's rows, in token order, start at a
 * multiple of 128, so that its scales are whole blocks.  clq_mx_plan_rows: how many
 * rows that takes at most (0 for bad arguments).  clq_mx_plan writes, into `plan`
 * (device, 16-byte aligned, clq_mx_plan_bytes bytes), what the grouped product
 * needs, and the row of each place into out_rows (device int32 [T][k], -1 where
 * experts holds no expert in [0, E)).  A token names an expert once.
 */
int32_t clq_mx_plan_rows(int32_t T, int32_t k, int32_t E);
size_t clq_mx_plan_bytes(int32_t T, int32_t k, int32_t E);
clq_status clq_mx_plan(const int32_t* experts, int32_t T, int32_t k, int32_t E, int32_t* out_rows,
                       void* plan, size_t plan_bytes, void* stream);

/*
 * The experts' products: row i of expert e (clq_mx_plan's rows) is multiplied with
 * W[e].  Xq / Xs / s_x: clq_mx_plan_rows rows; Wq: [E][N][K / 2], Ws: E arrays of
 * clq_mx_scale_bytes(N, K), s_w: [E][N]; bias: [E][N] or NULL; Y: device
 * [plan rows][N]; rows that no token has are left undefined.  Otherwise as clq_mx_linear.
 */
clq_status clq_mx_grouped_linear(const uint8_t* Xq, const uint8_t* Xs, const float* s_x,
                                 const void* plan, const uint8_t* Wq, const uint8_t* Ws,
                                 const float* s_w, const void* bias, int32_t T, int32_t k,
                                 int32_t E, int32_t N, int32_t K, int32_t b, clq_mx_format fmt,
                                 clq_dtype dtype, void* Y, void* stream);

/*
 * The same product in blocks of 32, with its output as the next product's operand: h =
 * out_dtype(x w^T / b + bias) as clq_mx_grouped_linear would store it, then act(h), quantized
 * as by clq_mx_quantize_rows, into Yq / Ys: codes and scales of clq_mx_plan_rows rows of N
 * codes (N / 2 for SWIGLU), N % 32 == 0 (64 for SWIGLU), at most 16384 codes.
 */
clq_status clq_mx_grouped_linear_act(const uint8_t* Xq, const uint8_t* Xs, const void* plan,
                                     const uint8_t* Wq, const uint8_t* Ws, const void* bias,
                                     int32_t T, int32_t k, int32_t E, int32_t N, int32_t K,
                                     int32_t b, clq_dtype dtype, clq_mx_act act, uint8_t* Yq,
                                     uint8_t* Ys, void* stream);

/*
 * The rows of a plan, act(X) without swap or rotation -> codes and scales: what
 * clq_mx_quantize makes of the rows that tokens have, the others undefined.  X: device
 * [clq_mx_plan_rows][ldx].
 */
clq_status clq_mx_quantize_rows(const void* X, clq_dtype dtype, const void* plan, int32_t T,
                                int32_t k, int32_t E, int32_t K, int32_t ldx, clq_mx_act act,
                                clq_mx_format fmt, uint8_t* codes, uint8_t* scales,
                                float* row_scale, void* stream);

/*
 * out[t] = sum_j weights[t][j] Y[rows[t][j]] over the places with rows >= 0, in
 * the order of j, in fp32.  Y: device [R][D] of `dtype`, D % 8 == 0, D <= 2^24; out:
 * [T][D]; T and k below 2^30.
 */
clq_status clq_mx_combine(const void* Y, clq_dtype dtype, const int32_t* rows,
                          const float* weights, int32_t T, int32_t k, int32_t D, int32_t R,
                          void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CLQ_MX_H */
