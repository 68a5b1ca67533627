/*
 * libsparq, microscaled formats -- the feed-forward block of a language model, trained and served, with 4-bit
 * floating point operands in its products and 8-bit activation checkpoints for its backward pass.
 *
 * A row of K values is cut into blocks of 32 along its length; a block shares one power of two, 2^s, stored as the
 * byte s + 127 (255: not a number).  With e = floor(log2(max |x| of the block)):
 *   4 bits  s = e - 2, a value is E2M1 (sign, 0 0.5 1 1.5 2 3 4 6) times 2^s: x / 2^s rounded to nearest, ties to
 *           the even code, at most 6;
 *   8 bits  s = e, a value is a signed integer / 64 times 2^s: 64 x / 2^s rounded to nearest, ties to even, clamped
 *           to [-127, 127].
 * s is clamped to [-127, 127]; a block of zeros has s = -127.  A block that holds a NaN or an infinity gets the scale
 * 255 and codes of zero: every value it stands for is NaN, and so is every result it enters.
 *
 * Storage: codes [rows][sparq_mx_code_bytes(K, bits)], two 4-bit codes a byte with the lower index in the low half;
 * scales [rows][sparq_mx_scale_bytes(K)].  Rows are whole units (128 values of codes, 512 of scales); what lies past K
 * is zero (scales: 0) and is written by the entry points that make them; readers rely on it.  Both buffers are
 * 16-byte aligned.
 *
 * Conventions are those of sparq.h: device pointers owned by the caller, a hipStream_t as void*, work only enqueued,
 * status codes, arguments checked on the host before anything is launched, nothing allocated and nothing kept between
 * calls.  Further:
 *   - x, y, dy and the like are row-major with a row stride ld* counted in elements (at least the row's length) and
 *     of one of the types below; any alignment of an element will do, 16-byte aligned rows are read faster.
 *   - Sums, statistics and everything between are fp32; a result is rounded once, to nearest even.
 *   - No result may overlap an input, the workspace or another result.
 *   - workspace: 256-byte aligned, at least the bytes its query names (NULL when that is 0), overwritten by the call;
 *     calls that share one must not overlap.
 *   - Results do not depend on timing: every sum is made in a fixed order.
 *   - K and N lie in [1, 2^28]; rows and M may be 0.  More rows than a call counts (2^31 / the row's units of 512; of
 *     the product's results 2^31 tiles, of weights' gradients 2^24, 64 x 64 or larger) return SPARQ_EUNSUPPORTED.
 *   - No rows: nothing is written, except gradients summed over the rows, which are zeros then.
 */
#ifndef SPARQ_MX_H
#define SPARQ_MX_H

#include "sparq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SPARQ_MX_F32 = 0, SPARQ_MX_F16 = 1, SPARQ_MX_BF16 = 2 } sparq_mx_type;
typedef enum { SPARQ_MX_SILU = 0, SPARQ_MX_GELU = 1 } sparq_mx_function;

/* Bytes of one row of codes (bits: 4 or 8) and of one row of scales; 0 for K < 1, K > 2^28 or another bits. */
size_t sparq_mx_code_bytes(int32_t K, int32_t bits);
size_t sparq_mx_scale_bytes(int32_t K);

/* Codes and scales of x [rows][K]: of the 4-bit form, of the 8-bit form, or of both from one pass over x (a layer's
 * input on its way into the product and into the backward pass).  Either pair of pointers may be NULL, not both. */
sparq_status sparq_mx_quantize(const void *x, int32_t type, int64_t ldx, int64_t rows, int32_t K,
                               void *codes4, void *scales4, void *codes8, void *scales8, void *stream);

/* y [rows][K] = the values that codes and scales stand for. */
sparq_status sparq_mx_dequantize(const void *codes, const void *scales, int32_t bits,
                                 void *y, int32_t type, int64_t ldy, int64_t rows, int32_t K, void *stream);

/* y[m][n] = sum_k A[m][k] W[n][k] + bias[n] over 4-bit A [M][K] and W [N][K] on the block-scaled matrix instruction.
 * bias: fp32 [N] or NULL.  K up to 2^23. */
size_t sparq_mx_gemm_workspace_bytes(int64_t M, int32_t N, int32_t K);
sparq_status sparq_mx_gemm(const void *a_codes, const void *a_scales, const void *w_codes, const void *w_scales,
                           const float *bias, void *y, int32_t type, int64_t ldy, int64_t M, int32_t N, int32_t K,
                           void *workspace, size_t workspace_bytes, void *stream);

/* The same with A = the 4-bit form of x [M][K], quantised on the way: a layer as it is served.  K up to 2^23. */
size_t sparq_mx_linear_workspace_bytes(int64_t M, int32_t N, int32_t K);
sparq_status sparq_mx_linear(const void *x, int32_t x_type, int64_t ldx, const void *w_codes, const void *w_scales,
                             const float *bias, void *y, int32_t y_type, int64_t ldy, int64_t M, int32_t N, int32_t K,
                             void *workspace, size_t workspace_bytes, void *stream);

/* Backward of the product, straight through the quantisers:
 *   dx[m][k] = sum_n dy[m][n] W[n][k]      over the 4-bit weights,
 *   dw[n][k] = sum_m dy[m][n] X[m][k]      over the 8-bit checkpoint X of the layer's input,
 *   db[n]    = sum_m dy[m][n]              (fp32; NULL: not wanted).
 * dy enters whole: bf16 as it is, fp16 and fp32 as the sum of two and three bf16 parts (of fp32, what lies below 2^-133
 * is left out). */
size_t sparq_mx_linear_dx_workspace_bytes(int64_t M, int32_t N, int32_t K);
sparq_status sparq_mx_linear_dx(const void *dy, int32_t dy_type, int64_t lddy, const void *w_codes, const void *w_scales,
                                void *dx, int32_t dx_type, int64_t lddx, int64_t M, int32_t N, int32_t K,
                                void *workspace, size_t workspace_bytes, void *stream);
size_t sparq_mx_linear_dw_workspace_bytes(int64_t M, int32_t N, int32_t K);
sparq_status sparq_mx_linear_dw(const void *dy, int32_t dy_type, int64_t lddy, const void *x_codes, const void *x_scales,
                                void *dw, int32_t dw_type, int64_t lddw, float *db, int64_t M, int32_t N, int32_t K,
                                void *workspace, size_t workspace_bytes, void *stream);

/* y = f(gate) * up over [rows][K], f(v) = v / (1 + exp(-v)) or v (1 + erf(v / sqrt 2)) / 2; up may be NULL (y = f(gate)).
 * Values of f below 2^-119 in magnitude may come as zero (fp32 does not hold what is between).
 * Where codes are given, the 8-bit checkpoints of gate and up are written as well (a pair of NULLs: not wanted). */
sparq_status sparq_mx_act(int32_t function, const void *gate, int64_t ldg, const void *up, int64_t ldu,
                          void *y, int64_t ldy, int32_t type, void *gate_codes, void *gate_scales,
                          void *up_codes, void *up_scales, int64_t rows, int32_t K, void *stream);

/* dgate = dy * up * f'(gate), dup = dy * f(gate), gate and up as their checkpoints stand for them.  Without up
 * (up_codes, up_scales and dup NULL): dgate = dy * f'(gate). */
sparq_status sparq_mx_act_grad(int32_t function, const void *dy, int64_t lddy, const void *gate_codes, const void *gate_scales,
                               const void *up_codes, const void *up_scales, void *dgate, int64_t lddg, void *dup, int64_t lddu,
                               int32_t type, int64_t rows, int32_t K, void *stream);

/* Layer norm over rows of K: y = (x - mean) rstd gamma + beta, rstd = 1 / sqrt(var + eps); gamma, beta fp32 [K], beta may
 * be NULL (none).  mean and rstd (fp32 [rows]) and the 8-bit checkpoint of x are what the backward pass needs; each pair
 * may be NULL. */
sparq_status sparq_mx_norm(const void *x, int64_t ldx, const float *gamma, const float *beta, float eps, void *y, int64_t ldy,
                           int32_t type, float *mean, float *rstd, void *codes, void *scales,
                           int64_t rows, int32_t K, void *stream);

/* With h = (X - mean) rstd over the checkpoint X and d = dy gamma:
 *   dx = rstd (d - avg(d) - h avg(d h)),   dgamma = sum over rows of dy h,   dbeta = sum over rows of dy
 * (averages over the row).  dgamma, dbeta: fp32 [K], either may be NULL. */
size_t sparq_mx_norm_grad_workspace_bytes(int64_t rows, int32_t K);
sparq_status sparq_mx_norm_grad(const void *dy, int64_t lddy, const void *codes, const void *scales,
                                const float *mean, const float *rstd, const float *gamma, void *dx, int64_t lddx, int32_t type,
                                float *dgamma, float *dbeta, int64_t rows, int32_t K,
                                void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPARQ_MX_H */
