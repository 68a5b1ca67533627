/*
 * libsparq, microscaled formats -- a feed-forward block with experts, and what a layer of any block does beside its
 * product: the router's choices sorted by expert, rows on their way to their experts and back, the experts' products with
 * bias, activation and residual, their gradients, and dropout.  Formats, storage and conventions are those of sparq_mx.h.
 *
 * A token t has `per` slots (up to 2^30), s = t per + j, each with the number of an expert, of a place and of a weight.  Sorted rows lie
 * expert after expert: expert e has the rows offsets[e] to offsets[e + 1] - 1.  Offsets, places and choices are int32 in
 * device memory and are never read by the host, so that a call can be captured into a graph and replayed on other choices.
 *   - offsets: [experts + 1], rising from 0 to at most the rows of the tensors they divide; what lies outside is cut off at
 *     these borders by the kernels.  Rows at offsets[experts] and behind belong to nobody: no call writes them and no result
 *     depends on what they hold, but they may be read, as may be rows that no slot has.
 *   - place: [tokens][per], a slot's sorted row; one outside of [0, rows) is a slot that was refused, which has no row.  No
 *     two slots may have the same row.
 */
#ifndef SPARQ_MX_EXPERTS_H
#define SPARQ_MX_EXPERTS_H

#include "sparq_mx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The most experts a call takes (more: SPARQ_EUNSUPPORTED). */
#define SPARQ_MX_EXPERTS_MOST 1024

/* Slots sorted by expert, slots of the same expert in their own order.  expert: [slots], a number outside of [0, experts) is
 * a slot refused.  offsets [experts + 1] and place [slots] (-1: refused) as above; order [slots] (NULL: not wanted): the slot
 * of each sorted row, -1 for the rows that nobody has.  slots up to 2^30; of none the offsets are zeros. */
size_t sparq_mx_sort_workspace_bytes(int64_t slots, int32_t experts);
sparq_status sparq_mx_sort(const int32_t *expert, int64_t slots, int32_t experts, int32_t *offsets, int32_t *place,
                           int32_t *order, void *workspace, size_t workspace_bytes, void *stream);

/* Row place[t][j] of the results = row t of x [tokens][K], for every slot that has one: as it is (y), as its 4-bit or its
 * 8-bit form, any of the three (NULL: not wanted; a pair for codes and scales).  rows: of the results; those that no slot has
 * stay as they are. */
sparq_status sparq_mx_gather(const void *x, int32_t type, int64_t ldx, int64_t tokens, int32_t K, const int32_t *place, int32_t per,
                             void *y, int64_t ldy, void *codes4, void *scales4, void *codes8, void *scales8, int64_t rows, void *stream);

/* y[t] = residual[t] + sum_j weights[t][j] x[place[t][j]] over the slots that have a row, added in the order of j, residual
 * last; weights: fp32 [tokens][per], NULL: ones (which is the gradient of sparq_mx_gather); residual [tokens][K], NULL: none.
 * x [rows][K], y and residual of one type. */
sparq_status sparq_mx_combine(const void *x, int64_t ldx, int64_t rows, const int32_t *place, const float *weights, int32_t per,
                              const void *residual, int64_t ldr, void *y, int64_t ldy, int32_t type, int64_t tokens, int32_t K,
                              void *stream);

/* Its gradient:  dx[place[t][j]] = weights[t][j] dy[t],   dweights[t][j] = sum_k dy[t][k] x[place[t][j]][k] (a slot without a
 * row: 0).  Either result may be NULL; x is read for dweights, weights for dx.  Rows of dx that no slot has stay as they are.
 * (The residual's gradient is dy.) */
sparq_status sparq_mx_combine_grad(const void *dy, int64_t lddy, const int32_t *place, const float *weights, int32_t per,
                                   void *dx, int64_t lddx, const void *x, int64_t ldx, int64_t rows, float *dweights,
                                   int32_t type, int64_t tokens, int32_t K, void *stream);

typedef enum { SPARQ_MX_NONE = -1 } sparq_mx_no_function;        /* beside sparq_mx_function */

/* y[m][n] = residual[m][n] + f(z[m][n]),   z[m][n] = sum_k A[m][k] W[e][n][k] + bias[e][n],   e the expert that has row m,
 * over 4-bit A [M][K] and W [experts][N][K].  offsets NULL: one expert (experts 1) has all rows, a layer as any.
 * function: SPARQ_MX_NONE, SPARQ_MX_SILU or SPARQ_MX_GELU; bias: fp32 [experts][N] or NULL; residual: [M][N] of y's type or
 * NULL.  Where kept_codes is given, z's 8-bit form [M][N] is written, from which sparq_mx_act_grad makes dz.  z stays in fp32
 * until all of this is done.  K up to 2^23, experts N up to 2^31 - 1, M below 2^31. */
size_t sparq_mx_experts_gemm_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts);
sparq_status sparq_mx_experts_gemm(const void *a_codes, const void *a_scales, const int32_t *offsets, int32_t experts,
                                   const void *w_codes, const void *w_scales, const float *bias, int32_t function,
                                   const void *residual, int64_t ldr, void *y, int32_t type, int64_t ldy, void *kept_codes,
                                   void *kept_scales, int64_t M, int32_t N, int32_t K, void *workspace, size_t workspace_bytes,
                                   void *stream);

/* The same with A = the 4-bit form of x [M][K], quantised on the way: as it is served. */
size_t sparq_mx_experts_linear_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts);
sparq_status sparq_mx_experts_linear(const void *x, int32_t x_type, int64_t ldx, const int32_t *offsets, int32_t experts,
                                     const void *w_codes, const void *w_scales, const float *bias, int32_t function,
                                     const void *residual, int64_t ldr, void *y, int32_t y_type, int64_t ldy, void *kept_codes,
                                     void *kept_scales, int64_t M, int32_t N, int32_t K, void *workspace, size_t workspace_bytes,
                                     void *stream);

/* Backward of the product, dy the gradient of z (without offsets: sparq_mx_linear_dx and sparq_mx_linear_dw):
 *   dx[m][k]    = sum_n dy[m][n] W[e][n][k],
 *   dw[e][n][k] = sum over expert e's rows m of dy[m][n] X[m][k]      (X: the rows' 8-bit form),
 *   db[e][n]    = sum over expert e's rows m of dy[m][n]              (fp32; NULL: not wanted).
 * An expert without rows gets zeros.  dx and dw: of dy's type or fp32; dw: rows lddw apart, expert after expert. */
size_t sparq_mx_experts_dx_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts);
sparq_status sparq_mx_experts_dx(const void *dy, int32_t dy_type, int64_t lddy, const int32_t *offsets, int32_t experts,
                                 const void *w_codes, const void *w_scales, void *dx, int32_t dx_type, int64_t lddx, int64_t M,
                                 int32_t N, int32_t K, void *workspace, size_t workspace_bytes, void *stream);
size_t sparq_mx_experts_dw_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts);
sparq_status sparq_mx_experts_dw(const void *dy, int32_t dy_type, int64_t lddy, const int32_t *offsets, int32_t experts,
                                 const void *x_codes, const void *x_scales, void *dw, int32_t dw_type, int64_t lddw, float *db,
                                 int64_t M, int32_t N, int32_t K, void *workspace, size_t workspace_bytes, void *stream);

/* y = residual + (kept ? x / (1 - q) : 0) over [rows][K], q = p rounded to a multiple of 2^-16, residual of x's type or NULL.
 * Element k of row r takes half k % 2 (the lower one first) of word k % 8 / 2 of the four words that Philox 4x32 with ten
 * rounds (Salmon, Moraes, Dror and Shaw, 2011) makes of the key seed and the counter (r ceil(K / 8) + k / 8, offset + *step), 64
 * bits each, and is kept where these 16 bits are at least 65536 q.  The backward pass is the same call on dy, without the residual:
 * no mask is stored.  step: a number in device memory or NULL for 0, for calls that are captured into a graph.  q = 1 leaves
 * the residual, or zeros. */
sparq_status sparq_mx_dropout(const void *x, int64_t ldx, double p, uint64_t seed, uint64_t offset, const uint64_t *step,
                              const void *residual, int64_t ldr, void *y, int64_t ldy, int32_t type, int64_t rows, int32_t K,
                              void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPARQ_MX_EXPERTS_H */
