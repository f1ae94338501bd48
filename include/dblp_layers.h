/*
 * dblp_layers -- the matrix products of a worker's layers on one AMD MI355X (gfx950), their gradients, and
 * the update that is made of a matrix' mean gradient: what lies between the two ends of a step in
 * dblp_worker.h, and what follows dblp_finalize.
 *
 *   dblp_linear              x W^T with bias, activation and residual in the product's own pass
 *   dblp_linear_grad_input   dy W, gated by an earlier activation's slope, onto the sum the caller holds
 *   dblp_linear_grad_weight  dy^T x and the bias' gradient, in fp32, what a packet carries
 *   dblp_activation_grad     the slope of an activation times a gradient
 *   dblp_orthogonalize       the nearly orthogonal matrix with a gradient's singular directions, onto the weights
 *
 * Conventions are those of dblp_worker.h: DBLP_OK or a negative DBLP_E*, dblp_worker_error() for the text, arguments
 * checked on the host before the device is touched, everything enqueued on `stream` of `device`, nothing allocated, nothing
 * waited for, calls that can be recorded into a HIP graph, types DBLP_F32, DBLP_BF16 and DBLP_F16, pointers aligned to one
 * element, row strides in ELEMENTS, an input's rows may overlap, an output overlaps no other argument except where "in
 * place" says so.  Every result is a function of the arguments alone: no floating-point atomics, sums cut by sizes, types, strides and the alignment of addresses.  Where a value
 * is not finite, or a float lies below 2^-110, other results of a large product of floats (those of its tile, at most 128 x 128) may differ in their last bits from what they are without it.
 * Rows whose address and stride are multiples of 16 bytes are fastest.
 *
 * Products are summed in fp32 (of 16-bit values each product is exact, of fp32 values it is within 2^-23 of itself), everything behind them is computed in fp32, and a result
 * is rounded once, to nearest even, when it is stored.  NaN and infinities go through the formulas.
 * Limits: tokens, columns and rows below 2^31, those of dblp_orthogonalize below 2^24.  Zero tokens, columns or rows are allowed: a sum of nothing is zero.
 * A workspace is DEVICE memory of the size that dblp_*_workspace gives, 256-byte aligned, of any contents; it is free
 * again when the stream has passed the call.  One of a larger call (more of any size) is large enough for a smaller one.
 */
#ifndef DBLP_LAYERS_H
#define DBLP_LAYERS_H

#include <stdint.h>

#include "dblp_worker.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations and their slopes.
 *   NONE       z                                                             1
 *   RELU       max(z, 0)                                                     1 where z > 0, else 0 (a gradient is taken or is +0)
 *   GELU       z Phi(z), Phi(z) = (1 + erf(z / sqrt 2)) / 2                  Phi(z) + z exp(-z z / 2) / sqrt(2 pi)
 *   GELU_TANH  z p, p = (1 + tanh u) / 2, u = sqrt(2 / pi) (z + 0.044715 z^3)  p + 2 z p (1 - p) sqrt(2 / pi) (1 + 0.134145 z z)
 *   SILU       z p, p = 1 / (1 + exp(-z))                                    p (1 + z (1 - p)) */
#define DBLP_ACT_NONE 0
#define DBLP_ACT_RELU 1
#define DBLP_ACT_GELU 2
#define DBLP_ACT_GELU_TANH 3
#define DBLP_ACT_SILU 4

/* z[t][o] = sum_i x[t][i] w[o][i] + bias[o],  y = act(z) + residual.  x is n_tokens x in, w out x in, both of `type`; y, z
 * and the residual are n_tokens x out, of out_type: `type` or DBLP_F32.  d_bias (of bias_type), d_residual may be NULL.  d_z:
 * z as well, rounded, for the way back; NULL: not kept.  In place: y may be the residual, with the same stride. */
int dblp_linear(int device, void* stream, uint64_t n_tokens, uint32_t in, uint32_t out, const void* d_x, uint64_t x_stride,
                const void* d_w, uint64_t w_stride, int type, const void* d_bias, int bias_type, int activation,
                const void* d_residual, uint64_t residual_stride, void* d_y, uint64_t y_stride, void* d_z, uint64_t z_stride,
                int out_type, void* d_workspace, uint64_t workspace_bytes);

/* dx[t][i] = (sum_o dy[t][o] w[o][i]) act'(z[t][i]) + base[t][i].  z is that of the layer whose result x was: dx is then that
 * layer's dy.  d_z NULL: no factor (then the activation must be NONE); d_base NULL: no term.  dy and w of `type`, z, base
 * and dx of out_type (`type` or DBLP_F32).  In place: dx may be z or the base, with the same stride. */
int dblp_linear_grad_input(int device, void* stream, uint64_t n_tokens, uint32_t in, uint32_t out, const void* d_dy,
                           uint64_t dy_stride, const void* d_w, uint64_t w_stride, int type, const void* d_z, uint64_t z_stride,
                           int activation, const void* d_base, uint64_t base_stride, void* d_dx, uint64_t dx_stride, int out_type,
                           void* d_workspace, uint64_t workspace_bytes);

/* dw[o][i] = base[o][i] + sum_t dy[t][o] x[t][i] and dbias[o] = bias_base[o] + sum_t dy[t][o], in fp32.  d_base, d_bias_base
 * NULL: zeros.  d_dbias NULL: no bias (then d_bias_base must be NULL).  In place: dw may be the base, with the same stride, and
 * dbias its base (a tied table's other gradient, or an earlier micro-batch). */
int dblp_linear_grad_weight(int device, void* stream, uint64_t n_tokens, uint32_t in, uint32_t out, const void* d_dy,
                            uint64_t dy_stride, const void* d_x, uint64_t x_stride, int type, const float* d_base,
                            uint64_t base_stride, float* d_dw, uint64_t dw_stride, const float* d_bias_base, float* d_dbias,
                            void* d_workspace, uint64_t workspace_bytes);
/* Bytes of the workspace of these three; 0 if an argument is out of range.  Up to 1 GB of it is for operands of 16-bit values whose rows do not begin
 * at multiples of four bytes, which are laid out anew there. */
uint64_t dblp_linear_workspace(uint64_t n_tokens, uint32_t in, uint32_t out);

/* dz = dy act'(z), for a layer whose activation is not followed by a product; dy, z and dz of one type.  In place: dz may
 * be dy or z, with the same stride. */
int dblp_activation_grad(int device, void* stream, uint64_t rows, uint32_t cols, const void* d_dy, uint64_t dy_stride,
                         const void* d_z, uint64_t z_stride, int activation, void* d_dz, uint64_t dz_stride, int type);

/* For each of `count` matrices G of rows x cols, `step` ELEMENTS apart: X = G / |G| (|G| the root of the sum of squares; a zero
 * matrix stays zero, one with a value that is not finite becomes NaN throughout), then `steps` times
 *   A = X X^T (X^T X where rows > cols),   X <- a X + (b A + c A A) X (from the right)
 * with a, b, c = h_coefficients[3 k ...] in step k (NULL: 3.4445, -4.7750, 2.0315 in each, which take singular values of 0.01 and
 * above to 0.7 to 1.2 in five steps), and out = base_scale base + scale X (d_base NULL: scale X).  The orthogonalised update
 * of the Muon optimiser is this call on a momentum of gradients, with the weights as base and out.  G is of g_type, base and out of out_type.
 * X, A and a + b A + c A A are held with 22 significant bits, or to 2^-50 of the largest value that they can have, and multiplied so.  Refused are
 * steps above 16 and coefficients under which a singular value could pass 32.  In place: out may be the base or G, with the same stride and step; out's matrices do not overlap. */
int dblp_orthogonalize(int device, void* stream, uint64_t count, uint32_t rows, uint32_t cols, const void* d_g, uint64_t g_stride,
                       uint64_t g_step, int g_type, const double* h_coefficients, uint32_t steps, float scale, const void* d_base,
                       uint64_t base_stride, uint64_t base_step, float base_scale, void* d_out, uint64_t out_stride,
                       uint64_t out_step, int out_type, void* d_workspace, uint64_t workspace_bytes);
/* Bytes of its workspace; 0 if an argument is out of range. */
uint64_t dblp_orthogonalize_workspace(uint64_t count, uint32_t rows, uint32_t cols);

#ifdef __cplusplus
}
#endif
#endif /* DBLP_LAYERS_H */
