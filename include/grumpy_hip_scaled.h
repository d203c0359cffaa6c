/*
 * grumpy_hip_scaled.h -- root-mean-square norms, 8-bit tensors with scales, and their products beside the lazy arrays of grumpy_hip.h.
 *
 * What stands between the residual stream of a network and its matrix products: the norm with the residual's addition, which can write
 * its result in 8 bits as the next product takes it, the norm's gradient, 8-bit forms of weights and gradients, and the product of
 * two 8-bit tensors.
 *
 * Conventions, beyond those of grumpy_hip.h
 *   - Like gr_assign, the calls launch at once: operands that are still unevaluated are evaluated first, results are WRITTEN into
 *     the arrays given for them, which must be materialised arrays or slice / transpose views of some; recorded but unevaluated arrays
 *     that read that storage are evaluated first.  Everything runs asynchronously on the context's stream.
 *   - GR_E4M3 arrays hold 8-bit floating-point values (4 bits of exponent, 3 of fraction, largest 448, no infinities).  Like bf16 ones they
 *     are leaves and views of leaves; no call but these computes with them (GR_ERR_DTYPE).
 *   - Scales (f32, any strides) belong to 128 neighbours along the last axis, the last ones of a row perhaps to fewer: of one row ("rows",
 *     shape (.., ceil(K / 128))), or of 128 rows together ("blocks", shape (ceil(M / 128), ceil(K / 128))).  A value stands for
 *     itself times its scale.  The scale is max|x| / 448, or 2^-126 where that is smaller; values are divided by it in f32 (right to a last place) and rounded to the
 *     nearest e4m3, ties to even.  Where one of the values of a scale is infinite or NaN, the scale and all its values are NaN.
 *   - The values of a row (the last axis) of every tensor are neighbours, or GR_ERR_UNSUPPORTED; rows may lie anywhere.  The elements of a result do
 *     not overlap (GR_ERR_UNSUPPORTED), nor do two results or a result and an operand (GR_ERR_ALIAS), except where a call says so.
 *   - A call that answers GR_ERR_HIP may have been launched: what its results hold is not known, and over operands it is not to be made again.
 *   - Temporary memory and captured graphs: as in grumpy_hip_attention.h, with whose calls these share it.
 *   - Results do not depend on timing: every sum is taken in an order fixed by the shapes.
 */
#ifndef GRUMPY_HIP_SCALED_H
#define GRUMPY_HIP_SCALED_H

#include "grumpy_hip.h"

#ifdef __cplusplus
extern "C" {
#endif

/* total = x + residual, rounded to its type (residual = 0: total is x, and no result; total = 0: not wanted);
 * r = 1 / sqrt(mean(total^2) + eps) over the last axis;  out = total r (offset + weight).
 * x, residual, total: f32 or bf16, one type, 1 to 4 axes, up to 32768 values in a row.  out: of that type, or GR_E4M3 with `scales` of rows.
 * weight: f32 or x's type, (D); 0 = a factor of 1 (offset must be 0).  eps: 1e-12 .. 1.  Squares are summed in f32: a row whose sum passes its range (values of 10^18 and more) has out 0, and a
 * gradient that may be NaN.
 * total and out may each be x or residual themselves (the same view). */
gr_status gr_rms_norm(gr_ctx* ctx, gr_array x, gr_array residual, gr_array weight, double eps, double offset, gr_array total, gr_array out, gr_array scales);

/* The gradients for the gradient `dout` of gr_rms_norm's out (before it was rounded to 8 bits, if it was), from total (x where there was no residual):
 * dx = r dout (offset + weight) - total r^3 mean(total dout (offset + weight)) + dtotal,  dweight = sum over all rows of dout total r.
 * dx is the gradient of x and of residual alike.  dtotal: the gradient that reaches total by other ways; 0 = none.  dweight: f32 (D); 0 = not wanted.
 * dx may be dout, total or dtotal itself (the same view). */
gr_status gr_rms_norm_grad(gr_ctx* ctx, gr_array dout, gr_array total, gr_array weight, gr_array dtotal, double eps, double offset, gr_array dx, gr_array dweight);

/* x (M, K), f32 or bf16, in 8 bits: out (M, K) and scales of rows, or of blocks (blocks = 1).  transposed = 1: the same of the transposed
 * tensor, out (K, M), whose rows are x's columns. */
gr_status gr_quantize(gr_ctx* ctx, gr_array x, int blocks, int transposed, gr_array out, gr_array scales);

/* out[m][n] = sum over k of the values that a[m][k] and b[n][k] stand for.  a (M, K), scales of rows; b (N, K), scales of blocks or of rows (told
 * by their shape); out (M, N), f32 or bf16.  With an f32 out the sum of each 128 products is f32; with a bf16 out it comes from the 8-bit matrix cores, which drop what lies
 * below 2^-13 of the largest of eight neighbouring products (1.5e-5 of a sum of normal numbers, a hundredth of the result's rounding).  Its product with the two scales' product
 * and the sum of those are f32: two scales whose product f32 does not hold give infinities or NaN (above 3.4e38), or lose places (below 1.2e-38). */
gr_status gr_dot_scaled(gr_ctx* ctx, gr_array a, gr_array a_scales, gr_array b, gr_array b_scales, gr_array out);

#ifdef __cplusplus
}
#endif
#endif /* GRUMPY_HIP_SCALED_H */
