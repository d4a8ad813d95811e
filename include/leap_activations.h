/*
 * leap_activations.h - C ABI of the operators for networks trained through the projector, with activations held in 8 bits.
 *
 * "PyTorch Interfaces and CT Parameters" puts the projector into a network's training loop.  What such training runs out of
 * is memory: every unrolled iteration keeps volume-sized activations for its backward pass.  These operators keep them in
 * 8 bits and work on them there: packing, a root-mean-square norm with the residual's addition whose output is packed,
 * products of packed rows with a weight (plain, and gated with a packed output), and the gradients of all of them.
 *
 * Packed in 8 bits: an array [rows][cols] is held as codes, one byte per value, and scales, one byte per group of 32
 * consecutive values of a row (the last group of a row may be shorter; its scale byte is there all the same), both without
 * gaps: codes[rows][cols], scales[rows][ceil(cols / 32)].  With amax the largest magnitude of a group's finite values and e
 * the smallest integer >= -127 with amax <= 448 * 2^e, the scale byte is e + 127 (0 for a group of zeros) and a code is the
 * 8-bit float (4 exponent bits, 3 mantissa bits, no infinities) nearest to x * 2^-e, ties to even.  Infinities and NaN are
 * held as NaN and do not touch their neighbours.  The value held is code * 2^e, which bfloat16 holds exactly (down to its
 * subnormal numbers, and but for 2^128, an infinity there, to which the largest numbers of 32 bits are rounded).
 *
 * Conventions
 *   - Data pointers are DEVICE pointers owned by the caller, of the current HIP device; nothing is kept, allocated or
 *     freed.  Calls are asynchronous on hip_stream (NULL: the default stream) and can be captured into a graph.
 *   - `type` is the element type of plain arrays.  A stride is the distance between rows in elements; the values of a row
 *     are neighbours.  No alignment beyond the element's is asked for.
 *   - Outputs are overwritten and must not overlap inputs.  Sums are formed in 32 bits or more, in an order fixed by the
 *     sizes: the same call gives the same bits.
 *   - Zero rows are fine and do nothing (gradients of weights become zeros).
 *   - Every function returns LEAP_OK (0) or a negative status of leap.h; the message is in leap_last_error().
 */
#ifndef LEAP_ACTIVATIONS_H
#define LEAP_ACTIVATIONS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { LEAP_F32 = 0, LEAP_BF16 = 1, LEAP_F16 = 2 };

/* codes, scales <- x [rows][cols] of `type`, rows `stride` elements apart. */
int leap_pack8(const void *d_x, int32_t type, int64_t stride, int64_t rows, int64_t cols, uint8_t *d_codes, uint8_t *d_scales,
               void *hip_stream);

/* out [rows][cols] of `type` (no gaps) <- the values held, rounded to nearest where the type does not hold them. */
int leap_unpack8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, void *d_out, int32_t type,
                 void *hip_stream);

/* The same, but for values beyond the type's largest number (2^128, float16's from 63488 on), which become that number instead of an infinity:
 * what was finite stays finite. */
int leap_unpack8_finite(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, void *d_out, int32_t type, void *hip_stream);

/* s = x + residual, rounded to `type` (residual NULL: s = x);  rstd = 1 / sqrt(mean over the row of s^2 + eps);
 * normed = packed s * rstd * weight;  kept = packed s, what the backward pass reads.
 * x, residual: [rows][cols] of `type` with strides; weight: [cols] of weight_type; sum: [rows][cols] of `type` or NULL;
 * kept codes and scales: both or neither (NULL); rstd: [rows] float or NULL. */
int leap_rms_norm8(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, int32_t type, const void *d_weight,
                   int32_t weight_type, int64_t rows, int64_t cols, float eps, void *d_sum, uint8_t *d_normed_codes,
                   uint8_t *d_normed_scales, uint8_t *d_kept_codes, uint8_t *d_kept_scales, float *d_rstd, void *hip_stream);

/* The gradient of leap_rms_norm8, the rounding to 8 bits taken as the identity.  With h = kept * rstd and
 * d = grad * weight:  grad_x = grad_sum + rstd * (d - h * mean over the row of d * h), which is the residual's gradient
 * too;  grad_weight = sum over rows of grad * h.  grad: [rows][cols] of grad_type with a stride; grad_sum (what reaches s
 * from elsewhere; NULL: none): [rows][cols] of `type` with a stride; grad_x: [rows][cols] of `type`; grad_weight: [cols] of
 * weight_type, or NULL.  d_work: leap_rms_norm8_work() floats (grad_weight NULL: may be NULL). */
int64_t leap_rms_norm8_work(int64_t rows, int64_t cols);
int leap_rms_norm8_backward(const void *d_grad, int32_t grad_type, int64_t grad_stride, const void *d_grad_sum, int64_t grad_sum_stride, int32_t type,
                            const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, const float *d_rstd, const void *d_weight,
                            int32_t weight_type, int64_t rows, int64_t cols, void *d_grad_x, void *d_grad_weight, float *d_work,
                            void *hip_stream);

/* y [rows][out] (bfloat16, no gaps) = v W^T, v the packed rows [rows][cols], W [out][cols] bfloat16, its rows w_stride apart.
 * d_work (all products): as many bytes as the function of that name + "_work" says, 16-byte aligned; NULL where it says 0.
 * It holds copies of what is not laid out for the kernels: codes whose columns are no multiple of 16, weights and gradients
 * whose rows do not begin and end at multiples of 16 bytes (the pointers handed over are looked at for that alone); and sums over
 * parts of long rows where outputs are few. */
int64_t leap_linear8_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out);
int leap_linear8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
                 int64_t out, void *d_y, void *d_work, void *hip_stream);

/* Its gradients: grad_x [rows][cols] = dy W, of grad_x_type (LEAP_BF16 or LEAP_F32), and grad_weight [out][cols] = dy^T v,
 * bfloat16; either may be NULL.  dy: [rows][out] bfloat16 with a stride. */
int64_t leap_linear8_backward_work(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight,
                                   int64_t w_stride, int64_t out);
int leap_linear8_backward(const void *d_dy, int64_t dy_stride, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols,
                          const void *d_weight, int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type,
                          void *d_grad_weight, void *d_work, void *hip_stream);

/* A fine gradient [rows][out] is the sum of two arrays of bfloat16, which holds it to 2^-17 of a value (bfloat16: 2^-9): its values rounded, and
 * what their rounding leaves.  They lie side by side: with P = out, up to a multiple of 8, a row is 2 * P long and has out values, zeros up to P, what
 * is left of each, and zeros; rows follow one another without gaps, from a multiple of 16 bytes on.  The same gradients as above from such a dy: products
 * take twice as long. */
int64_t leap_linear8_backward_fine_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out);
int leap_linear8_backward_fine(const void *d_dy, const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                               int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                               void *hip_stream);

/* The gated product.  u = v W^T in 32 bits with W [2 * out][cols], the gate's rows first: u = (g, p);
 * gated = packed g * sigmoid(g) * p, [rows][out];  kept = packed u as [rows][2][out] (the groups of the two halves apart), or
 * NULL.  d_work: leap_linear8_work() of this weight with its 2 * out rows. */
int leap_gated_linear8(const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride,
                       int64_t out, uint8_t *d_gated_codes, uint8_t *d_gated_scales, uint8_t *d_kept_codes, uint8_t *d_kept_scales,
                       void *d_work, void *hip_stream);

/* Its gradients from da = dL/d gated ([rows][out] bfloat16 with a stride): leap_gate8_backward (below), then leap_linear8_backward of du, which is
 * in the workspace, in bfloat16; grad_x [rows][cols] of grad_x_type and grad_weight [2 * out][cols], either may be NULL.  d_work:
 * leap_gated_linear8_backward_work() bytes, 16-byte aligned (no rows: may be NULL). */
int64_t leap_gated_linear8_backward_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out);
int leap_gated_linear8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales,
                                const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                                int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                                void *hip_stream);

/* The same with a fine du, so that grad_x and grad_weight are rounded once, at the end; the products take twice as long, and du twice the room. */
int64_t leap_gated_linear8_backward_fine_work(const uint8_t *d_codes, int64_t rows, int64_t cols, const void *d_weight, int64_t w_stride, int64_t out);
int leap_gated_linear8_backward_fine(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales,
                                     const uint8_t *d_codes, const uint8_t *d_scales, int64_t rows, int64_t cols, const void *d_weight,
                                     int64_t w_stride, int64_t out, void *d_grad_x, int32_t grad_x_type, void *d_grad_weight, void *d_work,
                                     void *hip_stream);

/* du [rows][2 * out] (bfloat16) from kept = (g, p) and da = dL/d gated: the gate's half da * p * s * (1 + g * (1 - s)), the
 * other da * g * s, with s = sigmoid(g).  With u's gradient in hand leap_linear8_backward gives those of v and W.
 * leap_gate8_backward reads da [rows][out] (bfloat16, with a stride); leap_linear_gate8_backward forms it, in 32 bits, as
 * dy W with W [next][out] bfloat16 (the weight of the product that read `gated`) and dy [rows][next] bfloat16.
 * d_work: leap_linear_gate8_work() bytes. */
int leap_gate8_backward(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows,
                        int64_t out, void *d_du, void *hip_stream);
int64_t leap_linear_gate8_work(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next, int64_t rows, int64_t out);
int leap_linear_gate8_backward(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next,
                               const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                               void *d_work, void *hip_stream);

/* The same to a fine du (of 2 * out values a row, from a multiple of 16 bytes on). */
int leap_gate8_backward_fine(const void *d_da, int64_t da_stride, const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows,
                             int64_t out, void *d_du, void *hip_stream);
int leap_linear_gate8_backward_fine(const void *d_dy, int64_t dy_stride, const void *d_weight, int64_t w_stride, int64_t next,
                                    const uint8_t *d_kept_codes, const uint8_t *d_kept_scales, int64_t rows, int64_t out, void *d_du,
                                    void *d_work, void *hip_stream);

/* A feed-forward block of these, as one call:  s = x + residual (NULL: s = x);  y [rows][out] = gated(norm(s) up^T) down^T, with up
 * [2 * hidden][cols] and down [out][hidden], their rows up_stride and down_stride apart, everything plain in bfloat16 (the norm's
 * weight in norm_weight_type).  d_sum: [rows][cols], or NULL.  d_kept: leap_feed_forward8_kept() bytes, 16-byte aligned, that the backward
 * pass reads: what the operators above keep, in 8 bits.  d_work: leap_feed_forward8_work() bytes, NULL where that is 0.
 * Backward: grad_x (the residual's gradient too), and the weights' gradients, each [as its weight] without gaps; NULL for what is not
 * wanted (the norm's weight gradient comes with grad_x).  grad_sum: what reaches s from elsewhere, or NULL.  d_work:
 * leap_feed_forward8_backward_work() bytes, 16-byte aligned, never NULL. */
int64_t leap_feed_forward8_kept(int64_t rows, int64_t cols, int64_t hidden);
int64_t leap_feed_forward8_work(int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden, const void *d_down,
                                int64_t down_stride, int64_t out);
int leap_feed_forward8(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, const void *d_norm_weight,
                       int32_t norm_weight_type, int64_t rows, int64_t cols, float eps, const void *d_up, int64_t up_stride, int64_t hidden,
                       const void *d_down, int64_t down_stride, int64_t out, void *d_sum, void *d_y, void *d_kept, void *d_work,
                       void *hip_stream);
/* Forward with nothing kept, where no backward pass follows: y and d_sum are those of leap_feed_forward8.  d_work: as many bytes as the function
 * with "_work" says, 16-byte aligned, never NULL (no rows: may be NULL). */
int64_t leap_feed_forward8_alone_work(int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden, const void *d_down,
                                      int64_t down_stride, int64_t out);
int leap_feed_forward8_alone(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, const void *d_norm_weight,
                             int32_t norm_weight_type, int64_t rows, int64_t cols, float eps, const void *d_up, int64_t up_stride, int64_t hidden,
                             const void *d_down, int64_t down_stride, int64_t out, void *d_sum, void *d_y, void *d_work, void *hip_stream);
int64_t leap_feed_forward8_backward_work(const void *d_dy, int64_t dy_stride, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride,
                                         int64_t hidden, const void *d_down, int64_t down_stride, int64_t out);
int leap_feed_forward8_backward(const void *d_dy, int64_t dy_stride, const void *d_grad_sum, int64_t grad_sum_stride, const void *d_norm_weight,
                                int32_t norm_weight_type, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden,
                                const void *d_down, int64_t down_stride, int64_t out, const void *d_kept, void *d_grad_x,
                                void *d_grad_norm_weight, void *d_grad_up, void *d_grad_down, void *d_work, void *hip_stream);

/* The same with a fine du, the gradient of the product with `up` (leap_gated_linear8_backward_fine says what that takes and gives). */
int64_t leap_feed_forward8_backward_fine_work(const void *d_dy, int64_t dy_stride, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride,
                                              int64_t hidden, const void *d_down, int64_t down_stride, int64_t out);
int leap_feed_forward8_backward_fine(const void *d_dy, int64_t dy_stride, const void *d_grad_sum, int64_t grad_sum_stride, const void *d_norm_weight,
                                     int32_t norm_weight_type, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden,
                                     const void *d_down, int64_t down_stride, int64_t out, const void *d_kept, void *d_grad_x,
                                     void *d_grad_norm_weight, void *d_grad_up, void *d_grad_down, void *d_work, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
