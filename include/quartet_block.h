/*
 * quartet_block.h -- C ABI of what a transformer block runs around the quantized linear layers of quartet.h, in the same library:
 * a product's bias, activation, gate and residual in its epilogue (and their backward pass), the root-mean-square norm of the residual
 * stream straight into a layer's 4- or 8-bit operand (and its backward pass), and the norm and clipping of a step's gradients.
 *
 * Everything quartet.h says about its entry points holds here: device pointers owned by the caller, 16-byte aligned unless a function
 * says otherwise; row-major matrices with leading dimensions in elements; work enqueued on `stream`, no allocation, no synchronization,
 * nothing cleared by hipMemsetAsync (calls can be captured into a HIP graph); arguments are checked on the host before anything is
 * launched; the same return values.  Empty calls (a zero size) launch nothing where there is nothing to write.  Results do not depend on
 * anything but the arguments: there are no atomics, two calls on the same inputs give the same bits.
 *
 * Number formats: sums and activations are formed in fp32 (the squares of the norm's statistic and of the gradient norm, and their sums, in fp64) and every
 * result is rounded once, to nearest even, where it is stored.  Infinities and NaN pass through the arithmetic as IEEE rules have it, except where a result is an MX
 * operand (an E4M3 element saturates at 448, an E2M1 element at 6; a NaN makes its group's codes unspecified).
 */
#ifndef QUARTET_BLOCK_H
#define QUARTET_BLOCK_H

#include "quartet.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QUARTET_ACT_NONE 0 /* a(z) = z */
#define QUARTET_ACT_RELU 1 /* max(z, 0) */
#define QUARTET_ACT_GELU 2 /* z s(2 c (z + 0.044715 z^3)), c = sqrt(2 / pi), s(t) = 1 / (1 + exp(-t)): the tanh form of the Gaussian unit */
#define QUARTET_ACT_SILU 3 /* z s(z) */

#define QUARTET_FORMAT_NONE 0
#define QUARTET_FORMAT_MXFP4 1 /* quartet_quant_fwd's: rotated, E2M1 codes, tiled E8M0 scales */
#define QUARTET_FORMAT_MXFP8 2 /* quartet_mxfp8_quant's: E4M3 codes, tiled E8M0 scales */

/* kinds of launches in quartet_profile_read's record, beside those of quartet.h (quartet_mxfp4_gemm_act is a QUARTET_KIND_GEMM) */
#define QUARTET_KIND_NORM 8
#define QUARTET_KIND_ACT 9
#define QUARTET_KIND_CLIP 10

/*
 * Product with its epilogue:  z = alpha * A B^T + bias;  D = a(z) * multiplier + residual.
 * A [m x k], B [n x k], D [m x n] and their limits as quartet_mxfp4_gemm (m, n arbitrary, k % 32 == 0, n <= ldd <= 2^21).
 * bias [n] of bias_dtype (fp32 or bf16) or NULL; multiplier bf16 [m x ldmul] (a gated layer's other branch) or NULL; residual
 * [m x ldres] of residual_dtype or NULL; pre: where z is stored as bf16 [m x ldpre] for quartet_act_bwd, or NULL.  The activation works
 * on z in fp32, not on its stored copy.  Leading dimensions of the matrices that are given lie between n and 2^21.  multiplier or residual
 * may be d itself (same type and leading dimension): every element is read before it is written.  Other overlaps of d or pre with an
 * argument are errors the library does not look for.  It runs on the tiles that quartet_mxfp4_gemm would take (quartet_debug_set_gemm_plan
 * included), with the same order of sums; results of 256 MiB and more are stored through the caches here.  Fastest where n and all leading
 * dimensions are multiples of 4.
 */
int quartet_mxfp4_gemm_act(const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes, const uint8_t *b_scales,
                           int64_t m, int64_t n, int64_t k, float alpha, const void *bias, int bias_dtype, int activation,
                           const void *multiplier_bf16, int64_t ldmul, const void *residual, int residual_dtype, int64_t ldres,
                           void *pre_bf16, int64_t ldpre, void *d, int d_dtype, int64_t ldd, void *stream);

/*
 * Backward pass of that epilogue: with z = pre and dy = the gradient of D (also the residual's gradient as it stands),
 *   dz = dy * multiplier * a'(z)   (the product's gradient: what quartet_linear_bwd takes as dy; a'(0) = 0 for RELU),
 *   dmul = dy * a(z)               (the multiplier's gradient),
 *   dbias[j] = sum over the rows of dz[., j], of the unrounded values, in fp32 and in a fixed order.
 * dy, pre, multiplier, dz, dmul: bf16 [m x ld], m, n >= 0, leading dimensions multiples of 8 and at least n; dz, dmul and dbias may each be
 * NULL (not all three), multiplier may be NULL (ones); pre may be NULL for QUARTET_ACT_NONE without dmul.  dz may be dy itself, and dmul may be
 * multiplier or pre itself (with the same leading dimension).  workspace: quartet_act_bwd_workspace_bytes(m, n) bytes, 16-byte aligned, needed only
 * with dbias.  m < 2^31, n <= 2^26.
 */
size_t quartet_act_bwd_workspace_bytes(int64_t m, int64_t n);
int quartet_act_bwd(const void *dy_bf16, int64_t lddy, const void *pre_bf16, int64_t ldpre, const void *multiplier_bf16, int64_t ldmul,
                    int64_t m, int64_t n, int activation, void *dz_bf16, int64_t lddz, void *dmul_bf16, int64_t lddmul, float *dbias,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * Root-mean-square norm, over the residual stream where there is one:
 *   h = x + residual, rounded to h_dtype (without residual: h = x);  rstd = 1 / sqrt(mean(h^2) + eps);  v = h * rstd * weight.
 * x [rows x ldx] of x_dtype, residual [rows x ldres] of h_dtype or NULL, weight [n] of weight_dtype.  Stored, each if its pointer is not
 * NULL: h [rows x ldh] (only with residual; may be residual itself, or x where x_dtype = h_dtype, with the same leading dimension), v as bf16
 * y [rows x ldy], rstd [rows] fp32 (for quartet_rmsnorm_bwd).  format QUARTET_FORMAT_MXFP8 or _MXFP4: v, unrounded, as the operand that
 * quartet_mxfp8_quant or quartet_quant_fwd (Hadamard blocks of 32) makes of its argument: codes, tiled scales (quartet_scale_bytes(rows, n)) and, with
 * MXFP4, the clipping mask if it is not NULL (otherwise mask must be NULL); needs n % 32 == 0.  QUARTET_FORMAT_NONE: codes, scales and mask NULL.
 * 1 <= n <= 32768, leading dimensions multiples of 8, eps >= 0 and finite.  rows * ceil(n / 32) < 2^31.
 */
int quartet_rmsnorm_fwd(const void *x, int x_dtype, int64_t ldx, const void *residual, int64_t ldres, int64_t rows, int64_t n,
                        const void *weight, int weight_dtype, float eps, void *h, int h_dtype, int64_t ldh, void *y_bf16, int64_t ldy,
                        int format, uint8_t *codes, uint8_t *scales, uint32_t *mask, float *rstd, void *stream);

/*
 * Backward pass: dy bf16 [rows x lddy] is the gradient of v, dh (or NULL) the gradient that reaches h along the stream;
 *   g = dy * weight;  dx = rstd * (g - h * rstd^2 * mean(g * h)) + dh   (gradient of x and of residual alike);
 *   dweight[j] = sum over the rows of dy * h * rstd, in fp32 and in a fixed order.
 * h, dh, dx [rows x ld] of h_dtype (without a residual h is the forward pass's x, of its type).  dx16: a bf16 copy of dx beside an fp32 one (for
 * quartet_linear_bwd), or NULL; must be NULL for bf16.  dx and dweight may each be NULL (not both; dx16 goes with dx).  dx may be dh itself or h itself (with
 * the same leading dimension), dx16 may be dy itself.  Sizes as above; workspace:
 * quartet_rmsnorm_bwd_workspace_bytes(rows, n) bytes, 16-byte aligned, needed only with dweight.
 */
size_t quartet_rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t n);
int quartet_rmsnorm_bwd(const void *dy_bf16, int64_t lddy, const void *h, int h_dtype, int64_t ldh, int64_t rows, int64_t n,
                        const void *weight, int weight_dtype, const float *rstd, const void *dh, int64_t lddh, void *dx, int64_t lddx,
                        void *dx16, int64_t lddx16, float *dweight, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Norm of all gradients of a step and their copies scaled to a largest norm:
 *   norm = sqrt(sum over all tensors of g^2);  out = g * min(1, max_norm / (norm + 1e-6)).
 * tensors: HOST array of `count` entries (read during the call); grad and out need the alignment of their elements only.  out may be grad itself (clipping
 * in place, same type): then nothing is written where the factor is 1.  No out may overlap any other out or grad (QUARTET_EINVAL).  A norm that is not
 * finite stands for a step to be skipped: the factor is 1 then, so out holds the gradients as they are.  norm: one device float.  max_norm >= 0; INFINITY: no
 * clipping, and with out = grad just the norm.  The squares are summed in fp64, in an order that depends on the sizes alone.  workspace:
 * quartet_grad_clip_workspace_bytes() bytes, 16-byte aligned.  The sizes together are below 2^43; count <= 2^15.
 */
typedef struct quartet_grad_tensor {
    const void *grad;
    void *out;
    int64_t size;               /* elements, >= 0; with 0 the pointers are not looked at */
    int grad_dtype, out_dtype;
} quartet_grad_tensor;
size_t quartet_grad_clip_workspace_bytes(void);
int quartet_grad_clip(const quartet_grad_tensor *tensors, int64_t count, float max_norm, float *norm, void *workspace,
                      size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* QUARTET_BLOCK_H */
