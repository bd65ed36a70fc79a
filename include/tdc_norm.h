/*
 * tdc_norm.h -- group normalisation with an activation on channels-last images, forward and backward.
 *
 * The norm of networks that normalise every image by itself, which cannot be folded into the weights of a convolution the way
 * tdc_epilogue's bias assumes.  x is [batch][H][W][C] (layout 1 of tdc.h); the C channels form `groups` groups of C/groups
 * neighbours.  With n = H*W*C/groups values in a group,
 *     mean[b][g] = sum x / n,   rstd[b][g] = 1 / sqrt(sum (x - mean)^2 / n + eps),
 *     xhat = (x - mean) * rstd,   pre = xhat * gamma[c] + beta[c] (+ residual),   y = act(pre).
 *
 * Rules that differ from tdc.h: activations are fp32, fp16 or bf16 (tdc_dtype), gamma, beta and the statistics fp32.
 * Arithmetic is fp32, rounded once where y is stored.  Activation pointers need only be aligned to their elements; calls are
 * fastest with C, the pitches and the pointers multiples of 16 bytes.  As in tdc.h the calls only enqueue work on `hip_stream`,
 * allocate nothing and may be captured into a HIP graph; a plan's workspace serves one call at a time, so calls on one plan,
 * and replays of graphs that hold such calls, must be ordered one after the other.  Outputs must not overlap inputs.
 * Results do not depend on timing: no atomics, the same bits every time.
 */
#ifndef TDC_NORM_H
#define TDC_NORM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of activations. */
enum { TDC_F32 = 0, TDC_F16 = 1, TDC_BF16 = 2 };

/* Activations.  TDC_ACT_SILU: v / (1 + exp(-v)). */
enum { TDC_ACT_NONE = 0, TDC_ACT_RELU = 1, TDC_ACT_SILU = 2 };

/* batch 1..65535, H*W < 2^31, C 1..8192 and a multiple of groups, eps >= 0; else TDC_ERR_BAD_SHAPE (sizes that mean nothing) or
 * TDC_ERR_UNSUPPORTED (unknown dtype or act, C, batch or H*W too large). */
typedef struct tdc_norm_shape {
    int32_t batch, H, W, C, groups;
    int32_t dtype;                /* of x, y, residual and their gradients */
    int32_t act;
    float eps;
} tdc_norm_shape;

typedef struct tdc_norm_plan tdc_norm_plan;   /* opaque, library-owned */

int tdc_norm_plan_create(tdc_norm_plan **out, const tdc_norm_shape *shape, int device);
int tdc_norm_plan_destroy(tdc_norm_plan *plan);                    /* NULL is accepted */
size_t tdc_norm_plan_workspace_bytes(const tdc_norm_plan *plan);   /* device bytes owned */
/* Launches of a tdc_group_norm and of a tdc_group_norm_mx4 call on 16-byte aligned tensors without gaps. */
int tdc_norm_plan_kernel_count(const tdc_norm_plan *plan);
int tdc_norm_plan_mx4_kernel_count(const tdc_norm_plan *plan);

/* Optional arguments.  A NULL tdc_norm_args, or zero in a field, is the default.
 * A pitch is the number of ELEMENTS from one pixel to the next (0: C; otherwise at least C), so a tensor may be a slice of the
 * channels of wider pixels; rows and images follow one another without gaps. */
typedef struct tdc_norm_args {
    const void *residual;         /* added before the activation, or NULL                      */
    float *mean, *rstd;           /* [batch][groups], written for the backward pass, or NULL   */
    int64_t x_pitch, residual_pitch, y_pitch;
} tdc_norm_args;

/* Enqueue y = act(group_norm(x) * gamma + beta + residual).  gamma, beta: [C], NULL for ones / zeros. */
int tdc_group_norm(tdc_norm_plan *plan, void *hip_stream, const void *x, const float *gamma, const float *beta, void *y,
                   const tdc_norm_args *args);

/* The same, written in 4 bits for a product that reads them (tdc_mx4.h: rows are pixels, blocks of 32 channels): the fp32
 * values before any rounding to dtype are quantised.  codes: [batch*H*W][ceil(C/32)][16], 16-byte aligned;
 * scales: [batch*H*W][ceil(C/32)]. */
int tdc_group_norm_mx4(tdc_norm_plan *plan, void *hip_stream, const void *x, const float *gamma, const float *beta,
                       uint8_t *codes, uint8_t *scales, const tdc_norm_args *args);

/* Optional arguments of the backward pass, as above.  residual is the forward pass's (needed for its activation, where there
 * is one); dresidual receives its gradient, shaped like residual. */
typedef struct tdc_norm_grad_args {
    const void *residual;
    void *dresidual;
    int64_t x_pitch, residual_pitch, dy_pitch, dx_pitch, dresidual_pitch;
} tdc_norm_grad_args;

/* Gradients of tdc_group_norm, from the mean and rstd that it wrote.  With d = dy * act'(pre) (TDC_ACT_RELU: dy where pre > 0, 0
 * where pre <= 0 whatever dy is, NaN where pre is one), g = d * gamma and m(.) the mean over a group of an image,
 *     dx = rstd * (g - m(g) - xhat * m(g * xhat)),   dgamma[c] = sum d * xhat,   dbeta[c] = sum d,   dresidual = d.
 * dx: like x.  dgamma, dbeta: [C], overwritten, NULL where not wanted. */
int tdc_group_norm_backward(tdc_norm_plan *plan, void *hip_stream, const void *x, const void *dy, const float *mean,
                            const float *rstd, const float *gamma, const float *beta, void *dx, float *dgamma, float *dbeta,
                            const tdc_norm_grad_args *args);

#ifdef __cplusplus
}
#endif
#endif /* TDC_NORM_H */
