/*
 * tdc_mx4.h -- microscaled 4-bit floating point: quantisation, and the 1x1 convolutions around a Tucker layer as products of it.
 *
 * Format.  A row of values is cut into blocks of 32; a block holds 32 codes of 4 bits (sign, 2 bits of exponent, 1 of mantissa:
 * 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) and one byte e, and stands for code * 2^(e - 127).  A row of `cols` values
 * has nb = ceil(cols/32) blocks: codes [rows][nb][16], value 2i in the low half of byte i, zeros behind the last value;
 * scales [rows][nb].  e = 255 makes the whole block NaN.
 * Quantisation.  With amax the block's largest magnitude, e = 127 + clamp(floor(log2 amax) - 2, -127, 127), e = 0 where amax is
 * 0; every value v becomes the code nearest to v * 2^(127 - e), ties to the even code, magnitudes above 6 become 6.  A block
 * that holds an infinity or a NaN gets e = 255.  The result is exact: it depends on nothing but the values.
 *
 * Products sum in fp32 on the matrix cores that multiply such blocks directly.  As in tdc.h the calls only enqueue work on
 * `hip_stream`, allocate nothing and may be captured; codes must be 16-byte aligned, the other pointers to their elements.  Rows
 * may have up to 2^30 values; what is more than a launch can cover, see each call, is TDC_ERR_UNSUPPORTED.
 * Outputs must not overlap inputs.  Calls without a plan run on the calling thread's CURRENT device, which must be the
 * stream's and the tensors'.
 */
#ifndef TDC_MX4_H
#define TDC_MX4_H

#include <stddef.h>
#include <stdint.h>

#include "tdc_norm.h"   /* tdc_dtype and the activations */

#ifdef __cplusplus
extern "C" {
#endif

/* codes, scales <- the rows of x: [rows] of `cols` values of dtype TDC_F32 / F16 / BF16, `pitch` elements apart (0: cols).
 * rows = 0 is accepted and does nothing.  TDC_ERR_UNSUPPORTED for more than 2^31 - 128 blocks, rows * ceil(cols/32). */
int tdc_mx4_quantize(void *hip_stream, const void *x, int dtype, int64_t rows, int64_t cols, int64_t pitch, uint8_t *codes,
                     uint8_t *scales);

/* y <- the values of codes and scales, rounded to dtype (fp16: values beyond its range become infinite).  The same limit. */
int tdc_mx4_dequantize(void *hip_stream, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *y,
                       int dtype, int64_t pitch);

/* What a product does to its sums before it stores them: y = act(sum + bias[n] + residual[m][n]).  bias: [N] fp32 or NULL;
 * residual: shaped like y, of its dtype, or NULL.  A NULL epilogue is none. */
typedef struct tdc_mx4_epilogue {
    const float *bias;
    const void *residual;
    int32_t act;
} tdc_mx4_epilogue;

/* y[M][N] = A[M][K] B[N][K]^T: both operands in rows of K values in 4 bits; y is stored in `dtype`.
 * M = 0 is accepted and does nothing.  TDC_ERR_UNSUPPORTED for N over 2^24, or when ceil(M/256) * ceil(N/256) reaches 2^23 (some
 * 2^39 outputs). */
int tdc_mx4_matmul(void *hip_stream, const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                   const uint8_t *b_scales, int32_t M, int32_t N, int32_t K, void *y, int dtype,
                   const tdc_mx4_epilogue *epilogue);

/* A 1x1 convolution on channels-last images with weights in 4 bits: x [batch][H][W][C] -> y [batch][Ho][Wo][N], with
 * Ho = ceil(H/stride), Wo = ceil(W/stride); output (i, j) reads input (i*stride, j*stride).  x_pitch: elements from one input
 * pixel to the next (0: C; else at least C).  TDC_ERR_UNSUPPORTED for an unknown dtype, for N over 2^24, when batch*H*W reaches
 * 2^31, or when the output's pixels, px = batch*Ho*Wo, pass 2^29 - 32, ceil(px/256) * ceil(N/256) reaches 2^23, or
 * px * ceil(C/32) passes 2^31 - 128. */
typedef struct tdc_mx4_shape {
    int32_t batch, H, W, C, N, stride;
    int32_t dtype;                /* of x, y and residual */
    int64_t x_pitch;
} tdc_mx4_shape;

typedef struct tdc_mx4_plan tdc_mx4_plan;   /* opaque, library-owned: the weights in 4 bits and the workspace */

int tdc_mx4_plan_create(tdc_mx4_plan **out, const tdc_mx4_shape *shape, int device);
int tdc_mx4_plan_destroy(tdc_mx4_plan *plan);                    /* NULL is accepted */
size_t tdc_mx4_plan_workspace_bytes(const tdc_mx4_plan *plan);   /* device bytes owned */
int tdc_mx4_plan_kernel_count(const tdc_mx4_plan *plan);         /* launches per tdc_conv_mx4 call */

/* Quantise W[C][N] (fp32, the dense kernel W[C][N][1][1] of tdc.h; blocks run along C) into plan-owned memory, once.  W is not
 * read afterwards.  A convolution on another stream must be ordered after this call by the caller.  A convolution before any
 * pack returns TDC_ERR_NULL. */
int tdc_mx4_plan_pack(tdc_mx4_plan *plan, void *hip_stream, const float *W);

/* y = conv(x) with x in floating point, which is quantised along C on the way, exactly as tdc_mx4_quantize would.  The plan's
 * workspace serves one call at a time, as in tdc_norm.h. */
int tdc_conv_mx4(tdc_mx4_plan *plan, void *hip_stream, const void *x, void *y, const tdc_mx4_epilogue *epilogue);

/* The same with x already in 4 bits, one row for every input pixel (tdc_group_norm_mx4, tdc_mx4_quantize). */
int tdc_conv_mx4_quantized(tdc_mx4_plan *plan, void *hip_stream, const uint8_t *codes, const uint8_t *scales, void *y,
                           const tdc_mx4_epilogue *epilogue);

#ifdef __cplusplus
}
#endif
#endif /* TDC_MX4_H */
