// What the 4-bit kernels' translation units share.
#ifndef TDC_MX4_INTERNAL_H
#define TDC_MX4_INTERNAL_H

#include "tdc_mx4_device.h"
#include "tdc_typed.h"

inline int tdc_mx4_blocks(int cols) { return (cols + TDC_MX4_BLOCK - 1) / TDC_MX4_BLOCK; }

// Which row of the operand an output row reads: itself, or the pixel that a strided 1x1 convolution reads.
struct TdcMx4Rows {
    int stride;              // 1: row m itself, the other fields unused
    int Wo, HoWo, W, HW;
    static TdcMx4Rows all() { return TdcMx4Rows{1, 0, 0, 0, 0}; }
    __host__ __device__ int64_t source(int64_t m) const
    {
        if (stride == 1) return m;
        const int64_t b = m / HoWo;
        const int q = (int)(m - b * HoWo), i = q / Wo, j = q - i * Wo;
        return b * HW + (int64_t)i * stride * W + (int64_t)j * stride;
    }
};

struct TdcMx4Epi {
    const float *bias;       // [N] or null
    const void *residual;    // shaped like y, of its type, or null
    int act;
};

// y[M][N] = A B^T, both in rows of nb blocks; row m of the product reads row a_rows.source(m) of A.
struct TdcMx4Product {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    int M, N, nb;
    TdcMx4Rows a_rows;
    void *y;
    TdcMx4Epi epi;
    bool vec;                // y and the residual can be accessed 16 bytes at a time
};

// Whether the kernels' grids cover M x N outputs.
inline bool tdc_mx4_product_fits(int64_t M, int64_t N) { return ((M + 31) / 32) * ((N + 31) / 32) < 0x7fffffff / 256; }

hipError_t tdc_launch_mx4_product(const TdcMx4Product &q, int dtype, hipStream_t s);

#endif  // TDC_MX4_INTERNAL_H
