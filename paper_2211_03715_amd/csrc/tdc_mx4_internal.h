// What the 4-bit kernels' translation units share.
#ifndef TDC_MX4_INTERNAL_H
#define TDC_MX4_INTERNAL_H

#include "tdc_div.h"
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
        const int b = (int)m / HoWo, q = (int)m - b * HoWo, i = q / Wo, j = q - i * Wo;    // a plan's pixels are under 2^31
        return (int64_t)b * HW + (int64_t)i * stride * W + (int64_t)j * stride;
    }
};

// Division of 64-bit indices by a launch-time constant: by 32-bit multiplication where the index allows it.
struct TdcMx4Div {
    int d;
    TdcDiv by;
    explicit TdcMx4Div(int n) : d(n), by(tdc_make_div(n)) {}
    __device__ int64_t of(int64_t i) const
    {
        if (i >> 32) return i / d;
        const unsigned u = (unsigned)i;
        return tdc_div_from_hi(u, __umulhi(by.m, u), by);
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
    bool vec;                // y, the residual and the bias can be accessed 16 bytes at a time
};

inline bool tdc_mx4_vec(const TdcMx4Product &q, int dtype)
{
    return q.N % (16 / tdc_dtype_bytes(dtype)) == 0 && tdc_aligned_to(q.y, 16) && tdc_aligned_to(q.epi.residual, 16) && tdc_aligned_to(q.epi.bias, 16);
}

// A launch counts its threads in 32 bits.  Workgroups of 256 threads quantise 128 blocks at least, or have 32 rows of a convolution;
// those of 512 have 256 x 256 outputs, or, in smaller tiles and by rows, launches are small.
constexpr int64_t TDC_MX4_MAX_WORKGROUPS = (1 << 24) - 1;
constexpr int64_t TDC_MX4_MAX_BLOCKS = 128 * TDC_MX4_MAX_WORKGROUPS;
constexpr int64_t TDC_MX4_MAX_ROWS = 32 * TDC_MX4_MAX_WORKGROUPS;
inline bool tdc_mx4_product_fits(int64_t M, int64_t N) { return ((M + 255) / 256) * ((N + 255) / 256) <= TDC_MX4_MAX_WORKGROUPS / 2; }

hipError_t tdc_launch_mx4_product(const TdcMx4Product &q, int dtype, hipStream_t s);

// Rows of A in floating point, quantised on the way (a_codes, a_scales unused), or x null.
struct TdcMx4Source {
    const void *x;
    int64_t pitch;
    int cols;
};

// Weights as tdc_mx4_rows.hip takes them.
size_t tdc_mx4_laid_out_bytes(int N, int nb);
size_t tdc_mx4_laid_out_scale_bytes(int N, int nb);
hipError_t tdc_launch_mx4_lay_out(const uint8_t *codes, const uint8_t *scales, int N, int nb, uint8_t *w, uint8_t *ws, hipStream_t s);
// The product with laid-out weights, or, w and ws null, with q's own second operand.  prepare_only: what must precede a first
// launch, without one.
hipError_t tdc_launch_mx4_rows(const TdcMx4Product &q, const TdcMx4Source &src, int dtype, const uint8_t *w, const uint8_t *ws, hipStream_t s, bool prepare_only = false);

constexpr int TDC_MX4_MAX_COLS = 1 << 30;
constexpr int TDC_MX4_MAX_OUT = 1 << 24;   // a lane's offset of some rows of y stays under 2^32 bytes

// A convolution that the matrix cores bound rather than memory runs as quantisation and a product in large tiles.  By rows and so, us:
// bf16, 4096 rows, 1024 -> 1024 14.1 and 11.5, 2048 -> 2048 40.5 and 20.5, 512 -> 1024 9.5 and 9.7, 1024 -> 512 12.1 and 11.3;
// 2048 rows, 512 -> 1024 7.1 and 9.1; 25088 rows, 1024 -> 1024 36.3 and 39.4, 2048 -> 1024 90.5 and 66.7; fp32, 4096 rows,
// 1024 -> 1024 17.2 and 13.2; 25088 rows, 64.0 and 57.6.  Below the limits
// either wins; long sums are better so from 2048 rows or 512 columns on (2048 rows, 2048 -> 2048 in bf16: 23.4 and 14.3).
inline bool tdc_mx4_large(int64_t rows, int N, int K) { return rows >= 4096 && N >= 1024 && K >= 1024; }

// Whether tdc_launch_mx4_rows gives a workgroup 32 rows and only 64 columns, eight wavefronts along k.
inline bool tdc_mx4_few(int64_t rows, int N) { return (rows + 31) / 32 * ((N + 63) / 64) <= 512; }

// Every one of those quantises its rows of x anew, which takes longer than a launch where they have over 192 KB.  On the way and in a
// launch of its own: 64 rows, 4096 -> 4096 in bf16 (262 KB) 18.9 us and 12.1; 1568 rows, 2048 -> 512 in fp32 (262 KB) 20.8 and 13.4;
// 49 such rows 9.4 and 8.8; in bf16 (131 KB) 1568 rows 16.5 and 12.3, 196 rows 10.2 and 9.0, but 1024 -> 256 in fp32 (131 KB), 196
// rows, 6.6 and 8.1; 6272 rows, 512 -> 128 in fp32 (66 KB) 9.1 and 10.8.
inline bool tdc_mx4_quantise_first(int64_t rows, int N, int K, int size) { return tdc_mx4_few(rows, N) && (double)(rows < 32 ? rows : 32) * K * size > 192e3; }

#endif  // TDC_MX4_INTERNAL_H
