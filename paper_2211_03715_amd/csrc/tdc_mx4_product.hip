// Products of operands in microscaled 4-bit floating point on the matrix cores (tdc_mx4.h).
//
// Large ones in tiles (tdc_mx4_tile.h), the others by rows (tdc_mx4_rows.hip).
//
// v_mfma_scale_f32_32x32x64: lane l holds the 32 values of row l%32 that one block of k holds (block l/32 of the two), 16
// bytes, with the block's scale beside it, so an operand in the format's own layout needs no rearrangement.  Of the result,
// register i of lane l is element [m = 8*(i/4) + 4*(l/32) + i%4][n = l%32] with rows of A as m and rows of B as n.
#include "tdc_mx4_tile.h"

namespace {

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

hipError_t tdc_launch_mx4_product(const TdcMx4Product &given, int dtype, hipStream_t s)
{
    TdcMx4Product q = given;
    q.vec = tdc_mx4_vec(q, dtype);
    // Tiles of 256 x 256 where over half of the compute units get one (3300 x 2600 x 900, 143 of them: 15.9 us, in tiles of
    // 128 x 128 18.4; 4096 x 2048 x 1024, 128 of them: 13.4 and 9.3; but 3200 x 2560 x 2048, 130 of them: 20.0 and 14.4), of
    // 128 x 128 from 64 of those on; below that, and for few rows, every 32 rows and 64 columns by themselves (700 x 700 x 2048, 36
    // tiles of 128 x 128: 9.4 us by rows, 15.2 in tiles).
    const int64_t large = up(q.M, 256) * up(q.N, 256), small = up(q.M, 128) * up(q.N, 128);
    if (q.M <= 64 || small < 64) return tdc_launch_mx4_rows(q, TdcMx4Source{nullptr, 0, 0}, dtype, nullptr, nullptr, s);
    const bool packed = q.nb % 16 == 0 && tdc_aligned_to(q.a_scales, 16) && tdc_aligned_to(q.b_scales, 16);
    TDC_FOR_DTYPE(dtype, T, {
        if (large > 128) {
            if (packed) tdc_mx4_product_tile<T, 4, 2, 2, 4, true><<<(unsigned)large, 512, 0, s>>>(q);
            else tdc_mx4_product_tile<T, 4, 2, 2, 4, false><<<(unsigned)large, 512, 0, s>>>(q);
        } else {
            if (packed) tdc_mx4_product_tile<T, 2, 2, 2, 2, true><<<(unsigned)small, 256, 0, s>>>(q);
            else tdc_mx4_product_tile<T, 2, 2, 2, 2, false><<<(unsigned)small, 256, 0, s>>>(q);
        }
    });
    return hipGetLastError();
}
