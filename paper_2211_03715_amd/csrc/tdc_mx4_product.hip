// Products of operands in microscaled 4-bit floating point on the matrix cores (tdc_mx4.h).
//
// v_mfma_scale_f32_32x32x64: lane l holds the 32 values of row l%32 that one block of k holds (block l/32 of the two), 16
// bytes, with the block's scale beside it, so an operand in the format's own layout needs no rearrangement.  Of the result,
// register i of lane l is element [m = 8*(i/4) + 4*(l/32) + i%4][n = l%32] with rows of A as m and rows of B as n.
#include "tdc_mx4_tile.h"

namespace {

// A wavefront to 32 x 32 outputs, operands straight from memory.
template <typename T>
__global__ __launch_bounds__(256) void tdc_mx4_product_simple(TdcMx4Product q)
{
    const int l = threadIdx.x & 63, nblocks = (q.N + 31) / 32;
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), tiles = (int64_t)((q.M + 31) / 32) * nblocks;
    if (tile >= tiles) return;
    const int m0 = (int)(tile / nblocks) * 32, n0 = (int)(tile % nblocks) * 32;
    // rows past the end read the last one: what they give is not stored
    const size_t ra = (size_t)q.a_rows.source(min(m0 + (l & 31), q.M - 1)) * q.nb, rb = (size_t)min(n0 + (l & 31), q.N - 1) * q.nb;
    tdc_f16v acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    for (int k = 0; k < q.nb; k += 2) {
        const int kb = k + (l >> 5);
        tdc_i4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        unsigned sa = 0, sb = 0;
        if (kb < q.nb) {
            a = *reinterpret_cast<const tdc_i4 *>(q.a_codes + (ra + kb) * 16);
            b = *reinterpret_cast<const tdc_i4 *>(q.b_codes + (rb + kb) * 16);
            sa = q.a_scales[ra + kb];
            sb = q.b_scales[rb + kb];
        }
        acc = tdc_mx4_mfma<0>(a, sa, b, sb, acc);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int m = m0 + 8 * (i / 4) + 4 * (l >> 5) + i % 4, n = n0 + (l & 31);
        float v[1] = {acc[i]};
        if (m < q.M && n < q.N) tdc_mx4_finish<T, 1>(q, v, m, n);
    }
}

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

hipError_t tdc_launch_mx4_product(const TdcMx4Product &given, int dtype, hipStream_t s)
{
    TdcMx4Product q = given;
    q.vec = tdc_mx4_vec(q, dtype);
    if (q.M <= 64) return tdc_launch_mx4_rows(q, TdcMx4Source{nullptr, 0, 0}, dtype, nullptr, nullptr, s);
    const int64_t large = up(q.M, 256) * up(q.N, 256), small = up(q.M, 128) * up(q.N, 128), tiles = up(q.M, 32) * up(q.N, 32);
    const bool packed = q.nb % 16 == 0 && tdc_aligned_to(q.a_scales, 16) && tdc_aligned_to(q.b_scales, 16);
    TDC_FOR_DTYPE(dtype, T, {
        if (large >= 128) {
            if (packed) tdc_mx4_product_tile<T, 4, 2, 2, 4, true><<<(unsigned)large, 512, 0, s>>>(q);
            else tdc_mx4_product_tile<T, 4, 2, 2, 4, false><<<(unsigned)large, 512, 0, s>>>(q);
        } else if (small >= 64) {
            if (packed) tdc_mx4_product_tile<T, 2, 2, 2, 2, true><<<(unsigned)small, 256, 0, s>>>(q);
            else tdc_mx4_product_tile<T, 2, 2, 2, 2, false><<<(unsigned)small, 256, 0, s>>>(q);
        }
        else tdc_mx4_product_simple<T><<<(unsigned)((tiles + 3) / 4), 256, 0, s>>>(q);
    });
    return hipGetLastError();
}
