// Products of operands in microscaled 4-bit floating point on the matrix cores (tdc_mx4.h).
//
// v_mfma_scale_f32_32x32x64: lane l holds the 32 values of row l%32 that one block of k holds (block l/32 of the two), 16
// bytes, with the block's scale beside it, so an operand in the format's own layout needs no rearrangement.  Of the result,
// register i of lane l is element [m = 8*(i/4) + 4*(l/32) + i%4][n = l%32] with rows of A as m and rows of B as n.
#include "tdc_mx4_internal.h"

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ tdc_i8 widen(tdc_i4 a) { return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1); }

__device__ __forceinline__ f16v mfma(tdc_i4 a, unsigned sa, tdc_i4 b, unsigned sb, f16v c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(a), widen(b), c, 4, 4, 0, (int)sa, 0, (int)sb);
}

template <typename T> __device__ __forceinline__ void finish(const TdcMx4Product &q, float v, int m, int n)
{
    const size_t at = (size_t)m * q.N + n;
    if (q.epi.bias) v += q.epi.bias[n];
    if (q.epi.residual) v += (float)static_cast<const T *>(q.epi.residual)[at];
    if (q.epi.act == TDC_ACT_RELU) v = tdc_activate<TDC_ACT_RELU>(v);
    else if (q.epi.act == TDC_ACT_SILU) v = tdc_activate<TDC_ACT_SILU>(v);
    static_cast<T *>(q.y)[at] = (T)v;
}

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
    f16v acc;
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
        acc = mfma(a, sa, b, sb, acc);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int m = m0 + 8 * (i / 4) + 4 * (l >> 5) + i % 4, n = n0 + (l & 31);
        if (m < q.M && n < q.N) finish<T>(q, acc[i], m, n);
    }
}

}  // namespace

hipError_t tdc_launch_mx4_product(const TdcMx4Product &q, int dtype, hipStream_t s)
{
    const int64_t tiles = (int64_t)((q.M + 31) / 32) * ((q.N + 31) / 32);
    TDC_FOR_DTYPE(dtype, T, { tdc_mx4_product_simple<T><<<(unsigned)((tiles + 3) / 4), 256, 0, s>>>(q); });
    return hipGetLastError();
}
