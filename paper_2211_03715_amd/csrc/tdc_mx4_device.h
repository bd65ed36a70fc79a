// Device side of the 4-bit format (tdc_mx4.h): one block's scale, and its codes.
#ifndef TDC_MX4_DEVICE_H
#define TDC_MX4_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tdc_mx4.h"

constexpr int TDC_MX4_BLOCK = 32;       // values to a scale
constexpr int TDC_MX4_BLOCK_BYTES = 16; // their codes

typedef int tdc_i4 __attribute__((ext_vector_type(4)));
typedef int tdc_i8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ unsigned tdc_abs_bits(float v) { return __builtin_bit_cast(unsigned, v) & 0x7fffffffu; }

// The block's scale byte from the largest of its values' abs_bits: the exponent field of amax less 2, which makes amax 4 to 8
// in units of the scale; 255 where an infinity or a NaN (all larger than any number's bits) is among them.
__device__ __forceinline__ unsigned tdc_mx4_scale(unsigned top)
{
    const unsigned field = top >> 23;
    return field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
}

// Eight values (four below), in units of 2^(e - 127), as eight codes.  The conversion takes its scale from the exponent field of a float, 0
// for 2^-127, rounds to nearest even and saturates: checked for every e at every border between codes and its neighbours.
__device__ __forceinline__ unsigned tdc_mx4_codes8(const float *v, unsigned e)
{
    const float scale = __builtin_bit_cast(float, e << 23);
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return e == 255u ? 0u : c;
}

__device__ __forceinline__ unsigned tdc_mx4_codes4(const float *v, unsigned e)
{
    const float scale = __builtin_bit_cast(float, e << 23);
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    return e == 255u ? 0u : c;
}

// A whole block held by one thread.
__device__ __forceinline__ tdc_i4 tdc_mx4_block(const float (&v)[32], unsigned &e)
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, tdc_abs_bits(v[i]));
    e = tdc_mx4_scale(top);
    return (tdc_i4){(int)tdc_mx4_codes8(v, e), (int)tdc_mx4_codes8(v + 8, e), (int)tdc_mx4_codes8(v + 16, e), (int)tdc_mx4_codes8(v + 24, e)};
}

// V codes as values.  e = 255: all NaN.
template <int V> __device__ __forceinline__ void tdc_mx4_values(unsigned c, unsigned e, float (&v)[V])
{
    // 2^(e - 127) in two factors, so that e = 0 and values below the normal range come out exactly
    const int up = (int)e - 127, half = up / 2;
    const float s1 = __builtin_bit_cast(float, (unsigned)(127 + half) << 23), s2 = __builtin_bit_cast(float, (unsigned)(127 + up - half) << 23);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const unsigned m = (c >> (4 * i)) & 7u, sign = (c >> (4 * i + 3)) & 1u;
        // magnitude code m: 0, 1/2, then (1 + (m & 1)/2) 2^((m >> 1) - 1)
        const float mag = m < 2u ? 0.5f * m : __builtin_bit_cast(float, ((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
        const float r = mag * s1 * s2;
        v[i] = e == 255u ? __builtin_nanf("") : (sign ? -r : r);
    }
}

#endif  // TDC_MX4_DEVICE_H
