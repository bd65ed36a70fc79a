// What the forward and backward kernels of the group norm share.
//
// An image is cut into `chunks` runs of `chunk_px` pixels.  A first kernel reduces every chunk by itself and leaves one pair
// per chunk and group (backward: per chunk and channel) in the plan's workspace; the next one combines an image's pairs, in a
// fixed order, and runs over the same pixels again, which by then come from the caches for all but the largest tensors.
//
// Threads of a workgroup run over V neighbouring channels of a pixel each: nv = C / V threads to a pixel and rows = 256 / nv
// pixels at a time, or, where a pixel has more than 256 such pieces, one pixel at a time in several sweeps.  V is the most
// that divides C and the pitches and that the pointers are aligned to, up to 16 bytes.
#ifndef TDC_NORM_INTERNAL_H
#define TDC_NORM_INTERNAL_H

#include "tdc_typed.h"

constexpr int TDC_NORM_THREADS = 256;
constexpr int TDC_NORM_MAX_C = 8192;   // per-channel pairs of a workgroup fill at most 64 KiB of LDS

struct TdcNormDims {
    int B, P, C, G, Cg;     // P pixels to an image, Cg channels to a group
    int chunk_px, chunks;
    float eps;
};

struct tdc_norm_plan {
    tdc_norm_shape shape;
    TdcNormDims dims;
    int device;
    float2 *partial;     // [B][chunks][G]: mean and sum of squares about it; backward: [B][chunks][C]
    float2 *means;       // [B][G]: backward, m(g) and m(g xhat)
    size_t ws_bytes;
};

// Pixels of chunk i of an image.
__host__ __device__ inline int tdc_chunk_len(const TdcNormDims &d, int i)
{
    const int left = d.P - i * d.chunk_px;
    return left < d.chunk_px ? left : d.chunk_px;
}

// Lanes that share a group when a workgroup combines things per group: a power of two.
__host__ __device__ inline int tdc_team(int groups, int terms)
{
    int l = 1;
    while (2 * l <= 64 && 2 * l * groups <= TDC_NORM_THREADS && 2 * l <= terms) l *= 2;
    return l;
}

// Mean and variance of every group of image b from its chunks' pairs, as {mean, rstd} into `stats` [G] in LDS.  Two sums, the
// second about the mean of the first: nothing cancels, whatever the mean is.  Every thread of the workgroup calls it.
__device__ __forceinline__ void tdc_combine_chunks(const TdcNormDims &d, const float2 *partial, int b, float2 *stats)
{
    const int L = tdc_team(d.G, d.chunks), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = TDC_NORM_THREADS / L;
    const float n = (float)d.P * d.Cg, inv = 1.f / n;
    for (int g0 = 0; g0 < d.G; g0 += teams) {          // the same trip count for every lane: lane sums need all of a team
        const int g = min(g0 + team, d.G - 1);
        const float2 *p = partial + (size_t)b * d.chunks * d.G + g;
        float s = 0.f;
        for (int i = lane; i < d.chunks; i += L) s += p[(size_t)i * d.G].x * ((float)tdc_chunk_len(d, i) * d.Cg);
        const float mean = tdc_lane_sum(s, L) * inv;
        float m2 = 0.f;
        for (int i = lane; i < d.chunks; i += L) {
            const float2 v = p[(size_t)i * d.G];
            const float off = v.x - mean;
            m2 += v.y + off * off * ((float)tdc_chunk_len(d, i) * d.Cg);
        }
        m2 = tdc_lane_sum(m2, L);
        if (lane == 0 && g0 + team < d.G) stats[g] = make_float2(mean, 1.f / sqrtf(m2 * inv + d.eps));
    }
    __syncthreads();
}

// The most neighbours that one access may take: V elements, at most 16 bytes, a power of two.
inline int tdc_norm_vec(int dtype, int C, std::initializer_list<int64_t> pitches, std::initializer_list<const void *> ptrs)
{
    const int size = tdc_dtype_bytes(dtype);
    for (int v = 16 / size; v > 1; v /= 2) {
        bool ok = C % v == 0;
        for (int64_t p : pitches) ok = ok && p % v == 0;
        for (const void *p : ptrs) ok = ok && tdc_aligned_to(p, (size_t)v * size);
        if (ok) return v;
    }
    return 1;
}

#endif  // TDC_NORM_INTERNAL_H
