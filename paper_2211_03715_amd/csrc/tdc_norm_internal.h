// What the forward and backward kernels of the group norm share.
//
// Two ways to the result.  Where an image's share of some whole groups fits the registers of one workgroup, the workgroup keeps
// it there: one launch, x read once ("resident").  Otherwise an image is cut into chunks of pixels: a first kernel reduces every
// chunk by itself and leaves its sums in the plan's workspace, the next one combines an image's sums, in a fixed order, and runs
// over the same pixels again, which by then come from the caches for all but the largest tensors.
//
// Threads of a workgroup run over V neighbouring channels of a pixel each: nv threads to a pixel and rows = THREADS / nv pixels
// at a time, or, where a pixel has more than THREADS such pieces, one pixel at a time in several sweeps.  V is the most that
// divides C and the pitches and that the pointers are aligned to, up to 16 bytes.
#ifndef TDC_NORM_INTERNAL_H
#define TDC_NORM_INTERNAL_H

#include <algorithm>
#include <initializer_list>

#include "tdc_typed.h"

constexpr int TDC_NORM_THREADS = 1024;   // of the kernels that run over chunks
constexpr int TDC_NORM_MAX_C = 8192;     // per-channel pairs of a workgroup fill at most 64 KiB of LDS
constexpr int TDC_NORM_UNROLL = 4;       // pixels that a thread has in flight

struct TdcNormDims {
    int B, P, C, G, Cg;     // P pixels to an image, Cg channels to a group
    int chunk_px, chunks;
    float eps;
};

struct tdc_norm_plan {
    tdc_norm_shape shape;
    TdcNormDims dims;
    int device;
    float4 *partial;     // [B][chunks][G]: number of values, their mean, sum of squares about it; backward: sums of g and g xhat
    float2 *sums;        // [min(B chunks, TDC_NORM_SUM_ROWS)][C]: backward, sums of d and d xhat over some images or chunks
    size_t ws_bytes;
};

// Workgroups to a channel in the backward pass, at most: as many rows of sums are left to add up for dgamma and dbeta.
constexpr int TDC_NORM_SUM_ROWS = 512;

// Pixels of chunk i of an image.
__host__ __device__ inline int tdc_chunk_len(const TdcNormDims &d, int i)
{
    const int left = d.P - i * d.chunk_px;
    return left < d.chunk_px ? left : d.chunk_px;
}

// How a workgroup's threads lie over `nv` pieces of a pixel.
struct TdcNormLanes {
    int rows, r, cv;     // pixels at a time; this thread's (>= rows: none) and its first piece
    __device__ __forceinline__ TdcNormLanes(int nv, int threads)
    {
        rows = nv < threads ? threads / nv : 1;
        r = rows == 1 ? 0 : threadIdx.x / nv;
        cv = threadIdx.x - r * nv;
    }
};

// Lanes that share a group when `threads` threads combine things for `groups` groups: a power of two up to a wavefront.
__host__ __device__ inline int tdc_team(int groups, int terms, int threads)
{
    int l = 1;
    while (2 * l <= 64 && 2 * l * groups <= threads && l < terms) l *= 2;
    return l;
}

// ---- statistics
//
// A thread takes its V channels of several pixels at a time into registers, their mean and the squares about it, and merges that
// into what it has (n_a, mean_a, S_a with n_b, mean_b, S_b: mean = mean_a + d n_b / n, S = S_a + S_b + d^2 n_a n_b / n,
// d = mean_b - mean_a).  No sum of squares is ever taken about anything but a mean next to the values, so fp32 does.
template <int V> struct TdcNormSums {
    float n, mean[V], m2[V];
    __device__ __forceinline__ TdcNormSums()
    {
        n = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) mean[v] = m2[v] = 0.f;
    }
    // the first k of U pixels
    template <typename T, int U> __device__ __forceinline__ void add(const TdcVec<T, V> (&in)[U], int k)
    {
        const float inv_k = 1.f / k, tot = n + k, w = k / tot;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) s += u < k ? (float)in[u].v[v] : 0.f;
            s *= inv_k;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float off = u < k ? (float)in[u].v[v] - s : 0.f;
                q += off * off;
            }
            const float off = s - mean[v];
            mean[v] += off * w;
            m2[v] += q + off * off * (n * w);
        }
        n = tot;
    }
    // as an item to combine: the piece as a whole (WHOLE: its channels are of one group), or every channel by itself
    template <bool WHOLE> __device__ __forceinline__ void put(float2 *items, int row, int nv, int cv) const
    {
        if constexpr (WHOLE) {
            float m = 0.f, q = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) m += mean[v];
            m *= 1.f / V;
#pragma unroll
            for (int v = 0; v < V; ++v) q += m2[v] + (mean[v] - m) * (mean[v] - m) * n;
            items[row * nv + cv] = make_float2(m, q);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) items[(row * nv + cv) * V + v] = make_float2(mean[v], m2[v]);
        }
    }
};

// The items of a workgroup's `used` rows (row r over full + (r < rem) pixels) combined group by group, a team of lanes to a
// group: f(g, values, mean, squares about it) in one lane of it.  per_group items of `width` channels to a row and group.
template <typename F> __device__ __forceinline__ void tdc_norm_groups(const float2 *items, int used, int full, int rem, int groups, int per_group, int width, int threads, F f)
{
    const int L = tdc_team(groups, used * per_group, threads), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = threads / L;
    const int pitch = groups * per_group, terms = used * per_group;
    for (int g0 = 0; g0 < groups; g0 += teams) {       // the same trip count for every lane: lane sums need all of a team
        const int g = min(g0 + team, groups - 1);
        float n = 0.f, s = 0.f;
        for (int i = lane; i < terms; i += L) {
            const int row = i / per_group;
            const float k = (float)((full + (row < rem)) * width);
            n += k;
            s += k * items[row * pitch + g * per_group + i - row * per_group].x;
        }
        n = tdc_lane_sum(n, L);
        const float mean = tdc_lane_sum(s, L) / n;
        float m2 = 0.f;
        for (int i = lane; i < terms; i += L) {
            const int row = i / per_group;
            const float2 o = items[row * pitch + g * per_group + i - row * per_group];
            m2 += o.y + (o.x - mean) * (o.x - mean) * (float)((full + (row < rem)) * width);
        }
        m2 = tdc_lane_sum(m2, L);
        if (lane == 0 && g0 + team < groups) f(g, n, mean, m2);
    }
}

__device__ __forceinline__ float tdc_rstd(float var, float eps) { return 1.f / sqrtf(var + eps); }

// The same rows' items as plain sums.
template <typename F> __device__ __forceinline__ void tdc_norm_group_sums(const float2 *items, int used, int groups, int per_group, int threads, F f)
{
    const int L = tdc_team(groups, used * per_group, threads), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = threads / L;
    const int pitch = groups * per_group, terms = used * per_group;
    for (int g0 = 0; g0 < groups; g0 += teams) {
        const int g = min(g0 + team, groups - 1);
        float s1 = 0.f, s2 = 0.f;
        for (int i = lane; i < terms; i += L) {
            const int row = i / per_group;
            const float2 o = items[row * pitch + g * per_group + i - row * per_group];
            s1 += o.x;
            s2 += o.y;
        }
        s1 = tdc_lane_sum(s1, L);
        s2 = tdc_lane_sum(s2, L);
        if (lane == 0 && g0 + team < groups) f(g, s1, s2);
    }
}

// The chunks' sums of image b as {mean, rstd} of every group into `stats` [G] in LDS.  Every thread of the workgroup calls it.
__device__ __forceinline__ void tdc_combine_chunks(const TdcNormDims &d, const float4 *partial, int b, float2 *stats, int threads)
{
    const int L = tdc_team(d.G, d.chunks, threads), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = threads / L;
    for (int g0 = 0; g0 < d.G; g0 += teams) {
        const int g = min(g0 + team, d.G - 1);
        const float4 *p = partial + (size_t)b * d.chunks * d.G + g;
        float n = 0.f, s = 0.f;
        for (int i = lane; i < d.chunks; i += L) {
            const float4 o = p[(size_t)i * d.G];
            n += o.x;
            s += o.x * o.y;
        }
        n = tdc_lane_sum(n, L);
        const float mean = tdc_lane_sum(s, L) / n;
        float m2 = 0.f;
        for (int i = lane; i < d.chunks; i += L) {
            const float4 o = p[(size_t)i * d.G];
            m2 += o.z + o.x * (o.y - mean) * (o.y - mean);
        }
        m2 = tdc_lane_sum(m2, L);
        if (lane == 0 && g0 + team < d.G) stats[g] = make_float2(mean, tdc_rstd(m2 / n, d.eps));
    }
    __syncthreads();
}

// The most neighbours that one access may take: V elements, at most 16 bytes, a power of two.
inline int tdc_norm_vec(int dtype, int C, std::initializer_list<int64_t> pitches, std::initializer_list<const void *> ptrs, int most = 8)
{
    const int size = tdc_dtype_bytes(dtype);
    for (int v = std::min(16 / size, most); v > 1; v /= 2) {
        bool ok = C % v == 0;
        for (int64_t p : pitches) ok = ok && p % v == 0;
        for (const void *p : ptrs) ok = ok && tdc_aligned_to(p, (size_t)v * size);
        if (ok) return v;
    }
    return 1;
}

// ---- the resident form

// Pieces of x that a thread holds at most: 64 values of fp32, fewer where the conversions need the registers, and fewer still
// backward, where dy is held too.  Twice as many spill.
__host__ __device__ constexpr int tdc_norm_held(int V, int size, bool backward) { return backward ? 4 : (V >= 4 && size == 2 ? 8 : 16); }

// A workgroup takes `width` channels, whole groups and whole pieces, of an image; `slices` of them to an image.
struct TdcNormSlice {
    int width, slices, threads, held;    // held: pieces to a thread; 0: the image does not fit
};

// Slices are lines of 128 bytes where a workgroup's registers hold that much (two workgroups of 512 threads to a compute unit,
// or one of 1024), and else less, down to one group.  A line that two or four workgroups share comes from memory once all the
// same: they run on the same XCD (tdc_norm_place).
inline TdcNormSlice tdc_norm_slice(const TdcNormDims &d, int dtype, int V, bool backward, int multiple)
{
    int unit = d.Cg;
    while (unit % V || unit % multiple) {
        unit += d.Cg;
        if (unit >= d.C) break;
    }
    if (unit > d.C || d.C % unit) unit = d.C;
    auto fits = [&](int width, int threads) {
        const int nv = width / V;
        return nv <= threads && width / d.Cg <= threads ? (d.P + threads / nv - 1) / (threads / nv) : 1 << 30;
    };
    const int most = tdc_norm_held(V, tdc_dtype_bytes(dtype), backward);
    TdcNormSlice best{0, 0, 0, 0};
    for (int width = unit; width <= d.C; width += unit) {
        if (d.C % width) continue;
        const int line = width * tdc_dtype_bytes(dtype);
        if (best.held && line > 128) break;
        for (int threads : {256, 512, 1024}) {
            const int held = fits(width, threads);
            if (held > most) continue;
            if (held > 4 && threads < 1024) continue;   // rather more threads than more to each
            best = TdcNormSlice{width, d.C / width, threads, held};
            break;
        }
        if (best.width != width) break;                 // wider ones fit even less
        // few images: as many workgroups as can be, for the one wave of them that there is
        if ((int64_t)d.B * (d.C / width) <= 512) break;
    }
    return best;
}

// Workgroup id -> (image, slice): the ids that one XCD gets, 8 apart, are neighbours.
__device__ __forceinline__ void tdc_norm_place(int id, int total, int slices, int &b, int &slice)
{
    const int per = total / 8, extra = total % 8, xcd = id % 8;
    const int t = xcd * per + (xcd < extra ? xcd : extra) + id / 8;
    b = t / slices;
    slice = t - b * slices;
}

// The statements with the constants THREADS and HELD that a slice asks for; MOST is what tdc_norm_held says.
#define TDC_FOR_SLICE(s, MOST, THREADS, HELD, ...)                                                                                  \
    do {                                                                                                                            \
        if ((s).threads == 256) { constexpr int THREADS = 256, HELD = 4; __VA_ARGS__; }                                             \
        else if ((s).threads == 512) { constexpr int THREADS = 512, HELD = 4; __VA_ARGS__; }                                        \
        else if ((s).held <= 4) { constexpr int THREADS = 1024, HELD = 4; __VA_ARGS__; }                                            \
        else if ((s).held <= 8) { if constexpr ((MOST) >= 8) { constexpr int THREADS = 1024, HELD = 8; __VA_ARGS__; } }             \
        else if constexpr ((MOST) >= 16) { constexpr int THREADS = 1024, HELD = 16; __VA_ARGS__; }                                  \
    } while (0)

#endif  // TDC_NORM_INTERNAL_H
