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

#include "tdc_norm_choice.h"
#include "tdc_typed.h"

constexpr int TDC_NORM_UNROLL = 4;       // pixels that a thread has in flight

struct tdc_norm_plan {
    tdc_norm_shape shape;
    TdcNormDims dims;
    int device;
    float4 *partial;     // [B][chunks][G]: number of values, their mean, sum of squares about it; backward: sums of g and g xhat
    float4 *whole;       // [B][G]: the same of an image
    float2 *sums;        // [tdc_norm_sum_rows][C]: backward, sums of d and d xhat over some images or chunks
    size_t ws_bytes;
};

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
// From there on it has I items: its piece as a whole where the channels are of one group (WHOLE), or every channel by itself.
template <int V, bool WHOLE> struct TdcNormSums {
    static constexpr int I = WHOLE ? 1 : V;
    float n, mean[V], m2[V];
    __device__ __forceinline__ TdcNormSums()
    {
        n = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) mean[v] = m2[v] = 0.f;
    }
    // pixel i of `in` counts where i < k; FULL: all of them do
    template <bool FULL, typename T, int U> __device__ __forceinline__ void add_some(const TdcVec<T, V> (&in)[U], int k)
    {
        const float inv_k = FULL ? 1.f / U : 1.f / k, tot = n + k, w = k * __builtin_amdgcn_rcpf(tot);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) s += FULL || u < k ? (float)in[u].v[v] : 0.f;
            s *= inv_k;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float off = FULL || u < k ? (float)in[u].v[v] - s : 0.f;
                q += off * off;
            }
            const float off = s - mean[v];
            mean[v] += off * w;
            m2[v] += q + off * off * (n * w);
        }
        n = tot;
    }
    template <typename T, int U> __device__ __forceinline__ void add(const TdcVec<T, V> (&in)[U], int k)
    {
        if (k == U) add_some<true>(in, U);
        else add_some<false>(in, k);
    }
};

// Items in LDS: `rows` rows of nv pieces, with the values that an item of the row stands for.  Where nv is a power of two below
// 64, a row is what a wavefront's lanes of the same piece have together, else what a pixel row of threads has.
struct TdcNormItems {
    float2 *item;
    float *count;
};

__device__ __forceinline__ bool tdc_norm_by_wave(int nv) { return nv < 64 && (nv & (nv - 1)) == 0; }

// Every thread of the workgroup calls this, `live` ones with the sums of piece cv, the others with none (n = 0); or those with
// one, where nv >= 64.  Returns the number of rows.  The caller synchronises.
template <int V, bool WHOLE, int THREADS>
__device__ __forceinline__ int tdc_norm_put(const TdcNormItems &to, TdcNormSums<V, WHOLE> &s, const TdcNormLanes &t, int cv, int nv, bool live, int used)
{
    constexpr int I = TdcNormSums<V, WHOLE>::I;
    if (WHOLE) {
        float m = 0.f, q = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) m += s.mean[v];
        m *= 1.f / V;
#pragma unroll
        for (int v = 0; v < V; ++v) q += s.m2[v] + (s.mean[v] - m) * (s.mean[v] - m) * s.n;
        s.mean[0] = m;
        s.m2[0] = q;
        s.n *= V;
    }
    int row = t.r, rows = used;
    bool writes = live;
    if (tdc_norm_by_wave(nv)) {
        // first the mean of the lanes that belong together, then the squares about that: plain sums both
        const float n = s.n;
        float sum[I], m2[I];
#pragma unroll
        for (int i = 0; i < I; ++i) sum[i] = n * s.mean[i];
        tdc_merge_lanes(nv, [&](auto first, auto second) {
            s.n = first(s.n) + second(s.n);
#pragma unroll
            for (int i = 0; i < I; ++i) sum[i] = first(sum[i]) + second(sum[i]);
        });
        const float inv = s.n > 0.f ? 1.f / s.n : 0.f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const float mean = sum[i] * inv, off = s.mean[i] - mean;
            m2[i] = s.m2[i] + n * off * off;
            s.mean[i] = mean;
        }
        tdc_merge_lanes(nv, [&](auto first, auto second) {
#pragma unroll
            for (int i = 0; i < I; ++i) m2[i] = first(m2[i]) + second(m2[i]);
        });
#pragma unroll
        for (int i = 0; i < I; ++i) s.m2[i] = m2[i];
        row = threadIdx.x / 64;
        rows = THREADS / 64;
        writes = (threadIdx.x & 63) < nv;
    }
    if (writes) {
#pragma unroll
        for (int i = 0; i < I; ++i) to.item[(row * nv + cv) * I + i] = make_float2(s.mean[i], s.m2[i]);
        if (cv == 0) to.count[row] = s.n;
    }
    return rows;
}

// How a team of L lanes lies over `rows` x `per_group` items: powers of two, so that no index needs a division.
struct TdcNormTeam {
    int L, lane, team, teams, k0, kstep, r0, rstep;
    __device__ __forceinline__ TdcNormTeam(int groups, int rows, int per_group, int threads)
    {
        L = tdc_team(groups, rows * per_group, threads);
        lane = threadIdx.x & (L - 1);
        team = threadIdx.x / L;
        teams = threads / L;
        kstep = 1;
        while (kstep < per_group && kstep < L) kstep *= 2;
        k0 = lane & (kstep - 1);
        rstep = L / kstep;
        r0 = lane / kstep;
    }
};

// The items combined group by group, a team of lanes to a group: f(g, values, mean, squares about it) in one lane of it.
template <int THREADS, typename F> __device__ __forceinline__ void tdc_norm_groups(const TdcNormItems &from, int rows, int groups, int per_group, F f)
{
    const TdcNormTeam t(groups, rows, per_group, THREADS);
    const int pitch = groups * per_group;
    for (int g0 = 0; g0 < groups; g0 += t.teams) {     // the same trip count for every lane: lane sums need all of a team
        const int g = min(g0 + t.team, groups - 1);
        float n = 0.f, s = 0.f;
        for (int r = t.r0; r < rows; r += t.rstep) {
            const float c = from.count[r];
            if (c > 0.f)
                for (int k = t.k0; k < per_group; k += t.kstep) {
                    n += c;
                    s += c * from.item[r * pitch + g * per_group + k].x;
                }
        }
        n = tdc_lane_sum(n, t.L);
        const float mean = tdc_lane_sum(s, t.L) / n;
        float m2 = 0.f;
        for (int r = t.r0; r < rows; r += t.rstep) {
            const float c = from.count[r];
            if (c > 0.f)
                for (int k = t.k0; k < per_group; k += t.kstep) {
                    const float2 o = from.item[r * pitch + g * per_group + k];
                    m2 += o.y + (o.x - mean) * (o.x - mean) * c;
                }
        }
        m2 = tdc_lane_sum(m2, t.L);
        if (t.lane == 0 && g0 + t.team < groups) f(g, n, mean, m2);
    }
}

// Group of each of V neighbouring channels from c0 on, f(v, group): one division, whatever V is.
template <int V, typename F> __device__ __forceinline__ void tdc_norm_channels(int c0, int Cg, F f)
{
    int g = c0 / Cg, rest = c0 - g * Cg;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        f(v, g);
        if (++rest == Cg) {
            rest = 0;
            ++g;
        }
    }
}

__device__ __forceinline__ float tdc_rstd(float var, float eps) { return 1.f / sqrtf(var + eps); }

// The same for items that are plain sums: [rows][groups * per_group].
template <typename F> __device__ __forceinline__ void tdc_norm_group_sums(const float2 *items, int rows, int groups, int per_group, int threads, F f)
{
    const TdcNormTeam t(groups, rows, per_group, threads);
    const int pitch = groups * per_group;
    for (int g0 = 0; g0 < groups; g0 += t.teams) {
        const int g = min(g0 + t.team, groups - 1);
        float s1 = 0.f, s2 = 0.f;
        for (int r = t.r0; r < rows; r += t.rstep)
            for (int k = t.k0; k < per_group; k += t.kstep) {
                const float2 o = items[r * pitch + g * per_group + k];
                s1 += o.x;
                s2 += o.y;
            }
        s1 = tdc_lane_sum(s1, t.L);
        s2 = tdc_lane_sum(s2, t.L);
        if (t.lane == 0 && g0 + t.team < groups) f(g, s1, s2);
    }
}

// Plain sums of I items to a thread into LDS, lanes of a wavefront with the same piece together where tdc_norm_by_wave says so.
// Returns the number of rows.  The caller synchronises.
template <int I, int THREADS> __device__ __forceinline__ int tdc_norm_put_sums(float2 *items, float (&s1)[I], float (&s2)[I], const TdcNormLanes &t, int cv, int nv, bool live, int used)
{
    int row = t.r, rows = used;
    bool writes = live;
    if (tdc_norm_by_wave(nv)) {
        tdc_merge_lanes(nv, [&](auto first, auto second) {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                s1[i] = first(s1[i]) + second(s1[i]);
                s2[i] = first(s2[i]) + second(s2[i]);
            }
        });
        row = threadIdx.x / 64;
        rows = THREADS / 64;
        writes = (threadIdx.x & 63) < nv;
    }
    if (writes) {
#pragma unroll
        for (int i = 0; i < I; ++i) items[(row * nv + cv) * I + i] = make_float2(s1[i], s2[i]);
    }
    return rows;
}

// `parts` sums of image b combined group by group: f(g, values, mean, squares about it) in one lane of a group's team.
template <typename F> __device__ __forceinline__ void tdc_combine(const TdcNormDims &d, const float4 *partial, int parts, int b, int threads, F f)
{
    const int L = tdc_team(d.G, parts, threads), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = threads / L;
    for (int g0 = 0; g0 < d.G; g0 += teams) {
        const int g = min(g0 + team, d.G - 1);
        const float4 *p = partial + (size_t)b * parts * d.G + g;
        float n = 0.f, s = 0.f;
#pragma unroll 4
        for (int i = lane; i < parts; i += L) {
            const float4 o = p[(size_t)i * d.G];
            n += o.x;
            s += o.x * o.y;
        }
        n = tdc_lane_sum(n, L);
        const float mean = tdc_lane_sum(s, L) / n;
        float m2 = 0.f;
#pragma unroll 4
        for (int i = lane; i < parts; i += L) {
            const float4 o = p[(size_t)i * d.G];
            m2 += o.z + o.x * (o.y - mean) * (o.y - mean);
        }
        m2 = tdc_lane_sum(m2, L);
        if (lane == 0 && g0 + team < d.G) f(g, n, mean, m2);
    }
}

// The same for plain sums: f(g, first sum, second sum).
template <typename F> __device__ __forceinline__ void tdc_combine_sums(const TdcNormDims &d, const float2 *partial, int parts, int b, int threads, F f)
{
    const int L = tdc_team(d.G, parts, threads), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = threads / L;
    for (int g0 = 0; g0 < d.G; g0 += teams) {
        const int g = min(g0 + team, d.G - 1);
        const float2 *p = partial + (size_t)b * parts * d.G + g;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll 4
        for (int i = lane; i < parts; i += L) {
            const float2 o = p[(size_t)i * d.G];
            s1 += o.x;
            s2 += o.y;
        }
        s1 = tdc_lane_sum(s1, L);
        s2 = tdc_lane_sum(s2, L);
        if (lane == 0 && g0 + team < d.G) f(g, s1, s2);
    }
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

// A launch of `fn` with dynamic LDS, which has to be allowed before a first one where it is much: up to 64 KiB for C near 8192.
template <typename... P, typename... A> hipError_t tdc_norm_launch(void (*fn)(P...), dim3 grid, size_t lds, hipStream_t s, A... args)
{
    const hipError_t e = tdc_allow_lds((const void *)fn, lds);
    if (e == hipSuccess) fn<<<grid, TDC_NORM_THREADS, lds, s>>>(args...);
    return e;
}

// Workgroup id -> (image, slice): the ids that one XCD gets, 8 apart, are neighbours.
__device__ __forceinline__ void tdc_norm_place(int id, int total, int slices, int &b, int &slice)
{
    const int per = total / 8, extra = total % 8, xcd = id % 8;
    const int t = xcd * per + (xcd < extra ? xcd : extra) + id / 8;
    b = t / slices;
    slice = t - b * slices;
}

// The statements with the constants THREADS and HELD that a slice asks for; MOST is what tdc_norm_held says, FORWARD what it was
// told.
#define TDC_FOR_SLICE(s, MOST, FORWARD, THREADS, HELD, ...)                                                                         \
    do {                                                                                                                            \
        if ((s).threads == 256) { constexpr int THREADS = 256, HELD = 4; __VA_ARGS__; }                                             \
        else if ((s).threads == 1024) { if constexpr (FORWARD) { constexpr int THREADS = 1024, HELD = MOST; __VA_ARGS__; } }        \
        else if ((s).held <= 4) { constexpr int THREADS = 512, HELD = 4; __VA_ARGS__; }                                             \
        else if ((s).held <= 8) { constexpr int THREADS = 512, HELD = 8; __VA_ARGS__; }                                             \
        else if constexpr ((MOST) >= 16) { constexpr int THREADS = 512, HELD = 16; __VA_ARGS__; }                                   \
    } while (0)

#endif  // TDC_NORM_INTERNAL_H
