// Group norm with an activation, channels last: plans, the forward kernels and their launches (tdc_norm.h).
#include <cmath>
#include <new>

#include "tdc_mx4_device.h"
#include "tdc_norm_internal.h"

namespace {

// Where a forward call's results go.
struct NormOut {
    void *y;                 // or null:
    uint8_t *codes, *scales;
    int64_t pitch;
    float *mean, *rstd;      // or null
    bool stream;             // how y is stored
};

struct NormIn {
    const void *x, *residual;
    const float *gamma, *beta;
    int64_t xp, rp;
    int act;                 // the same for every thread: a branch to V values costs next to nothing beside their way to memory
};

// Constants of a thread's V channels: their weights, which can be on their way while the statistics are made, then all of it.
template <int V> struct Affine {
    float mean[V], scale[V], shift[V];
    __device__ __forceinline__ void weights(const NormIn &in, int c0)
    {
        // one branch to all of them: behind a branch of its own each load would wait by itself
#pragma unroll
        for (int v = 0; v < V; ++v) scale[v] = 1.f, shift[v] = 0.f;
        if (in.gamma) {
#pragma unroll
            for (int v = 0; v < V; ++v) scale[v] = in.gamma[c0 + v];
        }
        if (in.beta) {
#pragma unroll
            for (int v = 0; v < V; ++v) shift[v] = in.beta[c0 + v];
        }
    }
    // stats: of the groups from g0 on
    __device__ __forceinline__ void statistics(const TdcNormDims &d, const float2 *stats, int g0, int c0)
    {
        tdc_norm_channels<V>(c0, d.Cg, [&](int v, int g) {
            const float2 st = stats[g - g0];
            mean[v] = st.x;
            scale[v] *= st.y;
        });
    }
};

template <typename T, int V>
__device__ __forceinline__ void apply(const Affine<V> &k, const TdcVec<T, V> &x, const TdcVec<T, V> &res, const NormIn &in, float (&o)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) o[v] = ((float)x.v[v] - k.mean[v]) * k.scale[v] + k.shift[v];
    if (in.residual) {
#pragma unroll
        for (int v = 0; v < V; ++v) o[v] += (float)res.v[v];
    }
    tdc_activate_all(in.act, o);
}

template <typename T, int V> __device__ __forceinline__ void store(const NormOut &out, T *p, const float (&o)[V])
{
    if (out.stream) tdc_store_stream<T, V>(p, o);
    else tdc_store<T, V>(p, o);
}

// V of a block's 32 channels to a lane, 32 / V neighbouring lanes to a block: all of them call this, `live` or not.
template <int V> __device__ __forceinline__ void store_mx4(const NormOut &out, const float (&o)[V], size_t px, int nb, int c0, bool live)
{
    unsigned top = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) top = max(top, tdc_abs_bits(o[v]));
    const unsigned e = tdc_mx4_scale(tdc_lane_max<32 / V>(top));
    if (!live) return;
    const size_t block = px * nb + c0 / 32;
    uint8_t *at = out.codes + block * 16 + (c0 % 32) / 2;
    if constexpr (V == 8) *reinterpret_cast<unsigned *>(at) = tdc_mx4_codes8(o, e);
    else *reinterpret_cast<uint16_t *>(at) = (uint16_t)tdc_mx4_codes4(o, e);
    if (c0 % 32 == 0) out.scales[block] = (uint8_t)e;
}

// ---- resident: a slice of an image's channels in the registers of a workgroup
template <typename T, int V, bool WHOLE, bool MX4, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS, 4) void tdc_norm_resident(TdcNormDims d, NormIn in, NormOut out, int width, int slices, int held_here)
{
    __shared__ float2 item[THREADS * (WHOLE ? 1 : V)], stats[THREADS];
    __shared__ float count[THREADS];
    const TdcNormItems items{item, count};
    int b, slice;
    tdc_norm_place(blockIdx.x, gridDim.x, slices, b, slice);
    const int nv = width / V, groups = width / d.Cg, c0 = slice * width;
    const TdcNormLanes t(nv, THREADS);
    const bool live = t.r < min(t.rows, d.P) && t.cv < nv;
    const T *x = static_cast<const T *>(in.x) + (size_t)b * d.P * in.xp + c0 + t.cv * V;
    TdcRaw<T, V> held[HELD];
    TdcNormSums<V, WHOLE> sums;
    if (live) {
        // held_here is the same for all threads: what lies behind it is skipped without a load
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < held_here) held[i].load(x + (size_t)min(t.r + i * t.rows, d.P - 1) * in.xp);
        TdcVec<T, V> v[HELD];
#pragma unroll
        for (int i = 0; i < HELD; ++i) v[i] = held[i].open();
        sums.add(v, (d.P - t.r + t.rows - 1) / t.rows);
    }
    const int rows = tdc_norm_put<V, WHOLE, THREADS>(items, sums, t, t.cv, nv, live, min(t.rows, d.P));
    __syncthreads();
    const size_t at = (size_t)b * d.G + c0 / d.Cg;
    tdc_norm_groups<THREADS>(items, rows, groups, WHOLE ? d.Cg / V : d.Cg, [&](int g, float n, float mean, float m2) {
        const float rstd = tdc_rstd(m2 / n, d.eps);
        stats[g] = make_float2(mean, rstd);
        if (out.mean) out.mean[at + g] = mean;
        if (out.rstd) out.rstd[at + g] = rstd;
    });
    Affine<V> a;
    a.weights(in, c0 + (live ? t.cv * V : 0));
    __syncthreads();
    if (!live && !MX4) return;
    a.statistics(d, stats, c0 / d.Cg, c0 + (live ? t.cv * V : 0));
    const T *res = in.residual ? static_cast<const T *>(in.residual) + (size_t)b * d.P * in.rp + c0 + t.cv * V : nullptr;
    // MX4: lanes that share a block have the same pixels, but their neighbours in the wavefront may have one less.  The residual
    // comes R pixels at a time, one such step ahead of the stores: behind a store, which might change it for all the compiler
    // knows, each of its loads would wait by itself.  Pieces of 8 leave no registers for that.
    constexpr int R = V == 8 ? 1 : HELD < 4 ? HELD : 4, AHEAD = V == 8 ? 0 : R;
    TdcRaw<T, V> rv[V == 8 ? 1 : 2][R];
    auto fetch = [&](int i0, TdcRaw<T, V> (&to)[R]) {
        if (!res || i0 >= held_here) return;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int p = tdc_anew(t.r + (i0 + i) * t.rows);
            if (live && p < d.P) to[i].load(res + (size_t)p * in.rp);
        }
    };
    if (AHEAD) fetch(0, rv[0]);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int p = tdc_anew(t.r + i * t.rows);
        const bool mine = live && p < d.P;
        if (MX4 ? i >= held_here : !mine) break;
        if (i % R == 0 && i + AHEAD < HELD) fetch(i + AHEAD, rv[AHEAD ? i / R + 1 & 1 : 0]);
        float o[V];
        apply(a, held[i].open(), rv[AHEAD ? i / R & 1 : 0][i % R].open(), in, o);
        const size_t px = (size_t)b * d.P + p;
        if constexpr (MX4) store_mx4<V>(out, o, px, (d.C + 31) / 32, c0 + t.cv * V, mine);
        else store(out, static_cast<T *>(out.y) + px * out.pitch + c0 + t.cv * V, o);
    }
}

// ---- statistics of a chunk: grid (chunks, batch)
template <typename T, int V, bool WHOLE>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_stats(TdcNormDims d, NormIn in, float4 *__restrict__ partial)
{
    constexpr int U = TDC_NORM_UNROLL;
    extern __shared__ float2 item[];
    __shared__ float count[TDC_NORM_THREADS];
    const TdcNormItems items{item, count};
    const int nv = d.C / V, b = blockIdx.y, chunk = blockIdx.x, len = tdc_chunk_len(d, chunk);
    const TdcNormLanes t(nv, TDC_NORM_THREADS);
    const T *base = static_cast<const T *>(in.x) + ((size_t)b * d.P + (size_t)chunk * d.chunk_px) * in.xp;
    const int used = min(t.rows, len);
    int rows = 1;
    for (int cv = t.cv; cv < nv || cv == t.cv; cv += TDC_NORM_THREADS) {   // once, but for pixels of more pieces than there are threads
        const bool live = t.r < used && cv < nv;
        TdcNormSums<V, WHOLE> sums;
        if (live)
            for (int p = t.r; p < len; p += t.rows * U) {
                TdcVec<T, V> v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = tdc_load<T, V>(base + (size_t)min(p + u * t.rows, len - 1) * in.xp + cv * V);
                sums.add(v, min(U, (len - p + t.rows - 1) / t.rows));
            }
        rows = tdc_norm_put<V, WHOLE, TDC_NORM_THREADS>(items, sums, t, cv, nv, live, used);
        if (t.rows > 1) break;
    }
    __syncthreads();
    float4 *out = partial + ((size_t)b * d.chunks + chunk) * d.G;
    tdc_norm_groups<TDC_NORM_THREADS>(items, rows, d.G, WHOLE ? d.Cg / V : d.Cg, [&](int g, float n, float mean, float m2) { out[g] = make_float4(n, mean, m2, 0.f); });
}

// ---- an image's chunks in one: a wavefront to a group, grid (groups, batch)
__global__ __launch_bounds__(64) void tdc_norm_combine(TdcNormDims d, const float4 *__restrict__ partial, float4 *__restrict__ whole)
{
    const size_t b = blockIdx.y, g = blockIdx.x;
    const float4 *p = partial + b * d.chunks * d.G + g;
    float n = 0.f, s = 0.f, m2 = 0.f;
#pragma unroll 8
    for (int i = threadIdx.x; i < d.chunks; i += 64) {
        const float4 o = p[(size_t)i * d.G];
        n += o.x;
        s += o.x * o.y;
    }
    n = tdc_lane_sum(n, 64);
    const float mean = tdc_lane_sum(s, 64) / n;
#pragma unroll 8
    for (int i = threadIdx.x; i < d.chunks; i += 64) {
        const float4 o = p[(size_t)i * d.G];
        m2 += o.z + o.x * (o.y - mean) * (o.y - mean);
    }
    m2 = tdc_lane_sum(m2, 64);
    if (threadIdx.x == 0) whole[b * d.G + g] = make_float4(n, mean, m2, 0.f);
}

// {mean, rstd} of every group of image b into `stats` [G] in LDS; the workgroup of the first chunk writes them out.
__device__ __forceinline__ void statistics(const TdcNormDims &d, const NormOut &out, const float4 *partial, int parts, int b, int chunk, float2 *stats)
{
    tdc_combine(d, partial, parts, b, TDC_NORM_THREADS, [&](int g, float n, float mean, float m2) {
        const float rstd = tdc_rstd(m2 / n, d.eps);
        stats[g] = make_float2(mean, rstd);
        if (chunk) return;
        if (out.mean) out.mean[(size_t)b * d.G + g] = mean;
        if (out.rstd) out.rstd[(size_t)b * d.G + g] = rstd;
    });
    __syncthreads();
}

// ---- y = act((x - mean) * (rstd gamma) + beta + residual): grid (chunks, batch)
template <typename T, int V, bool MX4>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_apply(TdcNormDims d, NormIn in, NormOut out, const float4 *__restrict__ partial, int parts)
{
    constexpr int U = 2;
    extern __shared__ float2 stats[];                      // [G]
    const int nv = d.C / V, b = blockIdx.y, chunk = blockIdx.x, len = tdc_chunk_len(d, chunk);
    const TdcNormLanes t(nv, TDC_NORM_THREADS);
    const size_t first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    const T *x = static_cast<const T *>(in.x) + first * in.xp, *res = in.residual ? static_cast<const T *>(in.residual) + first * in.rp : nullptr;
    TdcRaw<T, V> v[U], rv[U];
    auto fetch = [&](int cv, int p0) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(x + (size_t)min(p0 + u * t.rows, len - 1) * in.xp + cv * V);
        if (res) {
#pragma unroll
            for (int u = 0; u < U; ++u) rv[u].load(res + (size_t)min(p0 + u * t.rows, len - 1) * in.rp + cv * V);
        }
    };
    // the first pixels and the weights are on their way while the statistics are put together
    Affine<V> a;
    if (t.r < t.rows && t.cv < nv) {
        fetch(t.cv, t.r);
        a.weights(in, t.cv * V);
    }
    statistics(d, out, partial, parts, b, chunk, stats);
    // MX4: the lanes of a block go through the loops together (nv is a multiple of 32 / V)
    if (t.r >= t.rows) return;
    for (int cv = t.cv; cv < nv; cv += TDC_NORM_THREADS) {
        if (cv != t.cv) {
            fetch(cv, t.r);
            a.weights(in, cv * V);
        }
        a.statistics(d, stats, 0, cv * V);
        for (int p0 = t.r; p0 < len; p0 += t.rows * U) {
            float o[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) apply(a, v[u].open(), rv[u].open(), in, o[u]);
            if (p0 + t.rows * U < len) fetch(cv, p0 + t.rows * U);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = p0 + u * t.rows;
                if constexpr (MX4) store_mx4<V>(out, o[u], first + p, (d.C + 31) / 32, cv * V, p < len);
                else if (p < len) store(out, static_cast<T *>(out.y) + (first + p) * out.pitch + cv * V, o[u]);
            }
        }
        if (t.rows > 1) break;
    }
}

// ---- the same, written in 4 bits, where C is no multiple of 32: a thread takes a block of 32 channels of a pixel
template <typename T, int V>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_apply_blocks(TdcNormDims d, NormIn in, NormOut out, const float4 *__restrict__ partial, int parts)
{
    extern __shared__ float2 stats[];                      // [G]
    const int b = blockIdx.y, chunk = blockIdx.x;
    statistics(d, out, partial, parts, b, chunk, stats);
    const int nb = (d.C + 31) / 32;
    const T *x = static_cast<const T *>(in.x), *res = static_cast<const T *>(in.residual);
    const size_t total = (size_t)tdc_chunk_len(d, chunk) * nb, first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    for (size_t i = threadIdx.x; i < total; i += TDC_NORM_THREADS) {
        const size_t px = first + i / nb;
        const int c0 = (int)(i % nb) * 32;
        float o[32];
#pragma unroll
        for (int j = 0; j < 32; j += V) {
            float part[V];
#pragma unroll
            for (int v = 0; v < V; ++v) part[v] = 0.f;
            if (c0 + j < d.C) {                            // V divides C: all of them or none
                Affine<V> a;
                a.weights(in, c0 + j);
                a.statistics(d, stats, 0, c0 + j);
                TdcVec<T, V> rv;
                if (res) rv = tdc_load<T, V>(res + px * in.rp + c0 + j);
                apply(a, tdc_load<T, V>(x + px * in.xp + c0 + j), rv, in, part);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) o[j + v] = part[v];
        }
        unsigned e;
        const tdc_i4 c = tdc_mx4_block(o, e);
        *reinterpret_cast<tdc_i4 *>(out.codes + (px * nb + c0 / 32) * 16) = c;
        out.scales[px * nb + c0 / 32] = (uint8_t)e;
    }
}

int validate(const tdc_norm_shape &s)
{
    if (s.batch < 1 || s.H < 1 || s.W < 1 || s.C < 1 || s.groups < 1 || s.C % s.groups || !(s.eps >= 0.f) || !std::isfinite(s.eps)) return TDC_ERR_BAD_SHAPE;
    if (!tdc_known_dtype(s.dtype) || !tdc_known_act(s.act)) return TDC_ERR_UNSUPPORTED;
    if (s.batch > 65535 || s.C > TDC_NORM_MAX_C || (int64_t)s.H * s.W > 0x7fffffff) return TDC_ERR_UNSUPPORTED;
    return TDC_OK;
}

int64_t pitch_or(int64_t pitch, int C) { return pitch ? pitch : C; }

// Of a forward call on aligned tensors without gaps.
int launches(const tdc_norm_plan *p, bool mx4) { return tdc_norm_launches(p->dims, tdc_dtype_bytes(p->shape.dtype), tdc_norm_vec(p->shape.dtype, p->dims.C, {}, {}), mx4); }

}  // namespace

extern "C" {

int tdc_norm_plan_create(tdc_norm_plan **out, const tdc_norm_shape *shape, int device)
{
    if (!out || !shape) return TDC_ERR_NULL;
    *out = nullptr;
    int rc = validate(*shape);
    if (rc != TDC_OK) return rc;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || device < 0 || device >= ndev) return TDC_ERR_HIP;
    DeviceGuard guard(device);
    if (!guard.ok) return TDC_ERR_HIP;
    tdc_norm_plan *p = new (std::nothrow) tdc_norm_plan();
    if (!p) return TDC_ERR_ALLOC;
    p->shape = *shape;
    p->device = device;
    p->dims = TdcNormDims{shape->batch, shape->H * shape->W, shape->C, shape->groups, shape->C / shape->groups, 0, 0, shape->eps};
    tdc_norm_choose_chunks(p->dims, tdc_dtype_bytes(shape->dtype));
    const size_t groups = (size_t)p->dims.B * p->dims.G, partials = groups * p->dims.chunks;
    const size_t sums = tdc_norm_sum_rows(p->dims) * p->dims.C;
    p->ws_bytes = (partials + groups) * sizeof(float4) + sums * sizeof(float2);
    if (hipMalloc((void **)&p->partial, p->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete p;
        return TDC_ERR_ALLOC;
    }
    p->whole = p->partial + partials;
    p->sums = reinterpret_cast<float2 *>(p->whole + groups);
    *out = p;
    return TDC_OK;
}

int tdc_norm_plan_destroy(tdc_norm_plan *p)
{
    if (!p) return TDC_OK;
    DeviceGuard guard(p->device);
    const int rc = hipFree(p->partial) == hipSuccess ? TDC_OK : TDC_ERR_HIP;
    delete p;
    return rc;
}

size_t tdc_norm_plan_workspace_bytes(const tdc_norm_plan *p) { return p ? p->ws_bytes : 0; }

int tdc_norm_plan_kernel_count(const tdc_norm_plan *p) { return p ? launches(p, false) : 0; }

int tdc_norm_plan_mx4_kernel_count(const tdc_norm_plan *p) { return p ? launches(p, true) : 0; }

}  // extern "C"

namespace {

// Both forward calls: y, or codes and scales.
int forward(tdc_norm_plan *p, hipStream_t s, const void *x, const float *gamma, const float *beta, void *y, uint8_t *codes, uint8_t *scales, const tdc_norm_args *args)
{
    const tdc_norm_args none{};
    const tdc_norm_args &a = args ? *args : none;
    const TdcNormDims &d = p->dims;
    const int dt = p->shape.dtype, size = tdc_dtype_bytes(dt);
    const int64_t xp = pitch_or(a.x_pitch, d.C), rp = pitch_or(a.residual_pitch, d.C), yp = pitch_or(a.y_pitch, d.C);
    if (xp < d.C || rp < d.C || yp < d.C) return TDC_ERR_BAD_SHAPE;
    if (!tdc_aligned_to(x, size) || !tdc_aligned_to(a.residual, size) || !tdc_aligned_to(y, size)) return TDC_ERR_UNSUPPORTED;
    if (!tdc_aligned_to(codes, 16)) return TDC_ERR_UNSUPPORTED;
    DeviceGuard guard(p->device);
    if (!guard.ok) return TDC_ERR_HIP;
    const NormIn in{x, a.residual, gamma, beta, xp, rp, p->shape.act};
    const int vx = tdc_norm_vec(dt, d.C, {xp}, {x});
    const int V0 = y ? tdc_norm_vec(dt, d.C, {xp, a.residual ? rp : 0, yp}, {x, a.residual, y}) : tdc_norm_vec(dt, d.C, {xp, a.residual ? rp : 0}, {x, a.residual});
    const bool lanes = codes && tdc_norm_block_lanes(d, size, V0);
    const TdcNormSlice sl = tdc_norm_forward_slice(d, size, V0, codes != nullptr);
    const NormOut out{y, codes, scales, yp, a.mean, a.rstd, y && tdc_norm_streams(d, size, V0, sl)};
    const bool whole = d.Cg % V0 == 0, whole_x = d.Cg % vx == 0;
    const dim3 grid(d.chunks, d.B);
    if (sl.held) {
        TDC_FOR_DTYPE(dt, T, TDC_FOR_VEC(V0, T, V, TDC_FOR_SLICE(sl, tdc_norm_held(V, sizeof(T), false), true, THREADS, HELD, {
            const unsigned wgs = (unsigned)d.B * sl.slices;
            if (lanes) {
                if constexpr (V * sizeof(T) == 16) {
                    if (whole) tdc_norm_resident<T, V, true, true, THREADS, HELD><<<wgs, THREADS, 0, s>>>(d, in, out, sl.width, sl.slices, sl.held);
                    else tdc_norm_resident<T, V, false, true, THREADS, HELD><<<wgs, THREADS, 0, s>>>(d, in, out, sl.width, sl.slices, sl.held);
                }
            } else {
                if (whole) tdc_norm_resident<T, V, true, false, THREADS, HELD><<<wgs, THREADS, 0, s>>>(d, in, out, sl.width, sl.slices, sl.held);
                else tdc_norm_resident<T, V, false, false, THREADS, HELD><<<wgs, THREADS, 0, s>>>(d, in, out, sl.width, sl.slices, sl.held);
            }
        })));
        return hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
    }
    hipError_t e = hipErrorInvalidValue;
    TDC_FOR_DTYPE(dt, T, {
        TDC_FOR_VEC(vx, T, V, {
            const int nv = d.C / V, rows = nv < TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
            const size_t lds = (size_t)rows * (whole_x ? nv : d.C) * sizeof(float2);
            e = tdc_norm_launch(whole_x ? tdc_norm_stats<T, V, true> : tdc_norm_stats<T, V, false>, grid, lds, s, d, in, p->partial);
        });
        if (e != hipSuccess) return TDC_ERR_HIP;
        const bool between = d.chunks > TDC_NORM_PARTS;
        if (between) tdc_norm_combine<<<dim3(d.G, d.B), 64, 0, s>>>(d, p->partial, p->whole);
        const float4 *sums = between ? p->whole : p->partial;
        const int parts = between ? 1 : d.chunks;
        TDC_FOR_VEC(V0, T, V, {
            const size_t lds = d.G * sizeof(float2);
            if (y) e = tdc_norm_launch(tdc_norm_apply<T, V, false>, grid, lds, s, d, in, out, sums, parts);
            else if (!lanes) e = tdc_norm_launch(tdc_norm_apply_blocks<T, V>, grid, lds, s, d, in, out, sums, parts);
            else if constexpr (V * sizeof(T) == 16) e = tdc_norm_launch(tdc_norm_apply<T, V, true>, grid, lds, s, d, in, out, sums, parts);
        });
    });
    return e == hipSuccess && hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}

}  // namespace

extern "C" {

int tdc_group_norm(tdc_norm_plan *p, void *hip_stream, const void *x, const float *gamma, const float *beta, void *y, const tdc_norm_args *args)
{
    if (!p || !x || !y) return TDC_ERR_NULL;
    return forward(p, (hipStream_t)hip_stream, x, gamma, beta, y, nullptr, nullptr, args);
}

int tdc_group_norm_mx4(tdc_norm_plan *p, void *hip_stream, const void *x, const float *gamma, const float *beta, uint8_t *codes, uint8_t *scales,
                       const tdc_norm_args *args)
{
    if (!p || !x || !codes || !scales) return TDC_ERR_NULL;
    return forward(p, (hipStream_t)hip_stream, x, gamma, beta, nullptr, codes, scales, args);
}

}  // extern "C"
