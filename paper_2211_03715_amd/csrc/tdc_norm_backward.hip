// Backward pass of the group norm with an activation (tdc_norm.h), in three kernels:
//   1. per chunk and channel, sum d and sum d xhat, with d = dy act'(pre) recomputed from x;
//   2. dgamma and dbeta, sums over all images and chunks; and for every image and group the means of g and g xhat, g = d gamma;
//   3. dx = rstd (g - m(g) - xhat m(g xhat)), and dresidual = d.
#include <initializer_list>

#include "tdc_norm_internal.h"

namespace {

struct GradPtrs {
    const float *mean, *rstd, *gamma, *beta;
    int64_t xp, rp, dyp, dxp, drp;
};

// What a thread needs to know of its V channels.
template <int V> struct Channels {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ Channels(const TdcNormDims &d, const GradPtrs &q, int b, int c0)
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const size_t g = (size_t)b * d.G + (c0 + v) / d.Cg;
            mean[v] = q.mean[g];
            rstd[v] = q.rstd[g];
            gamma[v] = q.gamma ? q.gamma[c0 + v] : 1.f;
            beta[v] = q.beta ? q.beta[c0 + v] : 0.f;
        }
    }
};

// d and xhat of V channels of a pixel.  pre is computed as the forward kernel does, so that both see the same side of a ReLU.
template <typename T, int V, int ACT>
__device__ __forceinline__ void tdc_norm_d(const Channels<V> &k, const TdcVec<T, V> &x, const TdcVec<T, V> &dy, const TdcVec<T, V> &res, bool has_res,
                                           float (&dd)[V], float (&xhat)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float off = (float)x.v[v] - k.mean[v];
        xhat[v] = off * k.rstd[v];
        dd[v] = (float)dy.v[v];
        if (ACT != TDC_ACT_NONE) {
            float pre = off * (k.rstd[v] * k.gamma[v]) + k.beta[v];
            if (has_res) pre += (float)res.v[v];
            dd[v] *= tdc_activate_grad<ACT>(pre);
        }
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_grad_sums(TdcNormDims d, GradPtrs q, const T *__restrict__ x, const T *__restrict__ dy,
                                                                        const T *__restrict__ res, float2 *__restrict__ partial)
{
    extern __shared__ float2 chan[];                       // [rows][C]
    const int nv = d.C / V, b = blockIdx.y, chunk = blockIdx.x;
    const int len = tdc_chunk_len(d, chunk);
    const int rows = nv <= TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
    const int r = rows == 1 ? 0 : threadIdx.x / nv;
    const size_t first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    float2 *out = partial + ((size_t)b * d.chunks + chunk) * d.C;
    if (r < rows)
        for (int cv = rows == 1 ? threadIdx.x : threadIdx.x - r * nv; cv < nv; cv += TDC_NORM_THREADS) {
            const Channels<V> k(d, q, b, cv * V);
            float s1[V], s2[V];
#pragma unroll
            for (int v = 0; v < V; ++v) s1[v] = s2[v] = 0.f;
            for (int p = r; p < len; p += rows) {
                const size_t px = first + p;
                const TdcVec<T, V> xv = tdc_load<T, V>(x + px * q.xp + cv * V), dv = tdc_load<T, V>(dy + px * q.dyp + cv * V);
                TdcVec<T, V> rv;
                if (ACT != TDC_ACT_NONE && res) rv = tdc_load<T, V>(res + px * q.rp + cv * V);
                float dd[V], xhat[V];
                tdc_norm_d<T, V, ACT>(k, xv, dv, rv, res != nullptr, dd, xhat);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    s1[v] += dd[v];
                    s2[v] += dd[v] * xhat[v];
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (rows == 1) out[cv * V + v] = make_float2(s1[v], s2[v]);
                else chan[r * d.C + cv * V + v] = make_float2(s1[v], s2[v]);
            }
            if (rows > 1) break;
        }
    if (rows == 1) return;
    __syncthreads();
    for (int c = threadIdx.x; c < d.C; c += TDC_NORM_THREADS) {
        float s1 = 0.f, s2 = 0.f;
        for (int i = 0; i < rows; ++i) {
            s1 += chan[i * d.C + c].x;
            s2 += chan[i * d.C + c].y;
        }
        out[c] = make_float2(s1, s2);
    }
}

// Workgroups 0 .. weight_blocks-1: dgamma and dbeta of 32 channels, eight threads to a channel.  The others: an image each.
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_grad_reduce(TdcNormDims d, const float *__restrict__ gamma, const float2 *__restrict__ partial,
                                                                          int weight_blocks, float *__restrict__ dgamma, float *__restrict__ dbeta, float2 *__restrict__ means)
{
    extern __shared__ float2 tot[];                        // [C], or [8][32]
    if ((int)blockIdx.x < weight_blocks) {
        const int c = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
        float s1 = 0.f, s2 = 0.f;
        if (c < d.C)
            for (size_t i = lane; i < (size_t)d.B * d.chunks; i += 8) {
                const float2 v = partial[i * d.C + c];
                s1 += v.x;
                s2 += v.y;
            }
        tot[threadIdx.x] = make_float2(s1, s2);
        __syncthreads();
        if (lane == 0 && c < d.C) {
            for (int i = 1; i < 8; ++i) {
                s1 += tot[32 * i + threadIdx.x].x;
                s2 += tot[32 * i + threadIdx.x].y;
            }
            if (dgamma) dgamma[c] = s2;
            if (dbeta) dbeta[c] = s1;
        }
        return;
    }
    const int b = blockIdx.x - weight_blocks;
    for (int c = threadIdx.x; c < d.C; c += TDC_NORM_THREADS) {
        const float2 *p = partial + (size_t)b * d.chunks * d.C + c;
        float s1 = 0.f, s2 = 0.f;
        for (int i = 0; i < d.chunks; ++i) {
            s1 += p[(size_t)i * d.C].x;
            s2 += p[(size_t)i * d.C].y;
        }
        const float w = gamma ? gamma[c] : 1.f;
        tot[c] = make_float2(s1 * w, s2 * w);
    }
    __syncthreads();
    const int L = tdc_team(d.G, d.Cg), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = TDC_NORM_THREADS / L;
    const float inv = 1.f / ((float)d.P * d.Cg);
    for (int g0 = 0; g0 < d.G; g0 += teams) {
        const int g = min(g0 + team, d.G - 1);
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < d.Cg; c += L) {
            s1 += tot[g * d.Cg + c].x;
            s2 += tot[g * d.Cg + c].y;
        }
        s1 = tdc_lane_sum(s1, L);
        s2 = tdc_lane_sum(s2, L);
        if (lane == 0 && g0 + team < d.G) means[(size_t)b * d.G + g] = make_float2(s1 * inv, s2 * inv);
    }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_grad_apply(TdcNormDims d, GradPtrs q, const T *__restrict__ x, const T *__restrict__ dy,
                                                                         const T *__restrict__ res, const float2 *__restrict__ means, T *__restrict__ dx, T *__restrict__ dres)
{
    const int nv = d.C / V, b = blockIdx.y, chunk = blockIdx.x;
    const int len = tdc_chunk_len(d, chunk);
    const int rows = nv <= TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
    const int r = rows == 1 ? 0 : threadIdx.x / nv;
    if (r >= rows) return;
    const size_t first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    for (int cv = rows == 1 ? threadIdx.x : threadIdx.x - r * nv; cv < nv; cv += TDC_NORM_THREADS) {
        const Channels<V> k(d, q, b, cv * V);
        float m1[V], m2[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float2 m = means[(size_t)b * d.G + (cv * V + v) / d.Cg];
            m1[v] = m.x;
            m2[v] = m.y;
        }
        for (int p = r; p < len; p += rows) {
            const size_t px = first + p;
            const TdcVec<T, V> xv = tdc_load<T, V>(x + px * q.xp + cv * V), dv = tdc_load<T, V>(dy + px * q.dyp + cv * V);
            TdcVec<T, V> rv;
            if (ACT != TDC_ACT_NONE && res) rv = tdc_load<T, V>(res + px * q.rp + cv * V);
            float dd[V], xhat[V], o[V];
            tdc_norm_d<T, V, ACT>(k, xv, dv, rv, res != nullptr, dd, xhat);
#pragma unroll
            for (int v = 0; v < V; ++v) o[v] = k.rstd[v] * (dd[v] * k.gamma[v] - m1[v] - xhat[v] * m2[v]);
            tdc_store<T, V>(dx + px * q.dxp + cv * V, o);
            if (dres) tdc_store<T, V>(dres + px * q.drp + cv * V, dd);
        }
        if (rows > 1) break;
    }
}

}  // namespace

extern "C" int tdc_group_norm_backward(tdc_norm_plan *p, void *hip_stream, const void *x, const void *dy, const float *mean, const float *rstd,
                                       const float *gamma, const float *beta, void *dx, float *dgamma, float *dbeta, const tdc_norm_grad_args *args)
{
    if (!p || !x || !dy || !mean || !rstd || !dx) return TDC_ERR_NULL;
    const tdc_norm_grad_args none{};
    const tdc_norm_grad_args &a = args ? *args : none;
    const TdcNormDims &d = p->dims;
    const int dt = p->shape.dtype, size = tdc_dtype_bytes(dt);
    auto pitch = [&](int64_t v) { return v ? v : (int64_t)d.C; };
    const GradPtrs q{mean, rstd, gamma, beta, pitch(a.x_pitch), pitch(a.residual_pitch), pitch(a.dy_pitch), pitch(a.dx_pitch), pitch(a.dresidual_pitch)};
    for (int64_t v : {q.xp, q.rp, q.dyp, q.dxp, q.drp})
        if (v < d.C) return TDC_ERR_BAD_SHAPE;
    for (const void *v : {x, dy, a.residual, (const void *)dx, (const void *)a.dresidual})
        if (!tdc_aligned_to(v, size)) return TDC_ERR_UNSUPPORTED;
    DeviceGuard guard(p->device);
    if (!guard.ok) return TDC_ERR_HIP;
    hipStream_t s = (hipStream_t)hip_stream;
    const dim3 grid(d.chunks, d.B);
    const int weight_blocks = dgamma || dbeta ? (d.C + 31) / 32 : 0;
    const int vec = tdc_norm_vec(dt, d.C, {q.xp, a.residual ? q.rp : 0, q.dyp, q.dxp, a.dresidual ? q.drp : 0}, {x, dy, a.residual, dx, a.dresidual});
    TDC_FOR_DTYPE(dt, T, {
        const T *xt = (const T *)x, *dyt = (const T *)dy, *rt = (const T *)a.residual;
        TDC_FOR_VEC(vec, T, V, TDC_FOR_ACT(p->shape.act, ACT, {
            const int nv = d.C / V, rows = nv <= TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
            tdc_norm_grad_sums<T, V, ACT><<<grid, TDC_NORM_THREADS, rows == 1 ? 0 : (size_t)rows * d.C * sizeof(float2), s>>>(d, q, xt, dyt, rt, p->partial);
            tdc_norm_grad_reduce<<<weight_blocks + d.B, TDC_NORM_THREADS, std::max(d.C, TDC_NORM_THREADS) * sizeof(float2), s>>>(d, gamma, p->partial, weight_blocks, dgamma, dbeta, p->means);
            tdc_norm_grad_apply<T, V, ACT><<<grid, TDC_NORM_THREADS, 0, s>>>(d, q, xt, dyt, rt, p->means, (T *)dx, (T *)a.dresidual);
        }));
    });
    return hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}
