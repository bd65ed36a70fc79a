// Backward pass of the group norm with an activation (tdc_norm.h).
//
// With d = dy act'(pre), recomputed from x, and g = d gamma: dx needs the sums of g and g xhat over a group of an image, dgamma
// and dbeta those of d xhat and d over all images.  Resident: a workgroup keeps its slice of x and dy in registers, reads them
// once, and goes through several images with its channels' sums; a second launch adds up what the workgroups have for each
// channel.  Over chunks: a first kernel leaves the sums of every chunk and group, and its channels' sums; the second combines an
// image's, runs over the pixels again, and in its last workgroups adds up the channels' sums.
#include "tdc_norm_internal.h"

namespace {

struct GradIn {
    const void *x, *dy, *residual;
    const float *mean, *rstd, *gamma, *beta;
    int64_t xp, dyp, rp;
    int act;
};

struct GradOut {
    void *dx, *dresidual;
    int64_t dxp, drp;
};

// What a thread needs to know of its V channels.
template <int V> struct Channels {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ void weights(const GradIn &q, int c0)
    {
        // one branch to all of them: behind a branch of its own each load would wait by itself
#pragma unroll
        for (int v = 0; v < V; ++v) gamma[v] = 1.f, beta[v] = 0.f;
        if (q.gamma) {
#pragma unroll
            for (int v = 0; v < V; ++v) gamma[v] = q.gamma[c0 + v];
        }
        if (q.beta) {
#pragma unroll
            for (int v = 0; v < V; ++v) beta[v] = q.beta[c0 + v];
        }
    }
    __device__ __forceinline__ void statistics(const TdcNormDims &d, const GradIn &q, int b, int c0)
    {
        tdc_norm_channels<V>(c0, d.Cg, [&](int v, int g) {
            mean[v] = q.mean[(size_t)b * d.G + g];
            rstd[v] = q.rstd[(size_t)b * d.G + g];
        });
    }
};

// d and xhat of V channels of a pixel.  pre is computed as the forward kernel does, so that both see the same side of a ReLU.
template <typename T, int V>
__device__ __forceinline__ void gradient(const Channels<V> &k, const TdcVec<T, V> &x, const TdcVec<T, V> &dy, const TdcVec<T, V> &res, const GradIn &q, float (&dd)[V],
                                         float (&xhat)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) {
        xhat[v] = ((float)x.v[v] - k.mean[v]) * k.rstd[v];
        dd[v] = (float)dy.v[v];
    }
    if (q.act != TDC_ACT_NONE) {
        float pre[V];
#pragma unroll
        for (int v = 0; v < V; ++v) pre[v] = ((float)x.v[v] - k.mean[v]) * (k.rstd[v] * k.gamma[v]) + k.beta[v];
        if (q.residual) {
#pragma unroll
            for (int v = 0; v < V; ++v) pre[v] += (float)res.v[v];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) dd[v] = q.act == TDC_ACT_RELU ? tdc_activate_back<TDC_ACT_RELU>(dd[v], pre[v]) : tdc_activate_back<TDC_ACT_SILU>(dd[v], pre[v]);
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_gradients(const Channels<V> &k, const GradOut &out, const float (&m1)[V], const float (&m2)[V], const float (&dd)[V], const float (&xhat)[V], size_t px, int c0)
{
    float o[V];
#pragma unroll
    for (int v = 0; v < V; ++v) o[v] = k.rstd[v] * (dd[v] * k.gamma[v] - m1[v] - xhat[v] * m2[v]);
    // Past the L2's replacement where pieces are whole; 32 images, otherwise and so: 56x56x256 in fp32 106.6 us and 90.9, in bf16
    // 61.8 and 57.5, 14x14x1024 18.1 and 17.9, 28x28x512 35.4 and 35.8; a choice at run time cost 4 %.
    auto store = [](T *p, const float (&f)[V]) {
        if constexpr (V == 4) tdc_store_stream<T, V>(p, f);
        else tdc_store<T, V>(p, f);
    };
    store(static_cast<T *>(out.dx) + px * out.dxp + c0, o);
    if (out.dresidual) store(static_cast<T *>(out.dresidual) + px * out.drp + c0, dd);
}

// A thread's channels' sums as items of groups, into LDS: with their weights, the piece as a whole (WHOLE) or every channel by
// itself.  Returns the number of rows of items.
template <int V, bool WHOLE, int THREADS>
__device__ __forceinline__ int put_items(float2 *items, const TdcNormLanes &t, int cv, int nv, bool live, int used, const Channels<V> &k, const float (&s1)[V], const float (&s2)[V])
{
    constexpr int I = WHOLE ? 1 : V;
    float a[I], b[I];
    if constexpr (WHOLE) {
        a[0] = b[0] = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            a[0] += s1[v] * k.gamma[v];
            b[0] += s2[v] * k.gamma[v];
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            a[v] = s1[v] * k.gamma[v];
            b[v] = s2[v] * k.gamma[v];
        }
    }
    return tdc_norm_put_sums<I, THREADS>(items, a, b, t, cv, nv, live, used);
}

// The threads' channels' sums added up over the workgroup into `out` [width], through `chan` in LDS, which every thread has left.
template <int V, int THREADS> __device__ __forceinline__ void add_rows(float2 *chan, float (&t1)[V], float (&t2)[V], const TdcNormLanes &t, int nv, bool live, int used, float2 *out)
{
    int rows = tdc_norm_put_sums<V, THREADS>(chan, t1, t2, t, t.cv, nv, live, used);
    __syncthreads();
    const int width = nv * V, per = max(1, min(THREADS / width, rows));
    if (per > 1) {
        const int k = threadIdx.x / width, c = threadIdx.x - k * width;
        float s1 = 0.f, s2 = 0.f;
        if (k < per)
            for (int i = k; i < rows; i += per) {
                s1 += chan[i * width + c].x;
                s2 += chan[i * width + c].y;
            }
        __syncthreads();
        if (k < per) chan[k * width + c] = make_float2(s1, s2);
        __syncthreads();
        rows = per;
    }
    for (int i = threadIdx.x; i < width; i += THREADS) {
        float s1 = 0.f, s2 = 0.f;
        for (int j = 0; j < rows; ++j) {
            s1 += chan[j * width + i].x;
            s2 += chan[j * width + i].y;
        }
        out[i] = make_float2(s1, s2);
    }
}

// dgamma and dbeta of 32 channels from `rows` rows of channels' sums, THREADS / 32 threads to a channel.
template <int THREADS> __device__ __forceinline__ void add_weights(int C, const float2 *sums, int rows, int c0, float *dgamma, float *dbeta)
{
    __shared__ float2 tot[THREADS];
    const int c = c0 + (threadIdx.x & 31), k = threadIdx.x >> 5;
    float s1 = 0.f, s2 = 0.f;
    if (c < C) {
#pragma unroll 4
        for (int i = k; i < rows; i += THREADS / 32) {
            const float2 v = sums[(size_t)i * C + c];
            s1 += v.x;
            s2 += v.y;
        }
    }
    tot[threadIdx.x] = make_float2(s1, s2);
    __syncthreads();
    if (k == 0 && c < C) {
        for (int i = 1; i < THREADS / 32; ++i) {
            s1 += tot[32 * i + threadIdx.x].x;
            s2 += tot[32 * i + threadIdx.x].y;
        }
        if (dgamma) dgamma[c] = s2;
        if (dbeta) dbeta[c] = s1;
    }
}

template <int THREADS> __global__ __launch_bounds__(THREADS) void tdc_norm_grad_weights(int C, const float2 *__restrict__ sums, int rows, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    add_weights<THREADS>(C, sums, rows, blockIdx.x * 32, dgamma, dbeta);
}

// An image's chunks in one, a wavefront to a group, and behind them the workgroups that add up the channels' sums.
__global__ __launch_bounds__(256) void tdc_norm_grad_combine(TdcNormDims d, const float2 *__restrict__ partial, float2 *__restrict__ whole, int wgs, const float2 *__restrict__ sums,
                                                             int rows, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    if ((int)blockIdx.x >= wgs) {
        add_weights<256>(d.C, sums, rows, (blockIdx.x - wgs) * 32, dgamma, dbeta);
        return;
    }
    const size_t at = (size_t)blockIdx.x * 4 + threadIdx.x / 64, b = at / d.G, g = at - b * d.G;
    if (b >= (size_t)d.B) return;
    const float2 *p = partial + b * d.chunks * d.G + g;
    float s1 = 0.f, s2 = 0.f;
#pragma unroll 8
    for (int i = threadIdx.x & 63; i < d.chunks; i += 64) {
        const float2 o = p[(size_t)i * d.G];
        s1 += o.x;
        s2 += o.y;
    }
    s1 = tdc_lane_sum(s1, 64);
    s2 = tdc_lane_sum(s2, 64);
    if ((threadIdx.x & 63) == 0) whole[at] = make_float2(s1, s2);
}

// ---- resident: workgroup (row, slice) takes images row, row + rows_of_images, ...
// After the sums a thread keeps x and d, in fp32: the residual is read once, the activation's slope computed once.
template <typename T, int V, bool WHOLE, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void tdc_norm_grad_resident(TdcNormDims d, GradIn q, GradOut out, int width, int slices, int held_here, float2 *__restrict__ sums)
{
    __shared__ float2 items[THREADS * V], means[THREADS];
    int image, slice;
    tdc_norm_place(blockIdx.x, gridDim.x, slices, image, slice);
    const int first = image, images = gridDim.x / slices, nv = width / V, groups = width / d.Cg;
    const TdcNormLanes t(nv, THREADS);
    const int used = min(t.rows, d.P);
    const bool live = t.r < used && t.cv < nv, has_res = q.residual && q.act != TDC_ACT_NONE;
    const int c0 = slice * width + (live ? t.cv * V : 0), g0 = slice * width / d.Cg;
    const float inv = 1.f / ((float)d.P * d.Cg);
    Channels<V> k;
    k.weights(q, c0);
    float t1[V], t2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) t1[v] = t2[v] = 0.f;
    for (; image < d.B; image += images) {
        const size_t first_px = (size_t)image * d.P;
        const T *px = static_cast<const T *>(q.x) + first_px * q.xp + c0, *pdy = static_cast<const T *>(q.dy) + first_px * q.dyp + c0;
        const T *pres = has_res ? static_cast<const T *>(q.residual) + first_px * q.rp + c0 : nullptr;
        TdcRaw<T, V> x[HELD];
        float dd[HELD][V], s1[V], s2[V];
#pragma unroll
        for (int v = 0; v < V; ++v) s1[v] = s2[v] = 0.f;
        if (live) {
            TdcRaw<T, V> dy[HELD], res[HELD];
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i < held_here) {
                    const int p = tdc_anew(min(t.r + i * t.rows, d.P - 1));
                    x[i].load(px + (size_t)p * q.xp);
                    dy[i].load(pdy + (size_t)p * q.dyp);
                    if (has_res) res[i].load(pres + (size_t)p * q.rp);
                }
            k.statistics(d, q, image, c0);
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (t.r + i * t.rows < d.P) {
                    float xhat[V];
                    gradient(k, x[i].open(), dy[i].open(), res[i].open(), q, dd[i], xhat);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        s1[v] += dd[i][v];
                        s2[v] += dd[i][v] * xhat[v];
                    }
                }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                t1[v] += s1[v];
                t2[v] += s2[v];
            }
        }
        const int rows = put_items<V, WHOLE, THREADS>(items, t, t.cv, nv, live, used, k, s1, s2);
        __syncthreads();
        tdc_norm_group_sums(items, rows, groups, WHOLE ? d.Cg / V : d.Cg, THREADS, [&](int g, float a, float b) { means[g] = make_float2(a * inv, b * inv); });
        __syncthreads();
        if (live) {
            float m1[V], m2[V];
            tdc_norm_channels<V>(c0, d.Cg, [&](int v, int g) {
                m1[v] = means[g - g0].x;
                m2[v] = means[g - g0].y;
            });
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int p = tdc_anew(t.r + i * t.rows);
                if (p >= d.P) break;
                const TdcVec<T, V> xv = x[i].open();
                float xhat[V];
#pragma unroll
                for (int v = 0; v < V; ++v) xhat[v] = ((float)xv.v[v] - k.mean[v]) * k.rstd[v];
                store_gradients<T, V>(k, out, m1, m2, dd[i], xhat, first_px + p, c0);
            }
        }
    }
    if (!sums) return;
    __syncthreads();
    add_rows<V, THREADS>(items, t1, t2, t, nv, live, used, sums + (size_t)first * d.C + slice * width);
}

// ---- sums of chunks: grid (chunks, rows of images)
template <typename T, int V, bool WHOLE>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_grad_sums(TdcNormDims d, GradIn q, float2 *__restrict__ partial, float2 *__restrict__ sums)
{
    constexpr int U = TDC_NORM_UNROLL / 2;
    extern __shared__ float2 items[];                      // rows * C
    const int nv = d.C / V, chunk = blockIdx.x, len = tdc_chunk_len(d, chunk);
    const TdcNormLanes t(nv, TDC_NORM_THREADS);
    const int used = min(t.rows, len);
    const T *res = q.act != TDC_ACT_NONE ? static_cast<const T *>(q.residual) : nullptr;
    float t1[V], t2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) t1[v] = t2[v] = 0.f;
    for (int b = blockIdx.y; b < d.B; b += gridDim.y) {
        const size_t first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
        int rows = 1;
        for (int cv = t.cv; cv < nv || cv == t.cv; cv += TDC_NORM_THREADS) {   // once, but for pixels of more pieces than there are threads
            const bool live = t.r < used && cv < nv;
            Channels<V> k;
            float s1[V], s2[V];
#pragma unroll
            for (int v = 0; v < V; ++v) s1[v] = s2[v] = 0.f;
            k.weights(q, live ? cv * V : 0);
            if (live) {
                k.statistics(d, q, b, cv * V);
                for (int p0 = t.r; p0 < len; p0 += t.rows * U) {
                    TdcRaw<T, V> xv[U], dv[U], rv[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const size_t px = first + min(p0 + u * t.rows, len - 1);
                        xv[u].load(static_cast<const T *>(q.x) + px * q.xp + cv * V);
                        dv[u].load(static_cast<const T *>(q.dy) + px * q.dyp + cv * V);
                        if (res) rv[u].load(res + px * q.rp + cv * V);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (p0 + u * t.rows >= len) break;
                        float dd[V], xhat[V];
                        gradient(k, xv[u].open(), dv[u].open(), rv[u].open(), q, dd, xhat);
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            s1[v] += dd[v];
                            s2[v] += dd[v] * xhat[v];
                        }
                    }
                }
                if (nv <= TDC_NORM_THREADS) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        t1[v] += s1[v];
                        t2[v] += s2[v];
                    }
                } else if (sums) {
                    // several sweeps to a pixel: the channels' sums of this workgroup, which no other touches, stay in its row
                    float2 *row = sums + (size_t)(blockIdx.y * gridDim.x + chunk) * d.C + cv * V;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float2 o = b == (int)blockIdx.y ? make_float2(0.f, 0.f) : row[v];
                        row[v] = make_float2(o.x + s1[v], o.y + s2[v]);
                    }
                }
            }
            rows = put_items<V, WHOLE, TDC_NORM_THREADS>(items, t, cv, nv, live, used, k, s1, s2);
            if (t.rows > 1) break;
        }
        __syncthreads();
        float2 *to = partial + ((size_t)b * d.chunks + chunk) * d.G;
        tdc_norm_group_sums(items, rows, d.G, WHOLE ? d.Cg / V : d.Cg, TDC_NORM_THREADS, [&](int g, float s1, float s2) { to[g] = make_float2(s1, s2); });
        __syncthreads();
    }
    if (!sums || nv > TDC_NORM_THREADS) return;
    add_rows<V, TDC_NORM_THREADS>(items, t1, t2, t, nv, t.r < used && t.cv < nv, used, sums + (size_t)(blockIdx.y * gridDim.x + chunk) * d.C);
}

// ---- gradients of chunks: grid (chunks, batch), and behind them the workgroups that add up the channels' sums
template <typename T, int V>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_grad_apply(TdcNormDims d, GradIn q, GradOut out, const float2 *__restrict__ partial, int parts, const float2 *__restrict__ sums, int rows,
                                                                         float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    constexpr int U = TDC_NORM_UNROLL / 2;
    extern __shared__ float2 means[];                      // [G]
    const int id = blockIdx.x, b = id / d.chunks, chunk = id - b * d.chunks;
    if (b >= d.B) {
        add_weights<TDC_NORM_THREADS>(d.C, sums, rows, (id - d.B * d.chunks) * 32, dgamma, dbeta);
        return;
    }
    const int nv = d.C / V, len = tdc_chunk_len(d, chunk);
    const float inv = 1.f / ((float)d.P * d.Cg);
    tdc_combine_sums(d, partial, parts, b, TDC_NORM_THREADS, [&](int g, float s1, float s2) { means[g] = make_float2(s1 * inv, s2 * inv); });
    __syncthreads();
    const TdcNormLanes t(nv, TDC_NORM_THREADS);
    if (t.r >= t.rows) return;
    const size_t first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    const T *res = q.act != TDC_ACT_NONE ? static_cast<const T *>(q.residual) : nullptr;
    for (int cv = t.cv; cv < nv; cv += TDC_NORM_THREADS) {
        Channels<V> k;
        k.weights(q, cv * V);
        k.statistics(d, q, b, cv * V);
        float m1[V], m2[V];
        tdc_norm_channels<V>(cv * V, d.Cg, [&](int v, int g) {
            m1[v] = means[g].x;
            m2[v] = means[g].y;
        });
        for (int p0 = t.r; p0 < len; p0 += t.rows * U) {
            TdcRaw<T, V> xv[U], dv[U], rv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const size_t px = first + min(p0 + u * t.rows, len - 1);
                xv[u].load(static_cast<const T *>(q.x) + px * q.xp + cv * V);
                dv[u].load(static_cast<const T *>(q.dy) + px * q.dyp + cv * V);
                if (res) rv[u].load(res + px * q.rp + cv * V);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p0 + u * t.rows >= len) break;
                float dd[V], xhat[V];
                gradient(k, xv[u].open(), dv[u].open(), rv[u].open(), q, dd, xhat);
                store_gradients<T, V>(k, out, m1, m2, dd, xhat, first + p0 + u * t.rows, cv * V);
            }
        }
        if (t.rows > 1) break;
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
    const GradIn q{x, dy, a.residual, mean, rstd, gamma, beta, pitch(a.x_pitch), pitch(a.dy_pitch), pitch(a.residual_pitch), p->shape.act};
    const GradOut out{dx, a.dresidual, pitch(a.dx_pitch), pitch(a.dresidual_pitch)};
    for (int64_t v : {q.xp, q.rp, q.dyp, out.dxp, out.drp})
        if (v < d.C) return TDC_ERR_BAD_SHAPE;
    for (const void *v : {x, dy, a.residual, (const void *)dx, (const void *)a.dresidual})
        if (!tdc_aligned_to(v, size)) return TDC_ERR_UNSUPPORTED;
    DeviceGuard guard(p->device);
    if (!guard.ok) return TDC_ERR_HIP;
    hipStream_t s = (hipStream_t)hip_stream;
    const int weight_blocks = dgamma || dbeta ? (d.C + 31) / 32 : 0;
    float2 *sums = weight_blocks ? p->sums : nullptr;
    const int vec = tdc_norm_vec(dt, d.C, {q.xp, a.residual ? q.rp : 0, q.dyp, out.dxp, a.dresidual ? out.drp : 0}, {x, dy, a.residual, dx, a.dresidual}, 4);
    const bool whole = d.Cg % vec == 0;
    const TdcNormSlice sl = tdc_norm_slice(d, size, vec, true, 1);
    if (sl.held) {
        const int rows = tdc_norm_resident_rows(d, sl.slices);
        TDC_FOR_DTYPE(dt, T, TDC_FOR_VEC4(vec, V, TDC_FOR_SLICE(sl, tdc_norm_held(V, sizeof(T), true), false, THREADS, HELD, {
            const unsigned wgs = (unsigned)rows * sl.slices;
            if (whole) tdc_norm_grad_resident<T, V, true, THREADS, HELD><<<wgs, THREADS, 0, s>>>(d, q, out, sl.width, sl.slices, sl.held, sums);
            else tdc_norm_grad_resident<T, V, false, THREADS, HELD><<<wgs, THREADS, 0, s>>>(d, q, out, sl.width, sl.slices, sl.held, sums);
        })));
        if (sums) tdc_norm_grad_weights<256><<<weight_blocks, 256, 0, s>>>(d.C, sums, rows, dgamma, dbeta);
        return hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
    }
    const int images = tdc_norm_chunk_images(d);
    float2 *partial = reinterpret_cast<float2 *>(p->partial);
    hipError_t e = hipErrorInvalidValue;
    TDC_FOR_DTYPE(dt, T, TDC_FOR_VEC4(vec, V, {
        const int nv = d.C / V, rows = nv < TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
        const size_t lds = (size_t)rows * d.C * sizeof(float2);
        const dim3 grid(d.chunks, images);
        e = tdc_norm_launch(whole ? tdc_norm_grad_sums<T, V, true> : tdc_norm_grad_sums<T, V, false>, grid, lds, s, d, q, partial, sums);
        if (e != hipSuccess) return TDC_ERR_HIP;
        const size_t lds_means = d.G * sizeof(float2);
        if (d.chunks > TDC_NORM_PARTS) {
            float2 *all = reinterpret_cast<float2 *>(p->whole);
            const unsigned wgs = (unsigned)(((size_t)d.B * d.G + 3) / 4);
            tdc_norm_grad_combine<<<wgs + weight_blocks, 256, 0, s>>>(d, partial, all, (int)wgs, sums, images * d.chunks, dgamma, dbeta);
            e = tdc_norm_launch(tdc_norm_grad_apply<T, V>, (unsigned)d.B * d.chunks, lds_means, s, d, q, out, all, 1, (const float2 *)nullptr, 0, (float *)nullptr, (float *)nullptr);
        } else {
            e = tdc_norm_launch(tdc_norm_grad_apply<T, V>, (unsigned)d.B * d.chunks + weight_blocks, lds_means, s, d, q, out, partial, d.chunks, sums, images * d.chunks, dgamma, dbeta);
        }
    }));
    return e == hipSuccess && hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}
