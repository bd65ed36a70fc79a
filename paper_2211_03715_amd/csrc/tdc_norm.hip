// Group norm with an activation, channels last: plans, the forward kernels and their launches (tdc_norm.h).
#include <cmath>
#include <initializer_list>
#include <new>

#include "tdc_mx4_device.h"
#include "tdc_norm_internal.h"

namespace {

// ---- statistics of a chunk: grid (chunks, batch)
//
// A thread takes its V channels of eight pixels at a time into registers, their mean and the squares about it, and merges that
// into what it has (n_a, mean_a, S_a with n_b, mean_b, S_b: mean = mean_a + d n_b / n, S = S_a + S_b + d^2 n_a n_b / n,
// d = mean_b - mean_a).  No sum of squares is ever taken about anything but a mean next to the values, so fp32 does.
template <typename T, int V>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_stats(TdcNormDims d, const T *__restrict__ x, int64_t pitch, float2 *__restrict__ partial)
{
    constexpr int U = 8;
    extern __shared__ float2 chan[];                       // [rows][C]
    const int nv = d.C / V, b = blockIdx.y, chunk = blockIdx.x;
    const int len = tdc_chunk_len(d, chunk);
    const int rows = nv <= TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
    const int r = threadIdx.x / nv, step = nv <= TDC_NORM_THREADS ? nv : TDC_NORM_THREADS;
    const T *base = x + ((size_t)b * d.P + (size_t)chunk * d.chunk_px) * pitch;
    if (rows == 1 || r < rows)
        for (int cv = rows == 1 ? threadIdx.x : threadIdx.x - r * nv; cv < nv; cv += step) {
            float n = 0.f, mean[V], m2[V];
#pragma unroll
            for (int v = 0; v < V; ++v) mean[v] = m2[v] = 0.f;
            for (int p = rows == 1 ? 0 : r; p < len; p += rows * U) {
                TdcVec<T, V> in[U];
#pragma unroll
                for (int u = 0; u < U; ++u) in[u] = tdc_load<T, V>(base + (size_t)min(p + u * rows, len - 1) * pitch + cv * V);
                const int k = min(U, (len - p + rows - 1) / rows);
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
#pragma unroll
            for (int v = 0; v < V; ++v) chan[(rows == 1 ? 0 : r) * d.C + cv * V + v] = make_float2(mean[v], m2[v]);
            if (rows > 1) break;
        }
    __syncthreads();
    // rows of the workgroup into one, channel by channel
    const int used = min(rows, len);
    if (used > 1) {
        for (int c = threadIdx.x; c < d.C; c += TDC_NORM_THREADS) {
            float n = 0.f, mean = 0.f, m2 = 0.f;
            for (int i = 0; i < used; ++i) {
                const float2 o = chan[i * d.C + c];
                const float k = (float)((len - i + rows - 1) / rows), tot = n + k, off = o.x - mean;
                mean += off * (k / tot);
                m2 += o.y + off * off * (n * (k / tot));
                n = tot;
            }
            chan[c] = make_float2(mean, m2);
        }
        __syncthreads();
    }
    // channels into groups, a team of lanes to a group
    const int L = tdc_team(d.G, d.Cg), lane = threadIdx.x & (L - 1), team = threadIdx.x / L, teams = TDC_NORM_THREADS / L;
    for (int g0 = 0; g0 < d.G; g0 += teams) {
        const int g = min(g0 + team, d.G - 1);
        float s = 0.f, m2 = 0.f;
        for (int c = lane; c < d.Cg; c += L) s += chan[g * d.Cg + c].x;
        const float mean = tdc_lane_sum(s, L) / d.Cg;
        for (int c = lane; c < d.Cg; c += L) {
            const float2 o = chan[g * d.Cg + c];
            m2 += o.y + (o.x - mean) * (o.x - mean) * len;
        }
        m2 = tdc_lane_sum(m2, L);
        if (lane == 0 && g0 + team < d.G) partial[((size_t)b * d.chunks + chunk) * d.G + g] = make_float2(mean, m2);
    }
}

// ---- y = act((x - mean) * (rstd gamma) + beta + residual): grid (chunks, batch)
template <typename T, int V, int ACT>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_apply(TdcNormDims d, const T *__restrict__ x, int64_t xp, const float *__restrict__ gamma,
                                                                    const float *__restrict__ beta, const T *__restrict__ res, int64_t rp, T *__restrict__ y,
                                                                    int64_t yp, const float2 *__restrict__ partial, float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    extern __shared__ float2 stats[];                      // [G]
    const int nv = d.C / V, b = blockIdx.y, chunk = blockIdx.x;
    tdc_combine_chunks(d, partial, b, stats);
    if (chunk == 0)
        for (int g = threadIdx.x; g < d.G; g += TDC_NORM_THREADS) {
            if (mean_out) mean_out[(size_t)b * d.G + g] = stats[g].x;
            if (rstd_out) rstd_out[(size_t)b * d.G + g] = stats[g].y;
        }
    const int len = tdc_chunk_len(d, chunk);
    const int rows = nv <= TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
    const int r = rows == 1 ? 0 : threadIdx.x / nv;
    if (r >= rows) return;
    const size_t first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    for (int cv = rows == 1 ? threadIdx.x : threadIdx.x - r * nv; cv < nv; cv += TDC_NORM_THREADS) {
        float mean[V], a[V], shift[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = cv * V + v;
            const float2 st = stats[c / d.Cg];
            mean[v] = st.x;
            a[v] = gamma ? st.y * gamma[c] : st.y;
            shift[v] = beta ? beta[c] : 0.f;
        }
        for (int p = r; p < len; p += rows) {
            const size_t px = first + p;
            const TdcVec<T, V> in = tdc_load<T, V>(x + px * xp + cv * V);
            float o[V];
#pragma unroll
            for (int v = 0; v < V; ++v) o[v] = ((float)in.v[v] - mean[v]) * a[v] + shift[v];
            if (res) {
                const TdcVec<T, V> rv = tdc_load<T, V>(res + px * rp + cv * V);
#pragma unroll
                for (int v = 0; v < V; ++v) o[v] += (float)rv.v[v];
            }
#pragma unroll
            for (int v = 0; v < V; ++v) o[v] = tdc_activate<ACT>(o[v]);
            tdc_store<T, V>(y + px * yp + cv * V, o);
        }
        if (rows > 1) break;
    }
}

// ---- the same, written in 4 bits: a thread takes a block of 32 channels of a pixel
template <typename T, int V, int ACT>
__global__ __launch_bounds__(TDC_NORM_THREADS) void tdc_norm_apply_mx4(TdcNormDims d, const T *__restrict__ x, int64_t xp, const float *__restrict__ gamma,
                                                                        const float *__restrict__ beta, const T *__restrict__ res, int64_t rp,
                                                                        uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                                        const float2 *__restrict__ partial, float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    extern __shared__ float2 stats[];                      // [G]
    const int b = blockIdx.y, chunk = blockIdx.x;
    tdc_combine_chunks(d, partial, b, stats);
    if (chunk == 0)
        for (int g = threadIdx.x; g < d.G; g += TDC_NORM_THREADS) {
            if (mean_out) mean_out[(size_t)b * d.G + g] = stats[g].x;
            if (rstd_out) rstd_out[(size_t)b * d.G + g] = stats[g].y;
        }
    const int nb = (d.C + 31) / 32;
    const size_t total = (size_t)tdc_chunk_len(d, chunk) * nb, first = (size_t)b * d.P + (size_t)chunk * d.chunk_px;
    for (size_t i = threadIdx.x; i < total; i += TDC_NORM_THREADS) {
        const size_t px = first + i / nb;
        const int c0 = (int)(i % nb) * 32;
        float o[32];
#pragma unroll
        for (int j = 0; j < 32; j += V) {
            if (c0 + j < d.C) {                            // V divides C: all of them or none
                const TdcVec<T, V> in = tdc_load<T, V>(x + px * xp + c0 + j);
                TdcVec<T, V> rv;
                if (res) rv = tdc_load<T, V>(res + px * rp + c0 + j);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int c = c0 + j + v;
                    const float2 st = stats[c / d.Cg];
                    float f = ((float)in.v[v] - st.x) * (gamma ? st.y * gamma[c] : st.y) + (beta ? beta[c] : 0.f);
                    if (res) f += (float)rv.v[v];
                    o[j + v] = tdc_activate<ACT>(f);
                }
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) o[j + v] = 0.f;
            }
        }
        unsigned e;
        const tdc_i4 c = tdc_mx4_block(o, e);
        *reinterpret_cast<tdc_i4 *>(codes + (px * nb + c0 / 32) * 16) = c;
        scales[px * nb + c0 / 32] = (uint8_t)e;
    }
}

int validate(const tdc_norm_shape &s)
{
    if (s.batch < 1 || s.H < 1 || s.W < 1 || s.C < 1 || s.groups < 1 || s.C % s.groups || !(s.eps >= 0.f) || !std::isfinite(s.eps)) return TDC_ERR_BAD_SHAPE;
    if (!tdc_known_dtype(s.dtype) || !tdc_known_act(s.act)) return TDC_ERR_UNSUPPORTED;
    if (s.batch > 65535 || s.C > TDC_NORM_MAX_C || (int64_t)s.H * s.W > 0x7fffffff) return TDC_ERR_UNSUPPORTED;
    return TDC_OK;
}

// Pixels to a chunk: what keeps eight pieces of 16 bytes in flight for every thread of a workgroup, and more where that would
// make over 2048 workgroups (8 to a compute unit).
void choose_chunks(TdcNormDims &d, int dtype)
{
    const int pieces = (d.C * tdc_dtype_bytes(dtype) + 15) / 16;
    const int rows = pieces < TDC_NORM_THREADS ? TDC_NORM_THREADS / pieces : 1;
    const int most = d.B >= 2048 ? 1 : 2048 / d.B;
    const int64_t chunks = std::min<int64_t>(most, (d.P + 8 * rows - 1) / (8 * rows));
    d.chunk_px = (int)((d.P + chunks - 1) / chunks);
    d.chunks = (d.P + d.chunk_px - 1) / d.chunk_px;
}

int64_t pitch_or(int64_t pitch, int C) { return pitch ? pitch : C; }

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
    choose_chunks(p->dims, shape->dtype);
    const size_t pairs = (size_t)p->dims.B * p->dims.chunks * p->dims.C, means = (size_t)p->dims.B * p->dims.G;
    p->ws_bytes = (pairs + means) * sizeof(float2);
    if (hipMalloc((void **)&p->partial, p->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete p;
        return TDC_ERR_ALLOC;
    }
    p->means = p->partial + pairs;
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

int tdc_norm_plan_kernel_count(const tdc_norm_plan *p) { return p ? 2 : 0; }

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
    const dim3 grid(d.chunks, d.B);
    TDC_FOR_DTYPE(dt, T, {
        const T *xt = (const T *)x, *rt = (const T *)a.residual;
        TDC_FOR_VEC(tdc_norm_vec(dt, d.C, {xp}, {x}), T, V, {
            const int nv = d.C / V, rows = nv <= TDC_NORM_THREADS ? TDC_NORM_THREADS / nv : 1;
            tdc_norm_stats<T, V><<<grid, TDC_NORM_THREADS, (size_t)rows * d.C * sizeof(float2), s>>>(d, xt, xp, p->partial);
        });
        const int vec = y ? tdc_norm_vec(dt, d.C, {xp, rt ? rp : 0, yp}, {x, rt, y}) : tdc_norm_vec(dt, d.C, {xp, rt ? rp : 0}, {x, rt});
        TDC_FOR_VEC(vec, T, V, TDC_FOR_ACT(p->shape.act, ACT, {
            if (y) tdc_norm_apply<T, V, ACT><<<grid, TDC_NORM_THREADS, d.G * sizeof(float2), s>>>(d, xt, xp, gamma, beta, rt, rp, (T *)y, yp, p->partial, a.mean, a.rstd);
            else tdc_norm_apply_mx4<T, V, ACT><<<grid, TDC_NORM_THREADS, d.G * sizeof(float2), s>>>(d, xt, xp, gamma, beta, rt, rp, codes, scales, p->partial, a.mean, a.rstd);
        }));
    });
    return hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
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
