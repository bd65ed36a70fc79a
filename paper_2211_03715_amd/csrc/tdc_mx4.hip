// Microscaled 4-bit floating point: quantisation, its inverse, plans and launch dispatch (tdc_mx4.h).
#include <initializer_list>
#include <new>

#include "tdc_mx4_internal.h"

namespace {

// ---- x -> codes and scales: V neighbours to a lane, 16 bytes of x, or one by one where rows do not come in such pieces;
// 32 / V neighbouring lanes to a block.  Four pieces to a thread, 256 threads apart: what a wavefront reads, and writes, at a time
// is whole lines.
template <typename T, int V, bool VECTORS>
__global__ __launch_bounds__(256) void tdc_mx4_quantize_lanes(const T *__restrict__ x, TdcMx4Rows rows, int64_t total, int cols, TdcMx4Div blocks, int64_t pitch,
                                                              uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    constexpr int U = 4, LANES = 32 / V;
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t first = (int64_t)blockIdx.x * (256 * U / LANES) + threadIdx.x / LANES;
    float v[U][V];
    TdcRaw<T, V> in[U];
    int c0[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = min(first + u * (256 / LANES), total - 1), m = blocks.of(i);
        c0[u] = (int)(i - m * blocks.d) * 32 + lane * V;
        const T *p = x + rows.source(m) * pitch + c0[u];
        if constexpr (VECTORS) {
            if (c0[u] < cols) in[u].load(p);                   // V divides cols: all of them or none
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[u][j] = c0[u] + j < cols ? (float)p[j] : 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (VECTORS) {
            const TdcVec<T, V> o = in[u].open();
#pragma unroll
            for (int j = 0; j < V; ++j) v[u][j] = c0[u] < cols ? (float)o.v[j] : 0.f;
        }
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) top = max(top, tdc_abs_bits(v[u][j]));
        const unsigned e = tdc_mx4_scale(tdc_lane_max<LANES>(top));
        const int64_t i = first + u * (256 / LANES);
        if (i >= total) break;
        if constexpr (V == 8) reinterpret_cast<unsigned *>(codes)[i * LANES + lane] = tdc_mx4_codes8(v[u], e);
        else reinterpret_cast<uint16_t *>(codes)[i * LANES + lane] = (uint16_t)tdc_mx4_codes4(v[u], e);
        if (lane == 0) scales[i] = (uint8_t)e;
    }
}

// ---- W[C][N] -> codes and scales of [N][C]: a thread to a block, neighbours along N
__global__ __launch_bounds__(256) void tdc_mx4_pack_weights(const float *__restrict__ W, int C, int N, int nb, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    for (int kb = blockIdx.y; kb < nb; kb += gridDim.y) {
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = 32 * kb + j < C ? W[(size_t)(32 * kb + j) * N + n] : 0.f;
        unsigned e;
        const tdc_i4 c = tdc_mx4_block(v, e);
        *reinterpret_cast<tdc_i4 *>(codes + ((size_t)n * nb + kb) * 16) = c;
        scales[(size_t)n * nb + kb] = (uint8_t)e;
    }
}

// ---- codes and scales -> values, laid over the lanes the same way
template <typename T, int V, bool VECTORS>
__global__ __launch_bounds__(256) void tdc_mx4_dequantize_lanes(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t total, int cols, TdcMx4Div blocks,
                                                                int64_t pitch, T *__restrict__ y)
{
    constexpr int U = 4, LANES = 32 / V;
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t first = (int64_t)blockIdx.x * (256 * U / LANES) + threadIdx.x / LANES;
    unsigned c[U], e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = min(first + u * (256 / LANES), total - 1);
        c[u] = V == 8 ? reinterpret_cast<const unsigned *>(codes)[i * LANES + lane] : reinterpret_cast<const uint16_t *>(codes)[i * LANES + lane];
        e[u] = scales[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = first + u * (256 / LANES), m = blocks.of(i);
        const int c0 = (int)(i - m * blocks.d) * 32 + lane * V;
        if (i >= total) break;
        float v[V];
        tdc_mx4_values(c[u], e[u], v);
        T *out = y + m * pitch + c0;
        if constexpr (VECTORS) {
            if (c0 < cols) tdc_store_stream<T, V>(out, v);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (c0 + j < cols) out[j] = (T)v[j];
        }
    }
}

// Whether rows come in pieces of 16 bytes.
bool row_vectors(int dtype, int64_t cols, int64_t pitch, const void *p)
{
    const int v = 16 / tdc_dtype_bytes(dtype);
    return cols % v == 0 && pitch % v == 0 && tdc_aligned_to(p, 16);
}

// Workgroups of a launch along x, for at most TDC_MX4_MAX_BLOCKS blocks.
unsigned workgroups_for(int64_t blocks, int per_workgroup) { return (unsigned)((blocks + per_workgroup - 1) / per_workgroup); }

hipError_t launch_quantize(hipStream_t s, const void *x, int dtype, const TdcMx4Rows &rows, int64_t n_rows, int cols, int64_t pitch, uint8_t *codes, uint8_t *scales)
{
    const int nb = tdc_mx4_blocks(cols);
    const int64_t total = n_rows * nb;
    const bool vectors = row_vectors(dtype, cols, pitch, x);
    TDC_FOR_DTYPE(dtype, T, {
        constexpr int V = 16 / sizeof(T);
        const unsigned grid = workgroups_for(total, 32 * V);   // 1024 pieces of V
        if (vectors) tdc_mx4_quantize_lanes<T, V, true><<<grid, 256, 0, s>>>((const T *)x, rows, total, cols, TdcMx4Div(nb), pitch, codes, scales);
        else tdc_mx4_quantize_lanes<T, V, false><<<grid, 256, 0, s>>>((const T *)x, rows, total, cols, TdcMx4Div(nb), pitch, codes, scales);
    });
    return hipGetLastError();
}

int check_epilogue(const tdc_mx4_epilogue *e, int dtype)
{
    if (!e) return TDC_OK;
    if (!tdc_known_act(e->act)) return TDC_ERR_UNSUPPORTED;
    if (!tdc_aligned_to(e->bias, 4) || !tdc_aligned_to(e->residual, tdc_dtype_bytes(dtype))) return TDC_ERR_UNSUPPORTED;
    return TDC_OK;
}

TdcMx4Epi kernel_epilogue(const tdc_mx4_epilogue *e)
{
    return e ? TdcMx4Epi{e->bias, e->residual, e->act} : TdcMx4Epi{nullptr, nullptr, TDC_ACT_NONE};
}

}  // namespace

struct tdc_mx4_plan {
    tdc_mx4_shape shape;
    int device;
    int64_t rows;            // output pixels
    TdcMx4Rows map;          // output pixel -> input pixel
    uint8_t *w_codes, *w_scales, *x_codes, *x_scales;   // plain: for large products, and what the others are laid out from
    uint8_t *w_laid, *ws_laid;                          // as tdc_mx4_rows.hip takes them
    bool large, first;                                  // runs as a large product; quantises x in a launch of its own
    bool packed;
    size_t ws_bytes;
};

namespace {

// Rows in 4 bits times the plan's weights.
int multiply(const tdc_mx4_plan *p, hipStream_t s, const uint8_t *codes, const uint8_t *scales, const TdcMx4Rows &rows, void *y, const tdc_mx4_epilogue *epilogue)
{
    const TdcMx4Product q{codes, scales, p->w_codes, p->w_scales, (int)p->rows, p->shape.N, tdc_mx4_blocks(p->shape.C), rows, y, kernel_epilogue(epilogue), false};
    const hipError_t e = p->large ? tdc_launch_mx4_product(q, p->shape.dtype, s) : tdc_launch_mx4_rows(q, TdcMx4Source{nullptr, 0, 0}, p->shape.dtype, p->w_laid, p->ws_laid, s);
    return e == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}

}  // namespace

extern "C" {

int tdc_mx4_quantize(void *hip_stream, const void *x, int dtype, int64_t rows, int64_t cols, int64_t pitch, uint8_t *codes, uint8_t *scales)
{
    if (rows == 0 && cols > 0) return tdc_known_dtype(dtype) ? TDC_OK : TDC_ERR_UNSUPPORTED;
    if (!x || !codes || !scales) return TDC_ERR_NULL;
    if (pitch == 0) pitch = cols;
    if (rows < 0 || cols < 1 || pitch < cols) return TDC_ERR_BAD_SHAPE;
    if (!tdc_known_dtype(dtype) || cols > TDC_MX4_MAX_COLS || !tdc_aligned_to(codes, 16) || !tdc_aligned_to(x, tdc_dtype_bytes(dtype))) return TDC_ERR_UNSUPPORTED;
    if (rows > TDC_MX4_MAX_BLOCKS / tdc_mx4_blocks((int)cols)) return TDC_ERR_UNSUPPORTED;
    return launch_quantize((hipStream_t)hip_stream, x, dtype, TdcMx4Rows::all(), rows, (int)cols, pitch, codes, scales) == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}

int tdc_mx4_dequantize(void *hip_stream, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *y, int dtype, int64_t pitch)
{
    if (rows == 0 && cols > 0) return tdc_known_dtype(dtype) ? TDC_OK : TDC_ERR_UNSUPPORTED;
    if (!y || !codes || !scales) return TDC_ERR_NULL;
    if (pitch == 0) pitch = cols;
    if (rows < 0 || cols < 1 || pitch < cols) return TDC_ERR_BAD_SHAPE;
    if (!tdc_known_dtype(dtype) || cols > TDC_MX4_MAX_COLS || !tdc_aligned_to(codes, 16) || !tdc_aligned_to(y, tdc_dtype_bytes(dtype))) return TDC_ERR_UNSUPPORTED;
    const int nb = tdc_mx4_blocks((int)cols);
    if (rows > TDC_MX4_MAX_BLOCKS / nb) return TDC_ERR_UNSUPPORTED;
    const int64_t total = rows * nb;
    hipStream_t s = (hipStream_t)hip_stream;
    const bool vectors = row_vectors(dtype, cols, pitch, y);
    TDC_FOR_DTYPE(dtype, T, {
        constexpr int V = 16 / sizeof(T);
        const unsigned grid = workgroups_for(total, 32 * V);
        if (vectors) tdc_mx4_dequantize_lanes<T, V, true><<<grid, 256, 0, s>>>(codes, scales, total, (int)cols, TdcMx4Div(nb), pitch, (T *)y);
        else tdc_mx4_dequantize_lanes<T, V, false><<<grid, 256, 0, s>>>(codes, scales, total, (int)cols, TdcMx4Div(nb), pitch, (T *)y);
    });
    return hipGetLastError() == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}

int tdc_mx4_matmul(void *hip_stream, const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes, const uint8_t *b_scales, int32_t M, int32_t N, int32_t K,
                   void *y, int dtype, const tdc_mx4_epilogue *epilogue)
{
    if (M < 0 || N < 1 || K < 1) return TDC_ERR_BAD_SHAPE;
    if (!tdc_known_dtype(dtype)) return TDC_ERR_UNSUPPORTED;
    if (M == 0) return check_epilogue(epilogue, dtype);
    if (!a_codes || !a_scales || !b_codes || !b_scales || !y) return TDC_ERR_NULL;
    const int rc = check_epilogue(epilogue, dtype);
    if (rc != TDC_OK) return rc;
    if (K > TDC_MX4_MAX_COLS || N > TDC_MX4_MAX_OUT || !tdc_aligned_to(a_codes, 16) || !tdc_aligned_to(b_codes, 16) || !tdc_aligned_to(y, tdc_dtype_bytes(dtype))) return TDC_ERR_UNSUPPORTED;
    if (!tdc_mx4_product_fits(M, N)) return TDC_ERR_UNSUPPORTED;
    const TdcMx4Product q{a_codes, a_scales, b_codes, b_scales, M, N, tdc_mx4_blocks(K), TdcMx4Rows::all(), y, kernel_epilogue(epilogue), false};
    return tdc_launch_mx4_product(q, dtype, (hipStream_t)hip_stream) == hipSuccess ? TDC_OK : TDC_ERR_HIP;
}

int tdc_mx4_plan_create(tdc_mx4_plan **out, const tdc_mx4_shape *shape, int device)
{
    if (!out || !shape) return TDC_ERR_NULL;
    *out = nullptr;
    tdc_mx4_shape s = *shape;
    if (s.batch < 1 || s.H < 1 || s.W < 1 || s.C < 1 || s.N < 1 || s.stride < 1) return TDC_ERR_BAD_SHAPE;
    if (s.x_pitch == 0) s.x_pitch = s.C;
    if (s.x_pitch < s.C) return TDC_ERR_BAD_SHAPE;
    const int64_t Ho = (s.H - 1) / s.stride + 1, Wo = (s.W - 1) / s.stride + 1, lim = 0x7fffffff;
    if (!tdc_known_dtype(s.dtype) || s.C > TDC_MX4_MAX_COLS || s.N > TDC_MX4_MAX_OUT) return TDC_ERR_UNSUPPORTED;
    if ((double)s.batch * s.H * s.W > (double)lim) return TDC_ERR_UNSUPPORTED;
    const int64_t rows = s.batch * Ho * Wo;
    if (rows > TDC_MX4_MAX_ROWS || !tdc_mx4_product_fits(rows, s.N) || rows > TDC_MX4_MAX_BLOCKS / tdc_mx4_blocks(s.C)) return TDC_ERR_UNSUPPORTED;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || device < 0 || device >= ndev) return TDC_ERR_HIP;
    DeviceGuard guard(device);
    if (!guard.ok) return TDC_ERR_HIP;
    tdc_mx4_plan *p = new (std::nothrow) tdc_mx4_plan();
    if (!p) return TDC_ERR_ALLOC;
    p->shape = s;
    p->device = device;
    p->rows = rows;
    p->map = s.stride == 1 ? TdcMx4Rows::all() : TdcMx4Rows{s.stride, (int)Wo, (int)(Ho * Wo), s.W, s.H * s.W};
    const size_t nb = tdc_mx4_blocks(s.C);
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    p->large = tdc_mx4_large(rows, s.N, s.C);
    p->first = p->large || tdc_mx4_quantise_first(rows, s.N, s.C, tdc_dtype_bytes(s.dtype));
    const size_t parts[6] = {up(s.N * nb * 16), up(s.N * nb), p->first ? up(rows * nb * 16) : 0, p->first ? up(rows * nb) : 0,
                             p->large ? 0 : tdc_mx4_laid_out_bytes(s.N, (int)nb), p->large ? 0 : tdc_mx4_laid_out_scale_bytes(s.N, (int)nb)};
    for (size_t n : parts) p->ws_bytes += n;
    if (hipMalloc((void **)&p->w_codes, p->ws_bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete p;
        return TDC_ERR_ALLOC;
    }
    p->w_scales = p->w_codes + parts[0];
    p->x_codes = p->w_scales + parts[1];
    p->x_scales = p->x_codes + parts[2];
    p->w_laid = p->x_scales + parts[3];
    p->ws_laid = p->w_laid + parts[4];
    if (!p->large) {
        // whatever a first launch would have to set up, now: a convolution may be the first thing a capturing stream sees
        const TdcMx4Product q{nullptr, nullptr, nullptr, nullptr, (int)rows, s.N, (int)nb, p->map, nullptr, kernel_epilogue(nullptr), false};
        for (int kind = 0; kind < 3; ++kind) {   // x quantised, in pieces of 16 bytes, one value at a time
            const TdcMx4Source src{kind == 0 ? nullptr : (const char *)nullptr + (kind == 1 ? 16 : 2), s.x_pitch, s.C};
            if (tdc_launch_mx4_rows(q, src, s.dtype, p->w_laid, p->ws_laid, nullptr, true) != hipSuccess) {
                (void)hipGetLastError();
                tdc_mx4_plan_destroy(p);
                return TDC_ERR_HIP;
            }
        }
    }
    *out = p;
    return TDC_OK;
}

int tdc_mx4_plan_destroy(tdc_mx4_plan *p)
{
    if (!p) return TDC_OK;
    DeviceGuard guard(p->device);
    const int rc = hipFree(p->w_codes) == hipSuccess ? TDC_OK : TDC_ERR_HIP;
    delete p;
    return rc;
}

size_t tdc_mx4_plan_workspace_bytes(const tdc_mx4_plan *p) { return p ? p->ws_bytes : 0; }

int tdc_mx4_plan_kernel_count(const tdc_mx4_plan *p) { return !p ? 0 : p->first ? 2 : 1; }

int tdc_mx4_plan_pack(tdc_mx4_plan *p, void *hip_stream, const float *W)
{
    if (!p || !W) return TDC_ERR_NULL;
    if (!tdc_aligned_to(W, 4)) return TDC_ERR_UNSUPPORTED;
    DeviceGuard guard(p->device);
    if (!guard.ok) return TDC_ERR_HIP;
    const int C = p->shape.C, N = p->shape.N, nb = tdc_mx4_blocks(C);
    const dim3 grid((N + 255) / 256, nb < 65535 ? nb : 65535);
    tdc_mx4_pack_weights<<<grid, 256, 0, (hipStream_t)hip_stream>>>(W, C, N, nb, p->w_codes, p->w_scales);
    if (hipGetLastError() != hipSuccess) return TDC_ERR_HIP;
    if (!p->large && tdc_launch_mx4_lay_out(p->w_codes, p->w_scales, N, nb, p->w_laid, p->ws_laid, (hipStream_t)hip_stream) != hipSuccess) return TDC_ERR_HIP;
    p->packed = true;
    return TDC_OK;
}

int tdc_conv_mx4(tdc_mx4_plan *p, void *hip_stream, const void *x, void *y, const tdc_mx4_epilogue *epilogue)
{
    if (!p || !p->packed || !x || !y) return TDC_ERR_NULL;
    const tdc_mx4_shape &s = p->shape;
    const int rc = check_epilogue(epilogue, s.dtype);
    if (rc != TDC_OK) return rc;
    if (!tdc_aligned_to(x, tdc_dtype_bytes(s.dtype)) || !tdc_aligned_to(y, tdc_dtype_bytes(s.dtype))) return TDC_ERR_UNSUPPORTED;
    DeviceGuard guard(p->device);
    if (!guard.ok) return TDC_ERR_HIP;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!p->first) {
        const TdcMx4Product q{nullptr, nullptr, nullptr, nullptr, (int)p->rows, s.N, tdc_mx4_blocks(s.C), p->map, y, kernel_epilogue(epilogue), false};
        return tdc_launch_mx4_rows(q, TdcMx4Source{x, s.x_pitch, s.C}, s.dtype, p->w_laid, p->ws_laid, st) == hipSuccess ? TDC_OK : TDC_ERR_HIP;
    }
    if (launch_quantize(st, x, s.dtype, p->map, p->rows, s.C, s.x_pitch, p->x_codes, p->x_scales) != hipSuccess) return TDC_ERR_HIP;
    return multiply(p, st, p->x_codes, p->x_scales, TdcMx4Rows::all(), y, epilogue);
}

int tdc_conv_mx4_quantized(tdc_mx4_plan *p, void *hip_stream, const uint8_t *codes, const uint8_t *scales, void *y, const tdc_mx4_epilogue *epilogue)
{
    if (!p || !p->packed || !codes || !scales || !y) return TDC_ERR_NULL;
    const tdc_mx4_shape &s = p->shape;
    const int rc = check_epilogue(epilogue, s.dtype);
    if (rc != TDC_OK) return rc;
    if (!tdc_aligned_to(codes, 16) || !tdc_aligned_to(y, tdc_dtype_bytes(s.dtype))) return TDC_ERR_UNSUPPORTED;
    DeviceGuard guard(p->device);
    if (!guard.ok) return TDC_ERR_HIP;
    return multiply(p, (hipStream_t)hip_stream, codes, scales, p->map, y, epilogue);
}

}  // extern "C"
