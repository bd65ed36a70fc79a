// Products with one operand kept whole in LDS (tdc_mx4.h): 1x1 convolutions, which are bound by reading x and writing y, and
// products of few rows, which are bound by reading the weights and by latency.
//
// A workgroup takes 32 rows.  It quantises them on the way into LDS (or takes them quantised), all of k where that fits, and
// multiplies them with 64 columns of weights at a time: x is read once, y written once, in one launch; the weights come from the
// L2.  KW = 1: its four wavefronts take columns in turn.  KW = 8: eight wavefronts share the k of the same 64 columns and add up
// through LDS, so that few rows still keep many wavefronts reading weights.
//
// Weights of a plan are laid out as the matrix instruction takes them: for every 64 columns and every 64 values of k 2 KiB, first
// those of the even columns, then those of the odd ones, 16 bytes to a lane; and for every 256 values of k a dword of four scale
// bytes to a lane.  A lane's two results of a row are neighbours then, and rows of them whole lines.  PLAIN: rows of the format
// itself, for products whose second operand is not a plan's.
//
// In LDS the rows lie the same way: a fragment is one run of 1 KiB.
#include <algorithm>

#include "tdc_div.h"
#include "tdc_mx4_tile.h"

namespace {

enum { SRC_VECTORS = 0, SRC_VALUES = 1, SRC_CODES = 2 };   // x in pieces of 16 bytes, one by one, quantised

struct RowsArgs {
    TdcMx4Product q;
    const void *x;
    int64_t pitch;
    int cols;                // values of a row of x
    const uint8_t *w, *ws;   // laid-out weights and scales
    int groups, splits;      // columns by 64; workgroups that share them
    int quads, chunk;        // k by 256; how many of them are in LDS at a time
    TdcDiv blocks;           // by the blocks of a full chunk
    bool pairs;              // y and the residual can be accessed two values at a time
};

constexpr int QUAD_BLOCKS = 8;    // blocks to 256 values
constexpr size_t per_quad = 4096 + 256;   // their codes and scales, 32 rows
constexpr int PITCH = 64 + 8;     // floats to a row of sums: the halves of a wavefront, four rows apart, on different banks

// Eight values of a row of x, zeros past its end.  Those of 16 bits stay one piece until they are needed: 14x14x1024 -> 512 in
// bf16, 256 images: 60.6 us where they were made fp32 at once, 44.7 so; 56x56x64 -> 256, 32 images: 24.2 and 19.6.
template <typename T, int SRC> struct Eight {
    static constexpr bool WHOLE = SRC == SRC_VECTORS && sizeof(T) == 2;
    TdcRaw<T, 16 / sizeof(T)> w;
    float f[8];
    __device__ __forceinline__ void load(const T *row, int c0, int cols)
    {
        if constexpr (WHOLE) {
            if (c0 < cols) w.load(row + c0);      // cols is a multiple of 8
        } else if constexpr (SRC == SRC_VECTORS) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                TdcVec<T, 4> in;
                if (c0 < cols) in = tdc_load<T, 4>(row + c0 + j);
#pragma unroll
                for (int u = 0; u < 4; ++u) f[j + u] = c0 < cols ? (float)in.v[u] : 0.f;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = c0 + j < cols ? (float)row[c0 + j] : 0.f;
        }
    }
    __device__ __forceinline__ void open(int c0, int cols)
    {
        if constexpr (WHOLE) {
            const TdcVec<T, 8> in = w.open();
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = c0 < cols ? (float)in.v[j] : 0.f;
        }
    }
};

// The epilogue of a lane's columns n and n + 1: sums s of E rows, row(e) + 4 h from m0 on.  row(e) is the same for all lanes, so
// that a row's address is a scalar one, and the lane adds the same 32-bit offset to all of them.  What is read for some rows is
// read before any of them is stored: a store might change it, for all the compiler knows.
template <typename T, int E, typename Row> __device__ __forceinline__ void finish_columns(const RowsArgs &a, int m0, int rows, int n, int h, Row row, float (&s)[E][2])
{
    if (n >= a.q.N) return;
    const bool two = n + 1 < a.q.N;
    const unsigned lane = ((unsigned)(4 * h) * a.q.N + n) * sizeof(T);   // N <= TDC_MX4_MAX_OUT
    if (a.q.epi.bias) {
        const float b0 = a.q.epi.bias[n], b1 = two ? a.q.epi.bias[n + 1] : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s[e][0] += b0;
            s[e][1] += b1;
        }
    }
    if (a.q.epi.residual) {
        float r[E][2];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (row(e) + 4 * h >= rows) continue;
            const T *p = reinterpret_cast<const T *>(static_cast<const char *>(a.q.epi.residual) + (size_t)(m0 + row(e)) * a.q.N * sizeof(T) + lane);
            if (a.pairs) {
                const TdcVec<T, 2> v = tdc_load<T, 2>(p);
                r[e][0] = (float)v.v[0];
                r[e][1] = (float)v.v[1];
            } else {
                r[e][0] = (float)p[0];
                r[e][1] = two ? (float)p[1] : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (row(e) + 4 * h < rows) {
                s[e][0] += r[e][0];
                s[e][1] += r[e][1];
            }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) tdc_activate_all(a.q.epi.act, s[e]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (row(e) + 4 * h >= rows) continue;
        T *p = reinterpret_cast<T *>(static_cast<char *>(a.q.y) + (size_t)(m0 + row(e)) * a.q.N * sizeof(T) + lane);
        if (a.pairs) {
            tdc_store<T, 2>(p, s[e]);
        } else {
            p[0] = (T)s[e][0];
            if (two) p[1] = (T)s[e][1];
        }
    }
}

template <typename T, int SRC, int KW, bool PLAIN>
__global__ __launch_bounds__(KW == 1 ? 256 : 512, 4) void tdc_mx4_rows(RowsArgs a)
{
    constexpr int THREADS = KW == 1 ? 256 : 512, ROWS = 32;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    // codes [4 chunk][64 lanes][16], scales [chunk][64 lanes][4]
    uint8_t *const codes = lds, *const scales = lds + (size_t)a.chunk * 4096;
    const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = l & 31, h = l >> 5;
    const int tile = blockIdx.x / a.splits, split = blockIdx.x - tile * a.splits, m0 = tile * ROWS, rows = min(ROWS, a.q.M - m0);

    auto stage = [&](int quad0) {
        const int quads = min(a.chunk, a.quads - quad0), blocks = quads * QUAD_BLOCKS, per = SRC == SRC_CODES ? 1 : 4, total = rows * blocks * per;
        constexpr int U = 4;
        for (int i0 = tid; i0 < total; i0 += THREADS * U) {
            Eight<T, SRC> in[U];
            tdc_i4 c[U];
            unsigned sc[U];
            int row[U], kb[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = min(i0 + u * THREADS, total - 1) / per;    // per is 1 or 4
                // all chunks but the last have the same number of blocks; the last is divided the long way
                row[u] = quads == a.chunk ? (int)tdc_div_from_hi(i, __umulhi(a.blocks.m, i), a.blocks) : i / blocks;
                kb[u] = i - row[u] * blocks;
                const int k = quad0 * QUAD_BLOCKS + kb[u];
                const int64_t src = a.q.a_rows.source(m0 + row[u]);
                if constexpr (SRC == SRC_CODES) {
                    const size_t at = (size_t)src * a.q.nb + min(k, a.q.nb - 1);
                    c[u] = *reinterpret_cast<const tdc_i4 *>(a.q.a_codes + at * 16);
                    sc[u] = k < a.q.nb ? a.q.a_scales[at] : 0u;
                } else {
                    in[u].load(static_cast<const T *>(a.x) + src * a.pitch, k * 32 + (tid & 3) * 8, a.cols);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if constexpr (SRC != SRC_CODES) {
                    in[u].open((quad0 * QUAD_BLOCKS + kb[u]) * 32 + (tid & 3) * 8, a.cols);
                    unsigned top = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = max(top, tdc_abs_bits(in[u].f[j]));
                    sc[u] = tdc_mx4_scale(tdc_lane_max<4>(top));         // four neighbouring lanes have a block
                }
                if (i0 + u * THREADS >= total) break;
                const int s = kb[u] >> 1, lane = (kb[u] & 1) * 32 + row[u];
                uint8_t *to = codes + s * 1024 + lane * 16, *sto = scales + (s >> 2) * 256 + lane * 4 + (s & 3);
                if constexpr (SRC == SRC_CODES) {
                    *reinterpret_cast<tdc_i4 *>(to) = c[u];
                    *sto = (uint8_t)sc[u];
                } else {
                    *reinterpret_cast<unsigned *>(to + (tid & 3) * 4) = tdc_mx4_codes8(in[u].f, sc[u]);
                    if ((tid & 3) == 0) *sto = (uint8_t)sc[u];
                }
            }
        }
    };

    // 256 values of k of columns 64 p ..: the weights of quad t, and their product with what lies at quad `at` in LDS
    tdc_i4 b[4][2];
    unsigned sb[2];
    auto load = [&](int p, int t) {
        if constexpr (PLAIN) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const size_t row = (size_t)min(64 * p + 2 * r32 + j, a.q.N - 1) * a.q.nb;
                sb[j] = 0;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int k = 8 * t + 2 * s + h;
                    const size_t src = row + min(k, a.q.nb - 1);
                    b[s][j] = *reinterpret_cast<const tdc_i4 *>(a.q.b_codes + src * 16);
                    sb[j] |= k < a.q.nb ? (unsigned)a.q.b_scales[src] << (8 * s) : 0u;
                }
            }
        } else {
            const uint8_t *w = a.w + ((size_t)p * a.quads + t) * 8192 + l * 16;
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j) b[s][j] = *reinterpret_cast<const tdc_i4 *>(w + (2 * s + j) * 1024);
            const uint2 v = *reinterpret_cast<const uint2 *>(a.ws + ((size_t)p * a.quads + t) * 512 + l * 8);
            sb[0] = v.x;
            sb[1] = v.y;
        }
    };
    auto multiply = [&](int at, tdc_f16v (&acc)[2]) {
        const unsigned sa = *reinterpret_cast<const unsigned *>(scales + at * 256 + l * 4);
        tdc_i4 x[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] = *reinterpret_cast<const tdc_i4 *>(codes + (4 * at + s) * 1024 + l * 16);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            acc[j] = tdc_mx4_mfma<0>(x[0], sa, b[0][j], sb[j], acc[j]);
            acc[j] = tdc_mx4_mfma<1>(x[1], sa, b[1][j], sb[j], acc[j]);
            acc[j] = tdc_mx4_mfma<2>(x[2], sa, b[2][j], sb[j], acc[j]);
            acc[j] = tdc_mx4_mfma<3>(x[3], sa, b[3][j], sb[j], acc[j]);
        }
    };

    const int first = (int)((int64_t)a.groups * split / a.splits), end = (int)((int64_t)a.groups * (split + 1) / a.splits);
    const bool once = a.chunk >= a.quads;
    if (once) {
        stage(0);
        __syncthreads();
    }
    for (int p0 = first; p0 < end; p0 += KW == 1 ? 4 : 1) {   // the same trip count for every wavefront
        const int p = KW == 1 ? p0 + wave : p0;
        const bool mine = p < end;
        tdc_f16v acc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
        for (int quad0 = 0; quad0 < a.quads; quad0 += a.chunk) {
            if (!once) {
                __syncthreads();
                stage(quad0);
                __syncthreads();
            }
            const int quads = min(a.chunk, a.quads - quad0);
            // No fetch ahead: the registers for it cost a wavefront in four, which hides more (56x56x256 -> 512, every second pixel,
            // 32 images: 19.3 us without, 23.5 with).
            if (mine)
                for (int t = KW == 1 ? 0 : wave; t < quads; t += KW) {
                    load(p, quad0 + t);
                    multiply(t, acc);
                }
        }
        if constexpr (KW == 1) {
            // 16 rows at a time through a piece of LDS of the wavefront's own, so that stores are whole lines of 16 bytes a lane
            float *sums = reinterpret_cast<float *>(lds + (size_t)a.chunk * per_quad) + wave * 16 * PITCH;
            if (mine) {
#pragma unroll
                for (int e0 = 0; e0 < 16; e0 += 8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        *reinterpret_cast<float2 *>(sums + (8 * (e / 4) + 4 * h + e % 4) * PITCH + 2 * r32) = make_float2(acc[0][e0 + e], acc[1][e0 + e]);
                    __builtin_amdgcn_wave_barrier();
                    tdc_mx4_store_rows<T>(a.q, sums, PITCH, 16, 64, m0 + 2 * e0, 64 * p, l);
                    __builtin_amdgcn_wave_barrier();
                }
            }
        } else {
            // every wavefront's sums through LDS; wavefront w finishes registers 2w and 2w + 1
            float *sums = reinterpret_cast<float *>(lds);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) sums[((wave * 2 + j) * 16 + e) * 64 + l] = acc[j][e];
            __syncthreads();
            float v[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    v[u][j] = 0.f;
#pragma unroll
                    for (int w = 0; w < KW; ++w) v[u][j] += sums[((w * 2 + j) * 16 + 2 * wave + u) * 64 + l];
                }
            finish_columns<T, 2>(a, m0, rows, 64 * p + 2 * r32, h, [&](int u) { return 8 * ((2 * wave + u) / 4) + (2 * wave + u) % 4; }, v);
        }
    }
}

template <typename T, int SRC, int KW, bool PLAIN> hipError_t launch(const RowsArgs &a, unsigned wgs, size_t lds, hipStream_t s, bool prepare_only)
{
    const void *fn = (const void *)&tdc_mx4_rows<T, SRC, KW, PLAIN>;
    const hipError_t e = tdc_allow_lds(fn, lds);
    if (e != hipSuccess || prepare_only) return e;
    tdc_mx4_rows<T, SRC, KW, PLAIN><<<wgs, KW == 1 ? 256 : 512, lds, s>>>(a);
    return hipGetLastError();
}

// ---- plain weights -> laid out: a thread to a lane of a fragment
__global__ __launch_bounds__(256) void tdc_mx4_lay_out(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int N, int nb, int quads, int64_t total, uint8_t *__restrict__ w,
                                                       uint8_t *__restrict__ ws)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;    // [p][quad][s][j][lane]
    if (i >= total) return;
    const int l = (int)(i & 63), j = (int)(i >> 6) & 1, s = (int)(i >> 7) & 3;
    const int64_t pt = i >> 9, p = pt / quads;
    const int t = (int)(pt - p * quads), n = (int)p * 64 + 2 * (l & 31) + j, k = 8 * t + 2 * s + (l >> 5);
    const bool there = n < N && k < nb;
    const size_t at = (size_t)n * nb + k;
    *reinterpret_cast<tdc_i4 *>(w + i * 16) = there ? *reinterpret_cast<const tdc_i4 *>(codes + at * 16) : (tdc_i4){0, 0, 0, 0};
    ws[pt * 512 + l * 8 + j * 4 + s] = there ? scales[at] : (uint8_t)0;
}

int quads_of(int nb) { return (nb + QUAD_BLOCKS - 1) / QUAD_BLOCKS; }
int groups_of(int N) { return (N + 63) / 64; }

}  // namespace

size_t tdc_mx4_laid_out_bytes(int N, int nb) { return (size_t)groups_of(N) * quads_of(nb) * 8192; }
size_t tdc_mx4_laid_out_scale_bytes(int N, int nb) { return (size_t)groups_of(N) * quads_of(nb) * 512; }

hipError_t tdc_launch_mx4_lay_out(const uint8_t *codes, const uint8_t *scales, int N, int nb, uint8_t *w, uint8_t *ws, hipStream_t s)
{
    const int64_t total = (int64_t)groups_of(N) * quads_of(nb) * 512;
    tdc_mx4_lay_out<<<(unsigned)((total + 255) / 256), 256, 0, s>>>(codes, scales, N, nb, quads_of(nb), total, w, ws);
    return hipGetLastError();
}

hipError_t tdc_launch_mx4_rows(const TdcMx4Product &q, const TdcMx4Source &src, int dtype, const uint8_t *w, const uint8_t *ws, hipStream_t s, bool prepare_only)
{
    RowsArgs a{};
    a.q = q;
    a.x = src.x;
    a.pitch = src.pitch;
    a.cols = src.cols;
    a.w = w;
    a.ws = ws;
    a.groups = groups_of(q.N);
    a.quads = quads_of(q.nb);
    const int size = tdc_dtype_bytes(dtype);
    a.q.vec = tdc_mx4_vec(q, dtype);
    a.pairs = q.N % 2 == 0 && tdc_aligned_to(q.y, 2 * size) && tdc_aligned_to(q.epi.residual, 2 * size);
    const int64_t tiles = ((int64_t)q.M + 31) / 32;
    // Few tiles: a workgroup to 32 rows and 64 columns, eight wavefronts along k.  Many: the columns in turn, shared by as many
    // workgroups as it takes to have four to a compute unit.
    const bool few = tdc_mx4_few(q.M, q.N) || !w;
    a.splits = few ? a.groups : (int)std::max<int64_t>(1, std::min<int64_t>((a.groups + 3) / 4, 1024 / tiles));
    // besides, KW = 1 stores through 18 KiB, KW = 8 adds up in 64 KiB where the codes were
    a.chunk = (int)std::min<size_t>(a.quads, 139264 / per_quad);
    a.blocks = tdc_make_div(a.chunk * QUAD_BLOCKS);
    const size_t lds = few ? std::max<size_t>(a.chunk * per_quad, 65536) : a.chunk * per_quad + 4 * 16 * PITCH * sizeof(float);
    const unsigned wgs = (unsigned)(tiles * a.splits);
    const bool vectors = src.x && src.cols % 8 == 0 && tdc_aligned_to(src.x, 16) && src.pitch * size % 16 == 0;
    hipError_t e = hipErrorInvalidValue;
    TDC_FOR_DTYPE(dtype, T, {
        if (!w) e = launch<T, SRC_CODES, 8, true>(a, wgs, lds, s, prepare_only);
        else if (few) {
            if (!src.x) e = launch<T, SRC_CODES, 8, false>(a, wgs, lds, s, prepare_only);
            else if (vectors) e = launch<T, SRC_VECTORS, 8, false>(a, wgs, lds, s, prepare_only);
            else e = launch<T, SRC_VALUES, 8, false>(a, wgs, lds, s, prepare_only);
        } else {
            if (!src.x) e = launch<T, SRC_CODES, 1, false>(a, wgs, lds, s, prepare_only);
            else if (vectors) e = launch<T, SRC_VECTORS, 1, false>(a, wgs, lds, s, prepare_only);
            else e = launch<T, SRC_VALUES, 1, false>(a, wgs, lds, s, prepare_only);
        }
    });
    return e;
}
