// Products in tiles through LDS, for operands with many rows on both sides (tdc_mx4_product.hip).
//
// GM x GN wavefronts share a tile; each computes WM x WN blocks of 32 x 32.  A step takes 256 values of k, 128 bytes of codes to
// a row: a wavefront's fetch covers eight rows of one cache line each, straight from memory to LDS.  In LDS a row keeps its
// eight blocks of 16 bytes in the order (block ^ row/2 % 8), so that sixteen neighbouring rows fall on all 64 banks.  The next
// step's codes go to the other of two buffers while this step multiplies: one barrier to a step.
//
// Scales are a byte to 16 bytes of codes but as many cache lines as there are rows, and the L1 takes a cycle for each line:
// 8 bytes to a row and step, they would take half as long as the codes.  Where the rows' scales are whole pieces of 16 bytes
// (PACKED) they are fetched for four steps at once, two lanes to a row, and read from LDS for two.
//
// Per matrix instruction (32 cycles for 131 kFLOP) a wavefront reads (WM + WN) / (WM WN) KiB from LDS: 3/4 KiB at 4 x 2, with
// four such streams at a time three quarters of LDS's 128 bytes a cycle.
//
// Blocks of k past the end exist only where PACKED is false: the fetch reads the last block again, and both scales are zero
// bytes, 2^-127 each, so that what comes of them, below 2^-243, is lost in any fp32 sum.
#ifndef TDC_MX4_TILE_H
#define TDC_MX4_TILE_H

#include <type_traits>

#include "tdc_mx4_internal.h"

typedef float tdc_f16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ tdc_i8 tdc_mx4_widen(tdc_i4 a) { return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1); }

// OP: which byte of the scale registers counts.
template <int OP> __device__ __forceinline__ tdc_f16v tdc_mx4_mfma(tdc_i4 a, unsigned sa, tdc_i4 b, unsigned sb, tdc_f16v c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(tdc_mx4_widen(a), tdc_mx4_widen(b), c, 4, 4, OP, (int)sa, OP, (int)sb);
}

// V sums of row m, from column n on, into y, which has rows of whole V's and is read and written by V's where V > 1.
template <typename T, int V> __device__ __forceinline__ void tdc_mx4_finish(const TdcMx4Product &q, float (&v)[V], int m, int n)
{
    const size_t at = (size_t)m * q.N + n;
    if (q.epi.bias) {
        constexpr int W = V < 4 ? V : 4;
#pragma unroll
        for (int i = 0; i < V; i += W) {
            const TdcVec<float, W> b = tdc_load<float, W>(q.epi.bias + n + i);
#pragma unroll
            for (int u = 0; u < W; ++u) v[i + u] += b.v[u];
        }
    }
    if (q.epi.residual) {
        const TdcVec<T, V> r = tdc_load<T, V>(static_cast<const T *>(q.epi.residual) + at);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += (float)r.v[i];
    }
    if (q.epi.act == TDC_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = tdc_activate<TDC_ACT_RELU>(v[i]);
    } else if (q.epi.act == TDC_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = tdc_activate<TDC_ACT_SILU>(v[i]);
    }
    // y is not read again; 32 images, with ordinary stores and so: 56x56x256 -> 512 of every second pixel in fp32 17.6 and 16.8 us,
    // 56x56x64 -> 256 32.5 and 25.0, 28x28x128 -> 512 in bf16 12.3 and 10.2
    tdc_store_stream<T, V>(static_cast<T *>(q.y) + at, v);
}

// `rows` x `cols` sums that a wavefront holds in LDS, `pitch` floats to a row, into y from (m0, n0) on.
template <typename T> __device__ __forceinline__ void tdc_mx4_store_rows(const TdcMx4Product &q, const float *sums, int pitch, int rows, int cols, int m0, int n0, int lane)
{
    constexpr int V = 16 / sizeof(T);
    if (q.vec) {
        const int per = cols / V;
        for (int i = lane; i < rows * per; i += 64) {
            const int r = i / per, c = (i - r * per) * V;
            if (m0 + r < q.M && n0 + c < q.N) {
                float v[V];
#pragma unroll
                for (int u = 0; u < V; u += 4) *reinterpret_cast<float4 *>(v + u) = *reinterpret_cast<const float4 *>(sums + r * pitch + c + u);
                tdc_mx4_finish<T, V>(q, v, m0 + r, n0 + c);
            }
        }
    } else {
        for (int i = lane; i < rows * cols; i += 64) {
            const int r = i / cols, c = i - r * cols;
            if (m0 + r < q.M && n0 + c < q.N) {
                float v[1] = {sums[r * pitch + c]};
                tdc_mx4_finish<T, 1>(q, v, m0 + r, n0 + c);
            }
        }
    }
}

// The eight scale bytes of blocks k .. k+7 of a row, zeros past the end.
__device__ __forceinline__ uint2 tdc_mx4_scales8(const uint8_t *row, int k, int nb)
{
    uint2 v = make_uint2(0u, 0u);
    if (k + 8 <= nb) {
        __builtin_memcpy(&v, row + k, 8);
    } else {
        for (int i = 0; i < 4 && k + i < nb; ++i) v.x |= (unsigned)row[k + i] << (8 * i);
        for (int i = 0; i < 4 && k + 4 + i < nb; ++i) v.y |= (unsigned)row[k + 4 + i] << (8 * i);
    }
    return v;
}

// Tile number t of mt x nt in an order that keeps neighbours together: the workgroups that one XCD runs at a time (ids 8 apart)
// work on eight rows of tiles and a few columns, and read these operands from memory once.
__device__ __forceinline__ void tdc_mx4_tile_at(int id, int mt, int nt, int &m, int &n)
{
    const int total = mt * nt, per = total / 8, extra = total % 8, xcd = id % 8;
    const int t = xcd * per + (xcd < extra ? xcd : extra) + id / 8;
    const int group = t / (8 * nt), first = group * 8, rows = mt - first < 8 ? mt - first : 8, r = t - group * 8 * nt;
    m = first + r % rows;
    n = r / rows;
}

// A wavefront's 64 lanes fetch 16 bytes each from where they point into 1 KiB of LDS, lane after lane, past the registers.
__device__ __forceinline__ void tdc_mx4_fetch(const uint8_t *from, uint8_t *lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
}

template <typename T, int WM, int WN, int GM, int GN, bool PACKED>
__global__ __launch_bounds__(64 * GM * GN, 2) void tdc_mx4_product_tile(TdcMx4Product q)
{
    constexpr int BM = 32 * WM * GM, BN = 32 * WN * GN, ROWS = BM + BN, THREADS = 64 * GM * GN, WAVES = GM * GN;
    // separate objects: a read of one buffer then visibly does not depend on what is being fetched into the other
    __shared__ __attribute__((aligned(1024))) uint8_t codes0[ROWS * 128], codes1[ROWS * 128];
    __shared__ __attribute__((aligned(1024))) uint8_t scales[2][ROWS * (PACKED ? 32 : 8)];
    const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tm, tn;
    tdc_mx4_tile_at(blockIdx.x, (q.M + BM - 1) / BM, (q.N + BN - 1) / BN, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, steps = (q.nb + 7) / 8;
    auto row_of = [&](int r) { return r < BM ? (size_t)q.a_rows.source(min(m0 + r, q.M - 1)) : (size_t)min(n0 + r - BM, q.N - 1); };

    // codes: rows tid/8 + STEP i of both operands, the block that belongs at place tid%8 of the eight
    constexpr int STEP = THREADS / 8, F = ROWS / STEP;
    static_assert(BM % STEP == 0 && BN % STEP == 0 && STEP % 16 == 0, "every thread fetches the same share");
    const int fr = tid >> 3, fk = (tid & 7) ^ ((fr >> 1) & 7);
    const uint8_t *src[F];
#pragma unroll
    for (int i = 0; i < F; ++i) src[i] = (STEP * i < BM ? q.a_codes : q.b_codes) + row_of(fr + STEP * i) * q.nb * 16;
    auto fetch = [&](int t, uint8_t *codes) {
        const size_t at = (size_t)(PACKED ? 8 * t + fk : min(8 * t + fk, q.nb - 1)) * 16;
#pragma unroll
        for (int i = 0; i < F; ++i) tdc_mx4_fetch(src[i] + at, codes + (i * STEP + 8 * wave) * 128);
    };

    // scales, PACKED: rows 32 wave + l/2 + 32 WAVES i, 16 bytes to a lane; of the two pieces the second comes first in eight of sixteen
    // rows.  Otherwise: rows tid + THREADS i, eight bytes through a register.
    constexpr int SR = PACKED ? ROWS / (32 * WAVES) : ROWS / THREADS;
    const uint8_t *ssrc[SR];
    uint2 sin[PACKED ? 1 : SR];
    const int sr = 32 * wave + (l >> 1), sk = (l & 1) ^ ((l >> 4) & 1);
#pragma unroll
    for (int i = 0; i < SR; ++i) {
        const int r = PACKED ? sr + 32 * WAVES * i : tid + THREADS * i;
        ssrc[i] = (r < BM ? q.a_scales : q.b_scales) + row_of(r) * q.nb;
    }
    auto fetch_scales = [&](int chunk) {    // PACKED: of steps 4 chunk .. 4 chunk + 3, whose second half may be past the end
        const int at = min(2 * chunk + sk, q.nb / 16 - 1) * 16;
#pragma unroll
        for (int i = 0; i < SR; ++i) tdc_mx4_fetch(ssrc[i] + at, &scales[chunk & 1][32 * (32 * wave + 32 * WAVES * i)]);
    };
    auto load_scales = [&](int t) {         // otherwise: of step t
#pragma unroll
        for (int i = 0; i < SR && !PACKED; ++i) sin[i] = tdc_mx4_scales8(ssrc[i], 8 * t, q.nb);
    };
    // what was fetched is there for every wavefront
    auto arrive = [&](int t) {
#pragma unroll
        for (int i = 0; i < SR && !PACKED; ++i) *reinterpret_cast<uint2 *>(&scales[t & 1][8 * (tid + THREADS * i)]) = sin[i];
        __builtin_amdgcn_s_waitcnt(0x0070);    // vmcnt(0), lgkmcnt(0)
        __syncthreads();
    };

    const int r32 = l & 31, h = l >> 5, wm = (wave / GN) * 32 * WM, wn = (wave % GN) * 32 * WN;
    tdc_f16v acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // Scales of two steps (PACKED) or of one in registers, shifted so that bytes 0 and 2 are those of the lane's blocks.
    constexpr int SW = PACKED ? 4 : 2;
    unsigned sa[WM][SW], sb[WN][SW];
    auto read_scales = [&](int t) {
        auto read = [&](int r, unsigned (&s)[SW]) {
            if constexpr (PACKED) {
                const uint4 v = *reinterpret_cast<const uint4 *>(&scales[(t >> 2) & 1][32 * r + 16 * (((t >> 1) & 1) ^ ((r32 >> 3) & 1))]);
                s[0] = v.x >> (8 * h), s[1] = v.y >> (8 * h), s[2] = v.z >> (8 * h), s[3] = v.w >> (8 * h);
            } else {
                const uint2 v = *reinterpret_cast<const uint2 *>(&scales[t & 1][8 * r]);
                s[0] = v.x >> (8 * h), s[1] = v.y >> (8 * h);
            }
        };
#pragma unroll
        for (int i = 0; i < WM; ++i) read(wm + 32 * i + r32, sa[i]);
#pragma unroll
        for (int j = 0; j < WN; ++j) read(BM + wn + 32 * j + r32, sb[j]);
    };
    auto multiply = [&](const uint8_t *codes, auto second) {
        constexpr int W = decltype(second)::value && PACKED ? 2 : 0;
        const uint8_t *pa = codes + (wm + r32) * 128, *pb = codes + (BM + wn + r32) * 128;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = ((2 * s + h) ^ ((r32 >> 1) & 7)) << 4;
            tdc_i4 a[WM], b[WN];
#pragma unroll
            for (int i = 0; i < WM; ++i) a[i] = *reinterpret_cast<const tdc_i4 *>(pa + i * 32 * 128 + at);
#pragma unroll
            for (int j = 0; j < WN; ++j) b[j] = *reinterpret_cast<const tdc_i4 *>(pb + j * 32 * 128 + at);
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int j = 0; j < WN; ++j)
                    acc[i][j] = s & 1 ? tdc_mx4_mfma<2>(a[i], sa[i][W + s / 2], b[j], sb[j][W + s / 2], acc[i][j]) : tdc_mx4_mfma<0>(a[i], sa[i][W + s / 2], b[j], sb[j][W + s / 2], acc[i][j]);
        }
    };

    fetch(0, codes0);
    if constexpr (PACKED) fetch_scales(0);
    else load_scales(0);
    arrive(0);
    for (int t = 0;; t += 2) {
        // scales first: what is fetched into their array from here on must not be waited for by their reads
        read_scales(t);
        if (t + 1 < steps) {
            fetch(t + 1, codes1);
            if constexpr (!PACKED) load_scales(t + 1);
            else if ((t & 3) == 0 && t + 4 < steps) fetch_scales(t / 4 + 1);
        }
        multiply(codes0, std::false_type());
        if (t + 1 >= steps) break;
        arrive(t + 1);
        if constexpr (!PACKED) read_scales(t + 1);
        if (t + 2 < steps) {
            fetch(t + 2, codes0);
            if constexpr (!PACKED) load_scales(t + 2);
        }
        multiply(codes1, std::true_type());
        if (t + 2 >= steps) break;
        arrive(t + 2);
    }

    // 32 rows at a time through a piece of LDS of the wavefront's own, so that stores are rows of whole lines.  A pitch of 8 more
    // than a multiple of 32 keeps the two halves of a wavefront, four rows apart, on different banks.
    constexpr int COLS = 32 * WN, PITCH = COLS + 8;
    static_assert(GM * GN / 2 * 32 * PITCH * sizeof(float) <= sizeof(codes0), "the sums fit where the codes were");
    float *sums = reinterpret_cast<float *>(wave & 1 ? codes1 : codes0) + wave / 2 * 32 * PITCH;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WM; ++i) {
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[(8 * (e / 4) + 4 * h + e % 4) * PITCH + 32 * j + r32] = acc[i][j][e];
        __builtin_amdgcn_wave_barrier();
        tdc_mx4_store_rows<T>(q, sums, PITCH, 32, COLS, m0 + wm + 32 * i, n0 + wn, l);
        __builtin_amdgcn_wave_barrier();
    }
}

#endif  // TDC_MX4_TILE_H
