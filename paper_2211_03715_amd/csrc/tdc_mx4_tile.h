// Products in tiles through LDS, for operands with many rows on both sides (tdc_mx4_product.hip).
//
// Four wavefronts, two by two, share a tile of 64 WM x 64 WN outputs; each computes WM x WN blocks of 32 x 32.  A step takes 256
// values of k, 128 bytes of codes to a row: a wavefront's fetch covers eight rows of one cache line each.  In LDS a row keeps
// its 128 bytes, its eight blocks of 16 bytes in the order (block ^ row % 8), so that the eight rows that one pass of a 16-byte
// read covers fall on different banks.  The next step's codes go straight to the other of two buffers while this step
// multiplies, its scales through a register: one barrier to a step.
//
// Per matrix instruction (32 cycles for 64 kFLOP) a wavefront reads (WM + WN) / (WM WN) KiB from LDS, 0.5 KiB at 4 x 4: four
// wavefronts then take half of LDS's 128 bytes a cycle, and the writes a quarter.  At 2 x 2 they would take all of it; that
// form is for products too small to fill the chip with the large one.
//
// Blocks of k past the end: the fetch reads the last block again, and both scales are zero bytes, 2^-127 each, so that what
// comes of them, below 2^-243, is lost in any fp32 sum.
#ifndef TDC_MX4_TILE_H
#define TDC_MX4_TILE_H

#include "tdc_mx4_internal.h"

typedef float tdc_f16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ tdc_i8 tdc_mx4_widen(tdc_i4 a) { return __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1); }

// OP: which byte of the scale registers counts.
template <int OP> __device__ __forceinline__ tdc_f16v tdc_mx4_mfma(tdc_i4 a, unsigned sa, tdc_i4 b, unsigned sb, tdc_f16v c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(tdc_mx4_widen(a), tdc_mx4_widen(b), c, 4, 4, OP, (int)sa, OP, (int)sb);
}

// V sums of row m, from column n on, into y, which has rows of whole V's where V > 1.
template <typename T, int V> __device__ __forceinline__ void tdc_mx4_finish(const TdcMx4Product &q, float (&v)[V], int m, int n)
{
    const size_t at = (size_t)m * q.N + n;
    if (q.epi.bias) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += q.epi.bias[n + i];
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
    tdc_store<T, V>(static_cast<T *>(q.y) + at, v);
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

template <typename T, int WM, int WN, int GM, int GN>
__global__ __launch_bounds__(64 * GM * GN, 2) void tdc_mx4_product_tile(TdcMx4Product q)
{
    constexpr int BM = 32 * WM * GM, BN = 32 * WN * GN, THREADS = 64 * GM * GN;
    // two buffers, two objects: a read of one then visibly does not depend on what is being fetched into the other
    __shared__ __attribute__((aligned(128))) uint8_t codes0[(BM + BN) * 128], codes1[(BM + BN) * 128];
    __shared__ uint2 scales0[BM + BN], scales1[BM + BN];
    const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tm, tn;
    tdc_mx4_tile_at(blockIdx.x, (q.M + BM - 1) / BM, (q.N + BN - 1) / BN, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;

    // fetch: rows tid/8 + STEP i of both operands, the block that belongs at place tid%8 of the eight; scales of rows tid + THREADS i
    constexpr int STEP = THREADS / 8, FA = BM / STEP, FB = BN / STEP, SR = (BM + BN) / THREADS;
    static_assert((BM + BN) % THREADS == 0 && STEP % 16 == 0, "every thread fetches the same share");
    const int fr = tid >> 3, fk = (tid & 7) ^ ((fr >> 1) & 7);
    const uint8_t *src[FA + FB], *ssrc[SR];
#pragma unroll
    for (int i = 0; i < FA; ++i) src[i] = q.a_codes + (size_t)q.a_rows.source(min(m0 + fr + STEP * i, q.M - 1)) * q.nb * 16;
#pragma unroll
    for (int i = 0; i < FB; ++i) src[FA + i] = q.b_codes + (size_t)min(n0 + fr + STEP * i, q.N - 1) * q.nb * 16;
#pragma unroll
    for (int i = 0; i < SR; ++i) {
        const int r = tid + THREADS * i;
        ssrc[i] = r < BM ? q.a_scales + (size_t)q.a_rows.source(min(m0 + r, q.M - 1)) * q.nb : q.b_scales + (size_t)min(n0 + r - BM, q.N - 1) * q.nb;
    }
    uint2 sin[SR];
    auto fetch = [&](int k, uint8_t *codes) {
        const size_t at = (size_t)min(k + fk, q.nb - 1) * 16;
#pragma unroll
        for (int i = 0; i < FA + FB; ++i) tdc_mx4_fetch(src[i] + at, codes + (i * STEP + 8 * wave) * 128);
#pragma unroll
        for (int i = 0; i < SR; ++i) sin[i] = tdc_mx4_scales8(ssrc[i], k, q.nb);
    };
    // what was fetched is there for every wavefront
    auto arrive = [&](uint2 *scales) {
#pragma unroll
        for (int i = 0; i < SR; ++i) scales[tid + THREADS * i] = sin[i];
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

    auto multiply = [&](const uint8_t *codes, const uint2 *scales) {
        unsigned sa[WM][2], sb[WN][2];
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const uint2 v = scales[wm + 32 * i + r32];
            sa[i][0] = v.x >> (8 * h);
            sa[i][1] = v.y >> (8 * h);
        }
#pragma unroll
        for (int j = 0; j < WN; ++j) {
            const uint2 v = scales[BM + wn + 32 * j + r32];
            sb[j][0] = v.x >> (8 * h);
            sb[j][1] = v.y >> (8 * h);
        }
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
                    acc[i][j] = s & 1 ? tdc_mx4_mfma<2>(a[i], sa[i][s / 2], b[j], sb[j][s / 2], acc[i][j]) : tdc_mx4_mfma<0>(a[i], sa[i][s / 2], b[j], sb[j][s / 2], acc[i][j]);
        }
    };

    fetch(0, codes0);
    arrive(scales0);
    for (int k = 0;; k += 16) {
        if (k + 8 < q.nb) fetch(k + 8, codes1);
        multiply(codes0, scales0);
        if (k + 8 >= q.nb) break;
        arrive(scales1);
        if (k + 16 < q.nb) fetch(k + 16, codes0);
        multiply(codes1, scales1);
        if (k + 16 >= q.nb) break;
        arrive(scales0);
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
