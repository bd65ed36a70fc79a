// How the group norm's work is cut up: chunks of an image, or slices of channels that stay in a workgroup's registers.  Free of HIP,
// so that host-only code can check it.
#ifndef TDC_NORM_CHOICE_H
#define TDC_NORM_CHOICE_H

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#ifdef __HIPCC__
#define TDC_HOST_DEVICE __host__ __device__
#else
#define TDC_HOST_DEVICE
#endif

constexpr int TDC_NORM_THREADS = 512;    // of the kernels that run over chunks
constexpr int TDC_NORM_MAX_C = 8192;     // per-channel pairs of a workgroup fill at most 64 KiB of LDS
// Chunks of an image that every workgroup of the second kernel combines for itself.  More than that are combined by a kernel in
// between: 224x224x64 in fp16, 196 chunks, 16.5 us without it and 14.3 with it; at 64 chunks the two are even.
constexpr int TDC_NORM_PARTS = 64;

struct TdcNormDims {
    int B, P, C, G, Cg;     // P pixels to an image, Cg channels to a group
    int chunk_px, chunks;
    float eps;
};

// Backward, the workgroups to a channel leave a row of sums each, to be added up for dgamma and dbeta: some 512 rows.  Resident,
// every row is of some images; over chunks, there are as many rows to every chunk as this many images at a time make.
constexpr int TDC_NORM_SUM_ROWS = 512;
inline int tdc_norm_resident_rows(const TdcNormDims &d, int slices) { return std::min(d.B, std::max(1, TDC_NORM_SUM_ROWS / slices)); }
inline int tdc_norm_chunk_images(const TdcNormDims &d) { return std::min(d.B, std::max(1, TDC_NORM_SUM_ROWS / d.chunks)); }
inline size_t tdc_norm_sum_rows(const TdcNormDims &d)
{
    return std::max<size_t>((size_t)tdc_norm_chunk_images(d) * d.chunks, tdc_norm_resident_rows(d, 1));
}

// Pixels of chunk i of an image.
TDC_HOST_DEVICE inline int tdc_chunk_len(const TdcNormDims &d, int i)
{
    const int left = d.P - i * d.chunk_px;
    return left < d.chunk_px ? left : d.chunk_px;
}

// Pixels to a chunk: four workgroups to a compute unit over the batch, but four pieces to a thread, since what a thread does once,
// for its channels and for its sums, costs as much as some pieces (224x224x64 in fp16: 17.8 us with two, 14.6 with four); two or
// one where that leaves compute units without work (37x29x150 in bf16, 3 images: 12.7 us with four, 10.8 with two, 9.6 with one).
inline void tdc_norm_choose_chunks(TdcNormDims &d, int size)
{
    const int pieces = (d.C * size + 15) / 16;
    const int rows = pieces < TDC_NORM_THREADS ? TDC_NORM_THREADS / pieces : 1;
    const int most = d.B >= 1024 ? 1 : 1024 / d.B;
    int64_t chunks = 1;
    for (int each = 4; each; each /= 2) {
        chunks = ((int64_t)d.P + each * rows - 1) / (each * rows);
        if (d.B * chunks >= 128) break;
    }
    chunks = std::min<int64_t>(most, chunks);
    d.chunk_px = (int)((d.P + chunks - 1) / chunks);
    d.chunks = (d.P - 1) / d.chunk_px + 1;      // P + chunk_px may pass 2^31
}

// Pieces of x that a thread holds at most.  Forward, two workgroups of 512 threads to a compute unit have 128 registers a thread:
// 64 values of fp32, 32 of 16 bits that have to be converted.  Backward, where d is held too, in fp32, it is one with 256.
TDC_HOST_DEVICE constexpr int tdc_norm_held(int V, int size, bool backward) { return backward ? 8 : (V >= 4 && size == 2 ? 8 : 16); }

// A workgroup takes `width` channels, whole groups and whole pieces, of an image; `slices` of them to an image.
struct TdcNormSlice {
    int width, slices, threads, held;    // held: pieces to a thread; 0: the image does not fit
};

// The narrowest slices (whole groups, whole pieces, multiples of `multiple`) are widened to a line of 128 bytes of a pixel, or 64
// backward, and until there are no more than 1024 of them, as long as 512 threads hold them and 256 workgroups are left.  A line
// that several workgroups share comes from memory once all the same: they run on the same XCD (tdc_norm_place).  Measured,
// forward, fp32, 28x28x512, 32 images: 16 channels 21.8 us, 32 17.8; 28x28x128 in bf16, 32 images: 8 channels 9.6, 16 8.8, 32,
// with 128 workgroups, 9.8; 7x7x512, 256 images: 16 channels 30.9 us, 64 and 128 11.9.  Backward, 14x14x1024 in bf16, 32 images:
// 64 bytes 16.5, 128 18.9.  1024 threads lose (28x28x512, 32 images, 32 channels: 26.5; no second workgroup that reads while one
// writes) but where slices below 64 bytes of a tensor larger than the L2s can be wider by them.  With 512 threads and with 1024, over
// three sets of buffers in turn, fp32: 56x56x256, 16, 32 and 64 images 39.6 and 26.2 us, 65.1 and 54.9, 117.6 and 100.6; 32
// images of 48x48x256 50.0 and 41.8, 56x56x128 36.0 and 25.0, 64x64x256 86.4 and 65.4, 80x80x64 48.3 and 32.0, but 48x48x128 16.8
// and 17.0, 40x40x192 23.3 and 25.6; bf16: 56x56x256 50.4 and 38.3, 40x40x512 40.5 and 34.0.
inline TdcNormSlice tdc_norm_slice(const TdcNormDims &d, int size, int V, bool backward, int multiple)
{
    const int most = tdc_norm_held(V, size, backward), line = backward ? 64 : 128;
    int unit = d.Cg;
    while ((unit % V || unit % multiple) && unit < d.C) unit += d.Cg;
    if (unit > d.C || d.C % unit) unit = d.C;
    auto held = [&](int width, int threads) {
        const int nv = width / V;
        return nv <= threads && width / d.Cg <= threads ? (d.P - 1) / (threads / nv) + 1 : 1 << 30;
    };
    auto next = [&](int width) {
        do width += unit;
        while (width < d.C && d.C % width);
        return width;
    };
    auto fits = [&](int width) { return held(width, 512) <= most; };
    auto groups = [&](int width) { return (int64_t)d.B * (d.C / width); };
    auto launches = [&](int width, int threads) { return backward || groups(width) * threads <= 0xffffffffll; };   // a launch counts its threads in 32 bits
    if (!fits(unit)) return TdcNormSlice{};
    int width = unit;
    for (int w = next(width); w <= d.C && (width * size < line || groups(width) > 1024) && groups(w) >= 256 && fits(w); w = next(w)) width = w;
    if (!backward && width * size < 64 && (int64_t)d.B * d.P * d.C * size > (32 << 20)) {
        const int w = next(width);
        if (w <= d.C && held(w, 1024) <= most && launches(w, 1024)) return TdcNormSlice{w, d.C / w, 1024, held(w, 1024)};
    }
    const int threads = held(width, 256) <= 4 ? 256 : 512;
    if (!launches(width, threads)) return TdcNormSlice{};
    return TdcNormSlice{width, d.C / width, threads, held(width, threads)};
}

// A forward call's slice: of y, or of blocks of 4-bit values over neighbouring lanes, where C has whole blocks and accesses are 16 bytes.
inline bool tdc_norm_block_lanes(const TdcNormDims &d, int size, int V) { return d.C % 32 == 0 && V * size == 16; }
inline TdcNormSlice tdc_norm_forward_slice(const TdcNormDims &d, int size, int V, bool mx4)
{
    if (mx4 && !tdc_norm_block_lanes(d, size, V)) return TdcNormSlice{};
    return tdc_norm_slice(d, size, V, false, mx4 ? 32 : 1);
}
inline int tdc_norm_launches(const TdcNormDims &d, int size, int V, bool mx4)
{
    return tdc_norm_forward_slice(d, size, V, mx4).held ? 1 : d.chunks > TDC_NORM_PARTS ? 3 : 2;
}

// Whether the forward kernels store y past the L2's replacement: where workgroups write half lines or more of a tensor larger
// than an XCD's L2 at about the same time, in pieces of 8 bytes or more.  28x28x512 in bf16, 32 images, 64 bytes to a slice: 18.4
// us otherwise, 14.6 so.  Not where a compute unit has one workgroup of 1024 threads: 32 images in fp32, otherwise and so,
// 56x56x256 54.9 and 58.5, 64x64x256 65.4 and 78.1, 40x40x192 25.6 and 39.0, though 48x48x256 41.8 and 37.4; nor for small
// tensors: 56x56x64 in fp32, one image, 7.9 and 8.3.
inline bool tdc_norm_streams(const TdcNormDims &d, int size, int V, const TdcNormSlice &sl)
{
    return sl.threads != 1024 && (sl.held ? sl.width : d.C) * size >= 64 && V * size >= 8 && (double)d.B * d.P * d.C * size > 4e6;
}

#endif  // TDC_NORM_CHOICE_H
