"""csrc/tdc_norm_choice.h as a host library: how the group norm cuts its work up, without a GPU."""
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r'''
#include "tdc_norm_choice.h"
static TdcNormDims dims(const int64_t *s) {
    TdcNormDims d{(int)s[0], (int)(s[1] * s[2]), (int)s[3], (int)s[4], (int)(s[3] / s[4]), 0, 0, 1e-5f};
    tdc_norm_choose_chunks(d, (int)s[5]);
    return d;
}
extern "C" void chunks(const int64_t *s, int64_t *out) {
    const TdcNormDims d = dims(s);
    out[0] = d.chunk_px; out[1] = d.chunks; out[2] = tdc_norm_chunk_images(d); out[3] = (int64_t)tdc_norm_sum_rows(d);
}
extern "C" void slice(const int64_t *s, int V, int backward, int multiple, int64_t *out) {
    const TdcNormDims d = dims(s);
    const TdcNormSlice l = tdc_norm_slice(d, (int)s[5], V, backward != 0, multiple);
    out[0] = l.width; out[1] = l.slices; out[2] = l.threads; out[3] = l.held; out[4] = tdc_norm_streams(d, (int)s[5], V, l);
}
'''


@functools.lru_cache(maxsize=None)
def _lib():
    cxx = shutil.which("g++")
    assert cxx, "g++ is needed for this test"
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "choice.cpp"), os.path.join(tmp, "choice.so")
        with open(src, "w") as f:
            f.write(SRC)
        subprocess.run([cxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2211_03715_amd", "csrc"), src, "-o", so], check=True)
        return ctypes.CDLL(so)


def _numbers(shape, size):
    return (ctypes.c_int64 * 6)(*shape, size)


def chunks(shape, size):
    """{chunk_px, chunks, images, sum_rows} of (B, H, W, C, groups) with elements of ``size`` bytes: pixels to a chunk, chunks to an image,
    images that the backward pass takes at a time, rows of channels' sums in the workspace."""
    out = (ctypes.c_int64 * 4)()
    _lib().chunks(_numbers(shape, size), out)
    return dict(zip(("chunk_px", "chunks", "images", "sum_rows"), out))


def slices(shape, size, V, backward=False, multiple=1):
    """{width, slices, threads, held, streams} with V channels to an access; held = 0: not resident."""
    out = (ctypes.c_int64 * 5)()
    _lib().slice(_numbers(shape, size), V, int(backward), multiple, out)
    return dict(zip(("width", "slices", "threads", "held", "streams"), out))
