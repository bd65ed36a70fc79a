// Elements of the three activation types and what kernels do with them: loads and stores of V neighbours at once, sums over
// lanes, activations.  Shared by the norm and the 4-bit kernels.
#ifndef TDC_TYPED_H
#define TDC_TYPED_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "tdc_internal.h"
#include "tdc_norm.h"

typedef _Float16 tdc_half;
typedef __bf16 tdc_bf16;

inline int tdc_dtype_bytes(int dtype) { return dtype == TDC_F32 ? 4 : 2; }
inline bool tdc_known_dtype(int dtype) { return dtype == TDC_F32 || dtype == TDC_F16 || dtype == TDC_BF16; }
inline bool tdc_known_act(int act) { return act == TDC_ACT_NONE || act == TDC_ACT_RELU || act == TDC_ACT_SILU; }
inline bool tdc_aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// V neighbours, V * sizeof(T) <= 16 a power of two: one load.  The pointer is aligned to all of them.
template <typename T, int V> struct __align__(sizeof(T) * V) TdcVec {
    T v[V];
};

template <typename T, int V> __device__ __forceinline__ TdcVec<T, V> tdc_load(const T *p)
{
    return *reinterpret_cast<const TdcVec<T, V> *>(p);
}

// V neighbours as the words they are loaded as, for pieces that are held or fetched ahead.  Elements of TdcVec that live across a
// branch become values of their own to the compiler, and those of 16 bits are cut out of their words, and waited for, right behind
// the load: one load after the other.
template <typename T, int V> struct TdcRaw {
    static constexpr int BYTES = sizeof(T) * V;
    typedef unsigned Vector __attribute__((ext_vector_type(BYTES < 8 ? 2 : BYTES / 4)));
    typedef std::conditional_t<BYTES < 8, unsigned, Vector> Words;
    Words w;
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (BYTES < 4) w = *reinterpret_cast<const unsigned short *>(p);
        else w = *reinterpret_cast<const Words *>(p);
    }
    // The neighbours, made anew: the compiler takes them for something it has not seen, so that what it computed from them before is
    // computed again and not kept.  A kernel that goes twice over pieces in registers has no room for both the pieces and their values.
    __device__ __forceinline__ TdcVec<T, V> open()
    {
        asm volatile("" : "+v"(w));
        TdcVec<T, V> o;
        __builtin_memcpy(&o, &w, BYTES);
        return o;
    }
};

// The same for an index, whose addresses are then made where they are used and do not fill registers until then.
__device__ __forceinline__ int tdc_anew(int i)
{
    asm volatile("" : "+v"(i));
    return i;
}

template <typename T, int V> __device__ __forceinline__ void tdc_store(T *p, const float (&f)[V])
{
    TdcVec<T, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.v[i] = (T)f[i];
    *reinterpret_cast<TdcVec<T, V> *>(p) = o;
}

// The same past the L2's replacement: for results that fill whole lines at a time and are not read again by this kernel, which
// then has less to write back when it ends.
template <typename T, int V> __device__ __forceinline__ void tdc_store_stream(T *p, const float (&f)[V])
{
    TdcVec<T, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.v[i] = (T)f[i];
    if constexpr (sizeof(o) >= 4) {
        typedef unsigned Words __attribute__((ext_vector_type(sizeof(o) / 4)));
        Words w;
        __builtin_memcpy(&w, &o, sizeof(o));
        __builtin_nontemporal_store(w, reinterpret_cast<Words *>(p));
    } else {
        *reinterpret_cast<TdcVec<T, V> *>(p) = o;
    }
}

// 1 / (1 + exp(-v)): v_exp and v_rcp are good to about an ulp each, and both ends are right: exp(-v) = inf gives 0, 0 gives 1.
__device__ __forceinline__ float tdc_sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

template <int ACT> __device__ __forceinline__ float tdc_activate(float v)
{
    if constexpr (ACT == TDC_ACT_RELU) return v > 0.f ? v : (v != v ? v : 0.f);   // a NaN stays one
    if constexpr (ACT == TDC_ACT_SILU) return v * tdc_sigmoid(v);
    return v;
}

template <int V> __device__ __forceinline__ void tdc_activate_all(int act, float (&v)[V])
{
    if (act == TDC_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = tdc_activate<TDC_ACT_RELU>(v[i]);
    } else if (act == TDC_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = tdc_activate<TDC_ACT_SILU>(v[i]);
    }
}

// The gradient d of act(v) as that of v.  ReLU chooses: 0 where v <= 0 even for an infinite d, and a NaN of v stays one.
template <int ACT> __device__ __forceinline__ float tdc_activate_back(float d, float v)
{
    if constexpr (ACT == TDC_ACT_RELU) return v > 0.f ? d : (v != v ? v : 0.f);
    if constexpr (ACT == TDC_ACT_SILU) {
        const float s = tdc_sigmoid(v);
        return d * (s * (1.f + v * (1.f - s)));
    }
    return d;
}

// ---- lanes of a wavefront, without a trip through LDS

// The value of another lane of a row of 16; the constants are the ISA's (quad_perm, row_half_mirror, row_mirror, row_ror:n).
template <int CTRL> __device__ __forceinline__ float tdc_dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
constexpr int TDC_DPP_XOR1 = 0xb1, TDC_DPP_XOR2 = 0x4e, TDC_DPP_HALF_MIRROR = 0x141, TDC_DPP_MIRROR = 0x140, TDC_DPP_ROR = 0x120;

// What the two rows of 16 of every 32 lanes hold, and the two halves of the 64: lane by lane, the same pair in both.
__device__ __forceinline__ float2 tdc_rows16(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];
    return make_float2(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float2 tdc_rows32(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];
    return make_float2(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// Sum over the neighbouring `lanes` lanes (a power of two up to 64), the same in each of them.  The mirrors do for exchanges of 4
// and 8 lanes: what they swap is the same in all four or eight.
__device__ __forceinline__ float tdc_lane_sum(float v, int lanes)
{
    if (lanes > 1) v += tdc_dpp<TDC_DPP_XOR1>(v);
    if (lanes > 2) v += tdc_dpp<TDC_DPP_XOR2>(v);
    if (lanes > 4) v += tdc_dpp<TDC_DPP_HALF_MIRROR>(v);
    if (lanes > 8) v += tdc_dpp<TDC_DPP_MIRROR>(v);
    if (lanes > 16) {
        const float2 r = tdc_rows16(v);
        v = r.x + r.y;
    }
    if (lanes > 32) {
        const float2 r = tdc_rows32(v);
        v = r.x + r.y;
    }
    return v;
}

// The largest of unsigned bits over 4 or 8 neighbouring lanes.
template <int LANES> __device__ __forceinline__ unsigned tdc_lane_max(unsigned u)
{
    u = max(u, __builtin_bit_cast(unsigned, tdc_dpp<TDC_DPP_XOR1>(__builtin_bit_cast(float, u))));
    u = max(u, __builtin_bit_cast(unsigned, tdc_dpp<TDC_DPP_XOR2>(__builtin_bit_cast(float, u))));
    if (LANES > 4) u = max(u, __builtin_bit_cast(unsigned, tdc_dpp<TDC_DPP_HALF_MIRROR>(__builtin_bit_cast(float, u))));
    return u;
}

// f(first, second) over the lanes that are `from`, 2 `from`, ... apart, `from` a power of two below 64: first(v) is a lane's own
// value of v, second(v) another's, and what f leaves is merged further.  Below 16 apart lanes of a row go around, so lanes merge
// in orders of their own; the lanes below `from` are those to read.
template <typename F> __device__ __forceinline__ void tdc_merge_lanes(int from, F f)
{
    const auto own = [](float v) { return v; };
    if (from <= 1) f(own, [](float v) { return tdc_dpp<TDC_DPP_ROR + 1>(v); });
    if (from <= 2) f(own, [](float v) { return tdc_dpp<TDC_DPP_ROR + 2>(v); });
    if (from <= 4) f(own, [](float v) { return tdc_dpp<TDC_DPP_ROR + 4>(v); });
    if (from <= 8) f(own, [](float v) { return tdc_dpp<TDC_DPP_ROR + 8>(v); });
    if (from <= 16) f([](float v) { return tdc_rows16(v).x; }, [](float v) { return tdc_rows16(v).y; });
    if (from <= 32) f([](float v) { return tdc_rows32(v).x; }, [](float v) { return tdc_rows32(v).y; });
}

// The statements for a dtype with T its type, for V neighbours with the constant V.
#define TDC_FOR_DTYPE(dtype, T, ...)                                  \
    do {                                                              \
        if ((dtype) == TDC_F32) { using T = float; __VA_ARGS__; }     \
        else if ((dtype) == TDC_F16) { using T = tdc_half; __VA_ARGS__; } \
        else { using T = tdc_bf16; __VA_ARGS__; }                     \
    } while (0)

#define TDC_FOR_VEC(v, T, V, ...)                                                         \
    do {                                                                                  \
        if ((v) == 8) { if constexpr (sizeof(T) == 2) { constexpr int V = 8; __VA_ARGS__; } } \
        else if ((v) == 4) { constexpr int V = 4; __VA_ARGS__; }                          \
        else if ((v) == 2) { constexpr int V = 2; __VA_ARGS__; }                          \
        else { constexpr int V = 1; __VA_ARGS__; }                                        \
    } while (0)

#define TDC_FOR_VEC4(v, V, ...)                                                           \
    do {                                                                                  \
        if ((v) == 4) { constexpr int V = 4; __VA_ARGS__; }                               \
        else if ((v) == 2) { constexpr int V = 2; __VA_ARGS__; }                          \
        else { constexpr int V = 1; __VA_ARGS__; }                                        \
    } while (0)

#endif  // TDC_TYPED_H
