// Device helpers of the microbatch operators: rows of any alignment in steps
// of eight columns, and reductions over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gwtf {

using f16_t = _Float16;
using bf16_t = __bf16;

// Eight adjacent columns.  Loads and stores of whole eights are one 16-byte
// access (two for 32-bit types) that needs no more alignment than the element.
constexpr int kVec = 8;

template <class T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <class T, int w>
struct VecN {
    typedef T type __attribute__((ext_vector_type(w), aligned(sizeof(T))));
};

// Columns [0, n) of p, 0 < n < 8, as 4 + 2 + 1; the rest `fill`.
template <class T>
__device__ __forceinline__ typename Vec8<T>::type load_part(const T *p, int n, T fill)
{
    typename VecN<T, 4>::type f4 = {fill, fill, fill, fill};
    typename VecN<T, 2>::type f2 = {fill, fill};
    T f1 = fill;
    if (n & 4) f4 = *reinterpret_cast<const typename VecN<T, 4>::type *>(p);
    if (n & 2) f2 = *reinterpret_cast<const typename VecN<T, 2>::type *>(p + (n & 4));
    if (n & 1) f1 = p[n & 6];
    // the columns after the four: two and one, or one alone
    const T r0 = n & 2 ? f2[0] : f1, r1 = f2[1], r2 = n & 2 ? f1 : fill;
    typename Vec8<T>::type v = {f4[0], f4[1], f4[2], f4[3], r0, r1, r2, fill};
    if (!(n & 4)) {
        const typename Vec8<T>::type w = {r0, r1, r2, fill, fill, fill, fill, fill};
        v = w;
    }
    return v;
}
template <class T>
__device__ __forceinline__ void store_part(T *p, int n, const typename Vec8<T>::type &v)
{
    if (n & 4) {
        const typename VecN<T, 4>::type f4 = {v[0], v[1], v[2], v[3]};
        *reinterpret_cast<typename VecN<T, 4>::type *>(p) = f4;
    }
    const T r0 = n & 4 ? v[4] : v[0], r1 = n & 4 ? v[5] : v[1], r2 = n & 4 ? v[6] : v[2];
    if (n & 2) {
        const typename VecN<T, 2>::type f2 = {r0, r1};
        *reinterpret_cast<typename VecN<T, 2>::type *>(p + (n & 4)) = f2;
    }
    if (n & 1) p[n & 6] = n & 2 ? r2 : r0;
}

// Columns [0, n) of p as they lie in memory, the rest `fill`; n >= 8 is the
// common case, n <= 0 reads nothing.  STREAM: a read that leaves the caches to
// others (kStreamBytes).
template <class T, bool STREAM = false>
__device__ __forceinline__ typename Vec8<T>::type load8_raw(const T *p, int64_t n, T fill = T(0.f))
{
    if (n >= kVec) {
        if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const typename Vec8<T>::type *>(p));
        else return *reinterpret_cast<const typename Vec8<T>::type *>(p);
    }
    return load_part(p, n > 0 ? int(n) : 0, fill);
}

template <class T>
__device__ __forceinline__ void widen(const typename Vec8<T>::type &raw, float v[8])
{
    const f32x8 f = __builtin_convertvector(raw, f32x8);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = f[i];
}

// The same in 32 bits.
template <class T, bool STREAM = false>
__device__ __forceinline__ void load8(const T *p, int64_t n, float v[8], float fill = 0.f)
{
    widen<T>(load8_raw<T, STREAM>(p, n, T(fill)), v);
}

// Columns [col, col + 8) of a row of `width`, for reads that are to be in
// flight for long: a row's last ones come with the columns before them, in one
// access like all others, and columns_of() puts them into place when they are
// needed.  (Put together from parts here, they would be waited for at once.)
// WIDE: the caller knows that the width is 8 at least.
template <class T, bool STREAM = false, bool WIDE = false>
__device__ __forceinline__ typename Vec8<T>::type load_columns(const T *row, int64_t col, int64_t width)
{
    if (!WIDE && width < kVec) return load_part(row, col == 0 ? int(width) : 0, T(0.f));
    return load8_raw<T, STREAM>(row + (col + kVec <= width ? col : width - kVec), kVec);
}
// Whether any lane of the wave has columns past the row's end (uniform).
__device__ __forceinline__ bool ends_within(int64_t col, int64_t width) { return __ballot(col + kVec > width) != 0; }
template <class T>
__device__ __forceinline__ void columns_of(const typename Vec8<T>::type &raw, bool ends, int64_t col, int64_t width, float v[8])
{
    widen<T>(raw, v);
    if (!ends || width < kVec) return;
    const int over = int(col + kVec - width > 0 ? col + kVec - width : 0);
#pragma unroll
    for (int step = 4; step > 0; step >>= 1) {
        const bool move = over >= kVec || (over & step);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = move ? (i + step < kVec ? v[i + step] : 0.f) : v[i];
    }
    if (over >= kVec) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = 0.f;
    }
}

template <class T, bool STREAM = false>
__device__ __forceinline__ void store8(T *p, int64_t n, const float v[8])
{
    f32x8 f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) f[i] = v[i];
    const typename Vec8<T>::type r = __builtin_convertvector(f, typename Vec8<T>::type);
    if (n >= kVec) {
        if constexpr (STREAM) __builtin_nontemporal_store(r, reinterpret_cast<typename Vec8<T>::type *>(p));
        else *reinterpret_cast<typename Vec8<T>::type *>(p) = r;
    } else if (n > 0) {
        store_part(p, int(n), r);
    }
}

__device__ __forceinline__ int64_t load_token(const void *t, int is64, int64_t i)
{
    return is64 ? static_cast<const int64_t *>(t)[i] : int64_t(static_cast<const int32_t *>(t)[i]);
}

// Division of u < 2^32 by a fixed d >= 1 (Granlund and Montgomery): a high
// product and two shifts.
struct FastDiv {
    uint32_t d, m, s1, s2;
    static FastDiv make(uint32_t d)
    {
        uint32_t l = 0;
        while (l < 32 && (uint64_t(1) << l) < d) ++l;
        FastDiv f;
        f.d = d;
        f.m = uint32_t(((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1);
        f.s1 = l < 1 ? l : 1;
        f.s2 = l > 1 ? l - 1 : 0;
        return f;
    }
    __device__ __forceinline__ uint32_t div(uint32_t u) const
    {
        const uint32_t t = __umulhi(m, u);
        return (t + ((u - t) >> s1)) >> s2;
    }
};

// Lane exchanges within rows of 16 lanes (rotation by n).
template <int n>
__device__ __forceinline__ int row_ror(int v)
{
    return __builtin_amdgcn_update_dpp(v, v, 0x120 + n, 0xf, 0xf, false);
}
template <int n>
__device__ __forceinline__ float row_ror(float v)
{
    return __int_as_float(row_ror<n>(__float_as_int(v)));
}

__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// Sum over 16 lanes, in every one of them; over the wave, uniform.
__device__ __forceinline__ float row_sum(float v)
{
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    v += row_ror<1>(v);
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = row_sum(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

// The largest over the wave, uniform; of a number and a NaN the number.
__device__ __forceinline__ float wave_fmax(float v)
{
    v = fmaxf(v, row_ror<8>(v));
    v = fmaxf(v, row_ror<4>(v));
    v = fmaxf(v, row_ror<2>(v));
    v = fmaxf(v, row_ror<1>(v));
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

// The largest of unsigned words likewise (float magnitudes compare as their
// bits do, with infinities and NaN above all numbers).
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t row_umax(uint32_t v)
{
    v = umax(v, uint32_t(row_ror<8>(int(v))));
    v = umax(v, uint32_t(row_ror<4>(int(v))));
    v = umax(v, uint32_t(row_ror<2>(int(v))));
    v = umax(v, uint32_t(row_ror<1>(int(v))));
    return v;
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v)
{
    v = row_umax(v);
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return umax(umax(a, b), umax(c, d));
}

// 2^x and ln 2 / log2 e; the hardware's exponential and logarithm have base 2.
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLn2Low = float(0.69314718055994530942 - double(kLn2));
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

} // namespace gwtf
