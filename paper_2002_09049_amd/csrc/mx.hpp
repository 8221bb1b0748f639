// Microscaled formats (device side): a block of 32 consecutive elements
// shares the power of two 2^(s - 127), s one byte (255: the block is not a
// number); an element is E2M1 (kFp4, two a byte, the even one in the low
// half) or E4M3 (kFp8).
//
// With a the block's largest magnitude, s = floor(log2 a) + 127 - emax, at
// least 0, emax the exponent of the format's largest element (2 and 8): the
// exponent field of a's bits less emax, no logarithm.  x 2^(127 - s) is an
// exact product; the element is its nearest value, ties to even, at most the
// largest (6 and 448).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.hpp"
#include "reduce.hpp"

namespace mpq {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int kFp4 = 0, kFp8 = 1;   // MPQ_MX_FP4, MPQ_MX_FP8
constexpr int kMxBlock = 32;

// The work-items of a launch are counted in 32 bits along each dimension: more
// than kGridRow workgroups in x (of at most 1024) go in rows of that many, along
// the dimension left free.  The last row goes past the end.
constexpr int64_t kGridRow = 1 << 20;
inline unsigned grid_x(int64_t blocks) { return (unsigned)(blocks < kGridRow ? blocks : kGridRow); }
inline int64_t grid_rows(int64_t blocks) { return (blocks + kGridRow - 1) / kGridRow; }
__device__ __forceinline__ int64_t block_of(unsigned row) { return row * kGridRow + blockIdx.x; }

// Eight consecutive values of a row as they lie in memory: what a load in
// flight fills (their values taken apart, the load would have to be done).
template <class T>
struct Eight {
    uint32_t w[2 * sizeof(T)];

    __device__ __forceinline__ void values(float (&x)[8]) const
    {
        T v[8];
        __builtin_memcpy(v, w, sizeof v);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
};

// `live` of the eight are inside the row, the others are zero.  The row need
// only be aligned to its element: global loads of gfx950 take any address, and
// a whole vector goes in 16-byte loads.
template <class T>
__device__ __forceinline__ Eight<T> load_eight(const T *p, int live)
{
    Eight<T> e;
    if (live >= 8) {
        __builtin_memcpy(e.w, p, sizeof e.w);
    } else {
        T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < live ? p[i] : (T)0.0f;
        __builtin_memcpy(e.w, v, sizeof e.w);
    }
    return e;
}

template <class T>
__device__ __forceinline__ void load8(const T *p, int live, float (&x)[8])
{
    load_eight(p, live).values(x);
}

typedef uint32_t loose_vector __attribute__((ext_vector_type(4), aligned(2)));

// The first `live` of eight values to a row.  kPast: past the caches, for what
// fills whole lines and is not read again here (rows read back from fp4:
// 43 us, by ordinary stores 69).
template <bool kPast, class T>
__device__ __forceinline__ void store8(T *p, int live, const float (&x)[8])
{
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
    if (live >= 8) {
        loose_vector o[sizeof(T) / 2];
        __builtin_memcpy(o, v, sizeof v);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            if constexpr (kPast) __builtin_nontemporal_store(o[i], (loose_vector *)p + i);
            else ((loose_vector *)p)[i] = o[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < live) p[i] = v[i];
    }
}

// n / d for n + d below 2^22: a quotient is at least 1 / (2 d) away from
// (n + 1/2) / d's neighbouring integers, far more than the product's rounding.
__device__ __forceinline__ uint32_t small_quotient(uint32_t n, float inverse)
{
    return (uint32_t)(((float)n + 0.5f) * inverse);
}

// n / d, in 32 bits where n allows.
__device__ __forceinline__ int64_t quotient(int64_t n, int d)
{
    return n < 0x100000000LL ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

// The scale byte of a block whose largest magnitude has these bits (an
// infinity's and a NaN's bits are above every finite number's).
template <int kFmt>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits)
{
    constexpr int emax = kFmt == kFp4 ? 2 : 8;
    if (amax_bits >= 0x7f800000u) return 255u;
    const int e = (int)(amax_bits >> 23) - emax;
    return e > 0 ? (uint32_t)e : 0u;
}

// 2^(s - 127) as the bits whose exponent field is s, as the conversions with
// a scale take it (0: 2^-127, 255: not a number).
__device__ __forceinline__ float mx_scale(uint32_t s) { return __uint_as_float(s << 23); }

__device__ __forceinline__ uint32_t largest_bits(const float (&x)[8])
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(x[i]) & 0x7fffffffu);
    return a;
}

// A block's largest magnitude from the four lanes that hold it (a quad).
__device__ __forceinline__ uint32_t quad_max(uint32_t a)
{
    a = max(a, xstep<0>(a));
    return max(a, xstep<1>(a));
}

// The codes of eight elements under the scale byte s: one word (fp4) or two.
template <int kFmt>
__device__ __forceinline__ void mx_codes(const float (&x)[8], uint32_t s, uint32_t (&w)[kFmt == kFp4 ? 1 : 2])
{
    // s is at most 252, or 255, whose elements are zeros
    const float inv = __uint_as_float((254u - s) << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = s == 255u ? 0.0f : x[i] * inv;
    if constexpr (kFmt == kFp4) {
        uint32_t v = 0;
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[0], y[1], 1.0f, 0);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[2], y[3], 1.0f, 1);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[4], y[5], 1.0f, 2);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[6], y[7], 1.0f, 3);
        w[0] = v;
    } else {
        // the conversion gives NaN past 464: bounded first (a y is below 512)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(y[i], -448.0f), 448.0f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
            w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], v, true);
        }
    }
}

// The values of eight elements.
template <int kFmt>
__device__ __forceinline__ void mx_values(const uint32_t (&w)[kFmt == kFp4 ? 1 : 2], uint32_t s, float (&x)[8])
{
    const float sc = mx_scale(s);
    f32x2 v[4];
    if constexpr (kFmt == kFp4) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], sc, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], sc, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], sc, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], sc, 3);
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], sc, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], sc, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[1], sc, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[1], sc, true);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = v[i][0];
        x[2 * i + 1] = v[i][1];
    }
}

}  // namespace mpq
