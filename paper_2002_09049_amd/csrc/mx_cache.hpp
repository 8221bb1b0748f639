// Places in the paged cache, and eight elements of a row to and from them.
#pragma once

#include "mx.hpp"

namespace mpq {

// Where a slot is: page and the token's place in it.
__device__ __forceinline__ void find(const MxCacheView &c, int64_t slot, int64_t &page, int &at)
{
    if ((c.page & (c.page - 1)) == 0) {
        page = slot >> (31 - __clz(c.page));
        at = (int)slot & (c.page - 1);
    } else {
        page = quotient(slot, c.page);
        at = (int)(slot - page * c.page);
    }
}

// Bytes of eight elements' codes at j of the row, and of the block's scale.
template <int kFmt>
__device__ __forceinline__ int64_t code_at(const MxCacheView &c, int64_t ph, int at, int j)
{
    constexpr int kWords = kFmt == kFp4 ? 1 : 2;
    return (ph * c.page + at) * (c.nb * 16 * kWords) + j / 2 * kWords;
}
__device__ __forceinline__ int64_t scale_at(const MxCacheView &c, int64_t ph, int at, int j)
{
    return (ph * c.nb + j / kMxBlock) * c.page + at;
}

template <int kFmt>
__device__ __forceinline__ void write8(const float (&x)[8], uint8_t *codes, uint8_t *scale, bool first)
{
    constexpr int kWords = kFmt == kFp4 ? 1 : 2;
    const uint32_t s = mx_scale_byte<kFmt>(quad_max(largest_bits(x)));
    uint32_t w[kWords];
    mx_codes<kFmt>(x, s, w);
    __builtin_memcpy(__builtin_assume_aligned(codes, 4 * kWords), w, sizeof w);
    if (first) *scale = (uint8_t)s;
}

template <int kFmt>
__device__ __forceinline__ void read8(const uint8_t *codes, const uint8_t *scale, float (&x)[8])
{
    constexpr int kWords = kFmt == kFp4 ? 1 : 2;
    uint32_t w[kWords];
    __builtin_memcpy(w, __builtin_assume_aligned(codes, 4 * kWords), sizeof w);
    mx_values<kFmt>(w, *scale, x);
}

}  // namespace mpq
