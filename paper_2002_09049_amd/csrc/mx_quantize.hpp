// What one workgroup does to quantize rows to fp4 blocks (mx_quantize.hip has
// the layout and its reasons).
#pragma once

#include "mx.hpp"

namespace mpq {

constexpr int kRowThreads = 256, kRowElems = kRowThreads * 8;

// The row and the place in it of this thread's eight elements.
__device__ __forceinline__ void place_eight(int64_t block, int w, int64_t &row, int &j)
{
    const int64_t first = block * kRowElems;
    const int64_t row0 = quotient(first, w);
    const uint32_t off = (uint32_t)(first - row0 * w) + 8 * threadIdx.x;
    // rows of 2048 or more: the first one or the next
    const uint32_t more = w >= kRowElems ? (off >= (uint32_t)w ? 1u : 0u) : small_quotient(off, 1.0f / (float)w);
    row = row0 + more;
    j = (int)(off - more * (uint32_t)w);
}

template <class T>
__device__ __forceinline__ void quantize_eight(int64_t block, const T *X, int64_t rows, int d, int64_t ld, int w,
                                               uint8_t *codes, uint8_t *scales)
{
    int64_t row;
    int j;
    place_eight(block, w, row, j);
    if (row >= rows) return;   // whole quads: w is a multiple of 32
    float x[8];
    load8(X + row * ld + j, d - j, x);
    const uint32_t s = mx_scale_byte<kFp4>(quad_max(largest_bits(x)));
    uint32_t c[1];
    mx_codes<kFp4>(x, s, c);
    *(uint32_t *)(codes + row * (w / 2) + j / 2) = c[0];
    if (j % kMxBlock == 0) scales[row * (w / kMxBlock) + j / kMxBlock] = (uint8_t)s;
}

}  // namespace mpq
