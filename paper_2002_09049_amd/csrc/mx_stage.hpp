// Where the product's kernels load a stage's codes from: byte offsets into a
// buffer that begins at the workgroup's first row and ends behind the last row
// that it has (mx_product.hip).  A lane of a row past that end, and every lane
// of a stage past the rows' end, gets an offset outside the buffer, whose loads
// give zeros.  tests/host/mx_stage_host.cpp goes through them on the CPU.
#pragma once

#include <stdint.h>

namespace mpq {

constexpr uint32_t kOutside = 0x80000000u;   // past every buffer (256 rows of at most 2^21 bytes)

// Tiles: stages of 128 elements.  Load k of a wavefront whose rows begin at
// row0 covers 16 rows, lane l row row0 + 16 k + l / 4; its offset is the sum of
// the two.
constexpr int kStageBytes = 64;

__device__ __forceinline__ uint32_t tile_lane_offset(int row0, int lane, int row_bytes)
{
    return (uint32_t)((row0 + lane / 4) * row_bytes + ((lane % 4) ^ (lane / 16)) * 16);
}

__device__ __forceinline__ uint32_t tile_stage_offset(int k, int row_bytes, int st, int nb)
{
    return 4 * st < nb ? (uint32_t)(16 * k * row_bytes + st * kStageBytes) : kOutside;
}

// Slabs: stages of 512 elements.  A load covers four rows of 16; place r of
// row `row` takes piece r ^ row.
constexpr int kSlabBytes = 256;

__device__ __forceinline__ uint32_t slab_lane_offset(int row, int r, int row_bytes, int st, int nb)
{
    const int piece = r ^ row;
    return 16 * st + piece < nb ? (uint32_t)(row * row_bytes + piece * 16 + st * kSlabBytes) : kOutside;
}

}  // namespace mpq
