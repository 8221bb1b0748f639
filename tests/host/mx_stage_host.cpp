// The offsets that the product's kernels load stages from (mx_stage.hpp, the
// kernels' own source) on the CPU.
#define __device__
#define __forceinline__ inline

#include "mx_stage.hpp"

extern "C" {

uint32_t tile_offset(int row0, int k, int lane, int row_bytes, int st, int nb)
{
    return mpq::tile_lane_offset(row0, lane, row_bytes) + mpq::tile_stage_offset(k, row_bytes, st, nb);
}

uint32_t slab_offset(int row, int r, int row_bytes, int st, int nb)
{
    return mpq::slab_lane_offset(row, r, row_bytes, st, nb);
}

}
