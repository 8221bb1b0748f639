// The offsets that the products by expert load gathered rows from (mx_stage.hpp,
// the kernels' own source) on the CPU.
#define __device__
#define __forceinline__ inline

#include "mx_stage.hpp"

extern "C" uint32_t gather_offset(int64_t row, int lane, int row_bytes, int st, int nb)
{
    return mpq::tile_gather_stage(mpq::tile_gather_offset(row, lane, row_bytes), st, nb);
}
