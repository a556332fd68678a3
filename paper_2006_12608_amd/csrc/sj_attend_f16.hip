// sj_attend_f16.hip -- attention over a cache of binary16 rows.
#include "sj_attend_kernels.h"

namespace sjc {

uint32_t attend_tile_rows(uint32_t rows, uint32_t d)
{
    if (rows <= 32)
        return rows <= 16 ? 16 : 32;
    // (d > 128 has no tile of 64 rows; two of its waves then only load.  64 query rows on 8
    // sequences of 1000 to 7000 rows, d = 256: 106 us in two tiles of 32, which both read the
    // cache, 68 in one)
    if (rows <= 64)
        return d <= 128 ? 64 : 128;
    return rows > 128 && d <= 128 ? 256 : 128;
}

int attend_occupancy_f16(uint32_t d, uint32_t tile_rows)
{
    return attend_occupancy<sjk::DT_F16, 2>(d, tile_rows, 1);
}

hipError_t launch_attend_f16(const Attend &a, hipStream_t s)
{
    return launch_attend<sjk::DT_F16, 2>(a, s);
}

}  // namespace sjc
