// sj_attend8_f16.hip -- attention over a cache of e4m3 rows, queries and results in binary16.
#include "sj_attend_kernels.h"

namespace sjc {

int attend8_occupancy_f16(uint32_t d, uint32_t tile_rows, uint32_t heads)
{
    return attend_occupancy<sjk::DT_F16, 1>(d, tile_rows, heads);
}

hipError_t launch_attend8_f16(const Attend &a, hipStream_t s)
{
    return launch_attend<sjk::DT_F16, 1>(a, s);
}

}  // namespace sjc
