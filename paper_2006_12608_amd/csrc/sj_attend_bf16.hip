// sj_attend_bf16.hip -- attention over a cache of bfloat16 rows.
#include "sj_attend_kernels.h"

namespace sjc {

int attend_occupancy_bf16(uint32_t d, uint32_t tile_rows)
{
    return attend_occupancy<sjk::DT_BF16, 2>(d, tile_rows, 1);
}

hipError_t launch_attend_bf16(const Attend &a, hipStream_t s)
{
    return launch_attend<sjk::DT_BF16, 2>(a, s);
}

}  // namespace sjc
