// sj_attend_f16.hip -- attention over a cache of binary16 rows.
#include "sj_attend_kernels.h"

namespace sjc {

uint32_t attend_tile_rows(uint32_t rows, uint32_t) { return rows <= AT_Q ? AT_Q : 2 * AT_Q; }

hipError_t launch_attend_f16(const Attend &a, hipStream_t s)
{
    return launch_attend<sjk::DT_F16>(a, s);
}

}  // namespace sjc
