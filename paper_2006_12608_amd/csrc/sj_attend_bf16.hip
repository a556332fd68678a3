// sj_attend_bf16.hip -- attention over a cache of bfloat16 rows.
#include "sj_attend_kernels.h"

namespace sjc {

hipError_t launch_attend_bf16(const Attend &a, hipStream_t s)
{
    return launch_attend<sjk::DT_BF16>(a, s);
}

}  // namespace sjc
