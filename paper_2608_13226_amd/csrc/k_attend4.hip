// Attention of one new token of each sequence over a paged cache of 4 bits (attend.h).
#include "attend.h"

namespace cp {

hipError_t launch_attend4(const AttendParams& p, hipStream_t stream) { return launch_type<Held::kE2m1, false>(p, stream); }

}  // namespace cp
