// The same over a cache of 4 bits (attend.h).
#include "attend.h"

namespace cp {

hipError_t launch_attend4_mass(const AttendParams& p, hipStream_t stream) { return launch_type<Held::kE2m1, true>(p, stream); }

}  // namespace cp
