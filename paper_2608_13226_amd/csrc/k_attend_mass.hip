// Attention over a paged cache of 16 or 8 bits that adds the weights to each token's mass (attend.h).
#include "attend.h"

namespace cp {

hipError_t launch_attend_mass(const AttendParams& p, hipStream_t stream) {
  return p.held == ServeType::kE4m3 ? launch_type<Held::kE4m3, true>(p, stream) : launch_type<Held::kSame, true>(p, stream);
}

}  // namespace cp
