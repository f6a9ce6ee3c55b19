// Attention of one new token of each sequence over a paged cache of 16 or 8 bits
// (attend.h), and the sizes of the workspaces of all its forms.
#include "attend.h"

namespace cp {

size_t attend_workspace_bytes(int64_t batch, int64_t hq, int64_t hk, int64_t d, int64_t max_length, int64_t window, bool mass, bool four) {
  return size_t(layout(plan(batch, hq, hk, span_of(max_length, window), four && d <= 128), batch, hq, hk, d, mass).end) * sizeof(float);
}

bool attend_fits(int64_t batch, int64_t hq, int64_t hk, int64_t d, int64_t max_length, int64_t window, bool mass, bool four) {
  const Layout l = layout(plan(batch, hq, hk, span_of(max_length, window), four && d <= 128), batch, hq, hk, d, mass);
  // (256 threads a block of 512 tokens are the larger grid of the two forms that there are.)
  const int64_t blocks = batch * hq + (mass ? batch * hk * ((l.stride + 511) / 512) : 0);
  return l.whole || blocks < (int64_t(1) << 32) / 256;
}

hipError_t launch_attend(const AttendParams& p, hipStream_t stream) {
  return p.held == ServeType::kE4m3 ? launch_type<Held::kE4m3, false>(p, stream) : launch_type<Held::kSame, false>(p, stream);
}

}  // namespace cp
