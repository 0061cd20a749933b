// The split kernel over a cache in 8 bits.
#include "paged_split.h"

namespace tkphi {

void launch_split_codes(const PagedGeom& g, hipStream_t s) {
  if (g.d == 64) launch_split_rows<Code8, 64>(g, s);
  else launch_split_rows<Code8, 128>(g, s);
}

void launch_blocks_codes(const PagedGeom& g, hipStream_t s) {
  if (g.d == 64) launch_blocks<Code8, 64>(g, s);
  else launch_blocks<Code8, 128>(g, s);
}

}  // namespace tkphi
