// Cross entropy: one target per row.
#include "head_kernel.h"

namespace ffmlp {

hipError_t launch_head_ce(HeadPass pass, bool large, const HeadArgs& a, const RowLossArgs& r, hipStream_t s) {
  return launch_head<false>(pass, large, a, r, s);
}

}  // namespace ffmlp
