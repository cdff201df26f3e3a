// Cross entropy: one target per row.
#include "head_kernel.h"

namespace ffmlp {

hipError_t launch_head_ce(bool prob, bool large, bool direct, const HeadArgs& a, hipStream_t s) {
  return launch_head<false>(prob, large, direct, a, s);
}

}  // namespace ffmlp
