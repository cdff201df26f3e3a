// Distillation: a list of teacher entries per row.
#include "head_kernel.h"

namespace ffmlp {

hipError_t launch_head_distill(HeadPass pass, bool large, const HeadArgs& a, const RowLossArgs& r, hipStream_t s) {
  return launch_head<true>(pass, large, a, r, s);
}

}  // namespace ffmlp
