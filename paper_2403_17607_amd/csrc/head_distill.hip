// Distillation: a list of teacher entries per row.
#include "head_kernel.h"

namespace ffmlp {

hipError_t launch_head_distill(bool prob, bool large, bool direct, const HeadArgs& a, hipStream_t s) {
  return launch_head<true>(prob, large, direct, a, s);
}

}  // namespace ffmlp
