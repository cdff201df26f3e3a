// dX = dZ W^T: k along the rows of both sides.
#include "gemm_kernel.h"

namespace ffmlp {

hipError_t launch_gemm_dx(int tile, bool direct, const GemmArgs& a, hipStream_t s) {
  if (direct) {
    if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, false, false, true>(a, s);
    if (tile == GEMM_MEDIUM) return launch_gemm_tile<GemmMedium, false, false, true>(a, s);
    return launch_gemm_tile<GemmRows, false, false, true>(a, s);
  }
  if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, false, false, false>(a, s);
  if (tile == GEMM_MEDIUM) return launch_gemm_tile<GemmMedium, false, false, false>(a, s);
  return launch_gemm_tile<GemmRows, false, false, false>(a, s);
}

}  // namespace ffmlp
