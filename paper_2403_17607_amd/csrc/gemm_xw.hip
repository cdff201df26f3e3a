// Y = X W: k along the rows of X and across the rows of W.
#include "gemm_kernel.h"

namespace ffmlp {

hipError_t launch_gemm_xw(int tile, bool direct, const GemmArgs& a, hipStream_t s) {
  if (direct) {
    if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, false, true, true>(a, s);
    if (tile == GEMM_MEDIUM) return launch_gemm_tile<GemmMedium, false, true, true>(a, s);
    return launch_gemm_tile<GemmRows, false, true, true>(a, s);
  }
  if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, false, true, false>(a, s);
  if (tile == GEMM_MEDIUM) return launch_gemm_tile<GemmMedium, false, true, false>(a, s);
  return launch_gemm_tile<GemmRows, false, true, false>(a, s);
}

}  // namespace ffmlp
