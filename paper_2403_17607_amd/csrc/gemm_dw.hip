// dW = X^T dZ: k (the batch) across the rows of both sides.
#include "gemm_kernel.h"

namespace ffmlp {

hipError_t launch_gemm_dw(int tile, bool direct, const GemmArgs& a, hipStream_t s) {
  if (direct) {
    if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, true, true, true>(a, s);
    return launch_gemm_tile<GemmMedium, true, true, true>(a, s);
  }
  if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, true, true, false>(a, s);
  return launch_gemm_tile<GemmMedium, true, true, false>(a, s);
}

}  // namespace ffmlp
