// dW = X^T dZ: k (the batch) across the rows of both sides.
#include "gemm_kernel.h"

namespace ffmlp {

hipError_t launch_gemm_dw(int tile, const GemmArgs& a, hipStream_t s) {
  if (tile == GEMM_HALF) return launch_gemm_tile<GemmHalf, true, true>(a, s);
  if (tile == GEMM_SQUARE) return launch_gemm_tile<GemmSquare, true, true>(a, s);
  if (tile == GEMM_SMALL) return launch_gemm_tile<GemmSmall, true, true>(a, s);
  return launch_gemm_tile<GemmMedium, true, true>(a, s);
}

}  // namespace ffmlp
