// dX = dZ W^T: k along the rows of both sides.
#include "gemm_kernel.h"

namespace ffmlp {

hipError_t launch_gemm_dx(int tile, const GemmArgs& a, hipStream_t s) {
  if (tile == GEMM_HALF) return launch_gemm_tile<GemmHalf, false, false>(a, s);
  if (tile == GEMM_SQUARE) return launch_gemm_tile<GemmSquare, false, false>(a, s);
  if (tile == GEMM_ROWS) return launch_gemm_tile<GemmRows, false, false>(a, s);
  if (tile == GEMM_SMALL) return launch_gemm_tile<GemmSmall, false, false>(a, s);
  return launch_gemm_tile<GemmMedium, false, false>(a, s);
}

}  // namespace ffmlp
