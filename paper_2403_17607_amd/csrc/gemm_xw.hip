// Y = X W: k along the rows of X and across the rows of W.
#include "gemm_kernel.h"

namespace ffmlp {

hipError_t launch_gemm_xw(int tile, const GemmArgs& a, hipStream_t s) {
  if (tile == GEMM_HALF) return launch_gemm_tile<GemmHalf, false, true>(a, s);
  if (tile == GEMM_SQUARE) return launch_gemm_tile<GemmSquare, false, true>(a, s);
  if (tile == GEMM_LARGE) return launch_gemm_tile<GemmLarge, false, true>(a, s);
  if (tile == GEMM_ROWS) return launch_gemm_tile<GemmRows, false, true>(a, s);
  if (tile == GEMM_SMALL) return launch_gemm_tile<GemmSmall, false, true>(a, s);
  return launch_gemm_tile<GemmMedium, false, true>(a, s);
}

}  // namespace ffmlp
