// The 8-bit linear's products with an fp32 result (see gemm_mx8.h).
#include "gemm_mx8.h"

namespace ft {

hipError_t launch_gemm_mx8_f32(bool bwd, int tile, const MxArgs& a, int act, hipStream_t st) {
  return launch_gemm_mx8_t<true>(bwd, tile, a, act, st);
}

}  // namespace ft
