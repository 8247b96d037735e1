// The 8-bit linear's products with a bf16 result, and the choice of tiles (see
// gemm_mx8.h; the fp32 results are in a file of their own, compiled beside this one).
#include "gemm_mx8.h"

namespace ft {

// 32-bit offsets of the weight, a tile and the scales; the weight's scales in LDS.
bool gemm_mx8_supported(bool bwd, int M, int N, int K, int R) {
  const long NO = bwd ? K : N, KR = bwd ? N : K, lim = 1l << 31;
  return (long)N * K / 2 < lim && KR <= 65536 && NO <= 1 << 20 && (KR + 127) / 128 * 4 * M < lim && NO * std::max(R, 1) * 2 < lim;
}

// Which tile: the one whose rounds of workgroups cost least.
int gemm_mx8_tile(bool bwd, int M, int N, int K) {
  const long NO = bwd ? K : N, KR = bwd ? N : K;
  auto tiles = [&](int tm, int tn) { return ((M + tm - 1) / tm) * ((NO + tn - 1) / tn); };
  const bool big = MxGeom<256, 256>::SLOT * 3 + mx_slab(256, (int)((KR + 127) / 128)) <= kCuLdsBytes;
  const double c256 = (double)((tiles(256, 256) + 255) / 256) * 4.0;
  const double c128 = (double)((tiles(128, 128) + 255) / 256) * 1.3;
  const double c64 = (double)((tiles(64, 128) + 255) / 256) * 0.8;
  if (big && c256 <= c128 && c256 <= c64) return 256;
  return c128 <= c64 ? 128 : 64;
}

hipError_t launch_gemm_mx8(bool bwd, int tile, const MxArgs& a, int act, bool out_f32, hipStream_t st) {
  return out_f32 ? launch_gemm_mx8_f32(bwd, tile, a, act, st) : launch_gemm_mx8_bf16(bwd, tile, a, act, st);
}

hipError_t launch_gemm_mx8_bf16(bool bwd, int tile, const MxArgs& a, int act, hipStream_t st) {
  return launch_gemm_mx8_t<false>(bwd, tile, a, act, st);
}

}  // namespace ft
