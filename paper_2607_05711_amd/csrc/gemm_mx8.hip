// The 8-bit linear's products with a bf16 result, and the choice of tiles (see
// gemm_mx8.h; the fp32 results are in a file of their own, compiled beside this one).
#include "gemm_mx8.h"

namespace ft {

// 32-bit offsets of the weight, a tile and the scales; the weight's scales in
// LDS; fewer than 2^24 workgroups of 256 threads (see row_grid): 2^39 outputs are
// 1.4 * 2^23 tiles of 192x256, and the rule takes smaller ones only for outputs of
// up to 128 columns, whose rows end below 2^29, and for reductions whose weight
// leaves them fewer than 2^16 columns by 2^20 rows.
bool gemm_mx8_supported(bool bwd, int M, int N, int K, int R) {
  const long NO = bwd ? K : N, KR = bwd ? N : K, lim = 1l << 31;
  return (long)N * K / 2 < lim && KR <= 65536 && NO <= 1 << 20 && (KR + 127) / 128 * 4 * M < lim &&
         NO * std::max(R, 1) * 2 < lim && M * NO < 1l << 39;
}

// Which tile: the one of the least estimated time, in microseconds: rounds of
// workgroups (one a CU on the wide tiles, two on the others, whose last round
// may be of one) of a fixed part, the tile's start and end, and one per stage.
// Forward in bf16, the bare product over and over, measured and estimated, M x K ->
// N, 256x256 / 192x256 / 128x128 / 64x128:
//   4608 x 4096 -> 16384   256 / 243 / 272 / 329    232 / 221 / 275 / 360
//   4608 x 16384 -> 4096   311 / 244 / 264 / 309    323 / 252 / 274 / 298
//   18432 x 4096 -> 16384  906 / 954 / 1077 / 1351  835 / 882 / 1100 / 1440
//   2048 x 4096 -> 4096    47 / 38 / 33 / 41        46 / 37 / 31 / 40
//   512 x 4096 -> 4096     41 / 32 / 19 / 13        46 / 37 / 17 / 11
// The input gradient is within a tenth of these.  fp32 results have twice the
// matrix time and the same order, so the estimate serves them too: 446 / 418 / 445 /
// 509, 608 / 459 / 448 / 469 (the choice of 192 costs 2 %), 1652 / 1671 / 1822 / 2033,
// 88 / 70 / 56 / 63, 80 / 63 / 33 / 20.  The low-rank term's stages weigh the same on all.
int gemm_mx8_tile(bool bwd, int M, int N, int K) {
  const long NO = bwd ? K : N, nst = ((bwd ? N : K) + 127) / 128;
  const struct { int tm, tn, cap; double fix, stage, fix1, stage1; size_t slot; } t[] = {
      {256, 256, 256, 8.0, 1.2, 8.0, 1.2, MxGeom<256, 256>::SLOT},
      {192, 256, 256, 7.0, 0.93, 7.0, 0.93, MxGeom<192, 256>::SLOT},
      {128, 128, 512, 4.0, 0.83, 5.0, 0.38, 0},
      {64, 128, 512, 4.0, 0.5, 5.5, 0.16, 0}};
  int best = 64;
  double least = 1e30;
  for (const auto& g : t) {
    if (g.slot * 3 + mx_slab(g.tn, (int)nst) > (size_t)kCuLdsBytes) continue;
    const long n = ((M + g.tm - 1) / g.tm) * ((NO + g.tn - 1) / g.tn), full = n / g.cap, rest = n % g.cap;
    const double time = full * (g.fix + g.stage * nst) +
                        (rest == 0 ? 0.0 : rest <= 256 ? g.fix1 + g.stage1 * nst : g.fix + g.stage * nst);
    if (time < least) { least = time; best = g.tm; }
  }
  return best;
}

hipError_t launch_gemm_mx8(bool bwd, int tile, const MxArgs& a, int act, bool out_f32, hipStream_t st) {
  return out_f32 ? launch_gemm_mx8_f32(bwd, tile, a, act, st) : launch_gemm_mx8_bf16(bwd, tile, a, act, st);
}

hipError_t launch_gemm_mx8_bf16(bool bwd, int tile, const MxArgs& a, int act, hipStream_t st) {
  return launch_gemm_mx8_t<false>(bwd, tile, a, act, st);
}

}  // namespace ft
