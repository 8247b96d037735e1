// RMS norm of the residual stream with an MXFP8 output, and its gradients (gfx950).
//
//   h = bf16(x + residual);  rstd = 1 / sqrt(mean(h^2) + eps);  y = h rstd w
//   codes, scales = MXFP8(y), y unrounded (E4M3, one power of two per 32);  y in bf16
//   backward, with g = dy w and n = h rstd:
//     dx = dh + rstd (g - n mean(g n)),   dw = sum over the rows of dy n
//
// A row's elements stay in registers between the sum of squares and the
// result, so each input is read once and each output written once: both
// directions are bound by HBM.  A 32-element block lies in a lane quad, whose
// maximum takes two DPP steps; a row of 16 lanes makes the four scale bytes of
// 128 columns, which are one dword of the scales' [K / 128, M, 4].
//
// 4608 x 4096 with residual and every output moves 170 MB in 37 us, its gradients
// with dh and dw 151 MB in 34 us: 4.6 and 4.4 TB/s where a 2 GiB copy reaches
// 5.0.  One row takes 2.7 us.
#include "ft_device.h"
#include "ft_kernels.h"

namespace ft {

namespace {

// Rows in the order in which one XCD takes a contiguous range of them: the
// scale dwords of neighbouring rows share lines, which then meet in one L2.
__device__ __forceinline__ int xcd_order(int block, int blocks) {
  const int per = (blocks + 7) >> 3, t = (block & 7) * per + (block >> 3);
  return (block >> 3) < per ? t : blocks;
}

}  // namespace

// WPR waves hold a row (4 / WPR rows a workgroup), NC chunks of 8 elements a lane.
template <int NC, int WPR>
__global__ __launch_bounds__(256) void k_rmsnorm_q8(const uint16_t* x, const uint16_t* res,
                                                    const uint16_t* __restrict__ w, float eps, int rows, int K,
                                                    uint16_t* h, uint16_t* __restrict__ y, uint8_t* __restrict__ codes,
                                                    uint32_t* __restrict__ scales, float* __restrict__ rstd_out) {
  constexpr int LPR = 64 * WPR;
  __shared__ float part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = threadIdx.x % LPR;
  const int nwg = WPR == 4 ? rows : (rows + 3) / 4, block = xcd_order(blockIdx.x + kGridX * blockIdx.y, nwg);
  if (block >= nwg) return;                          // the whole workgroup
  const int row = block * (4 / WPR) + wave / WPR;
  if (WPR == 1 && row >= rows) return;
  const size_t base = (size_t)row * K;
  v4i hv[NC];
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int col = (c * LPR + lr) * 8;
    hv[c] = v4i{0, 0, 0, 0};
    if (col < K) hv[c] = *(const v4i*)(x + base + col);
  }
  if (res) {
    v4i rv[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int col = (c * LPR + lr) * 8;
      rv[c] = v4i{0, 0, 0, 0};
      if (col < K) rv[c] = *(const v4i*)(res + base + col);
    }
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int col = (c * LPR + lr) * 8;
      float a[8], b[8];
      unpack_bf16x8(hv[c], a);
      unpack_bf16x8(rv[c], b);
#pragma unroll
      for (int e = 0; e < 8; e++) a[e] += b[e];
      hv[c] = pack_bf16x8(a);                        // the stream as the next layer finds it is what is normed
      if (col < K) *(v4i*)(h + base + col) = hv[c];
    }
  }
#pragma unroll
  for (int c = 0; c < NC; c++) {
    float a[8];
    unpack_bf16x8(hv[c], a);
#pragma unroll
    for (int e = 0; e < 8; e++) ss = fmaf(a[e], a[e], ss);
  }
  ss = wave_sum(ss);
  if constexpr (WPR > 1) {
    if (lane == 0) part[wave] = ss;
    __syncthreads();
    ss = (part[0] + part[1]) + (part[2] + part[3]);
  }
  const float rstd = 1.0f / sqrtf(ss / (float)K + eps);
  if (rstd_out && lr == 0) rstd_out[row] = rstd;
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int col = (c * LPR + lr) * 8;
    float a[8], ww[8];
    unpack_bf16x8(hv[c], a);
    unpack_bf16x8(col < K ? *(const v4i*)(w + col) : v4i{0, 0, 0, 0}, ww);
#pragma unroll
    for (int e = 0; e < 8; e++) a[e] = a[e] * rstd * ww[e];
    if (y && col < K) *(v4i*)(y + base + col) = pack_bf16x8(a);
    if (codes) {
      uint32_t code;
      const v2i q = quad_mxfp8(a, code);
      const uint32_t four = row_bytes(col < K ? code : 127u, lane);
      if (col < K) {
        *(v2i*)(codes + base + col) = q;
        if ((lane & 15) == 0) scales[(size_t)(col >> 7) * rows + row] = four;
      }
    }
  }
}

hipError_t launch_rmsnorm_q8(const uint16_t* x, const uint16_t* res, const uint16_t* w, float eps, int rows, int K,
                             uint16_t* h, uint16_t* y, uint8_t* codes, uint8_t* scales, float* rstd, hipStream_t st) {
  // A workgroup a row where rows are long or too few to fill the chip with one
  // wave each.  With residual, on inputs that no cache holds: 4608 x 4096 with
  // every output 37.3 us against 49.7 on one wave a row (whose 244 registers leave
  // two waves a SIMD), 18432 x 2048 65.6 against 72.5, 4608 x 2048 20.3 against
  // 19.6; 4608 x 1024 12.8 against 11.3 and 18432 x 1024 without y 33.6 against 29.1,
  // where a workgroup's four waves would be half idle (2500 x 1024: 8.6 against 7.9).
  const bool wide = K > 2048 || rows < 4096;
  const int nc = (K + (wide ? 2047 : 511)) / (wide ? 2048 : 512);
  const int nwg = (wide ? rows : (rows + 3) / 4);
  const RowGrid rg = row_grid((unsigned)((nwg + 7) / 8 * 8));
  const dim3 grid(rg.x, rg.other);
#define FT_NORM(NC_, WPR_) \
  k_rmsnorm_q8<NC_, WPR_><<<grid, 256, 0, st>>>(x, res, w, eps, rows, K, h, y, codes, (uint32_t*)scales, rstd)
  if (wide) {
    if (nc <= 1) FT_NORM(1, 4);
    else if (nc <= 2) FT_NORM(2, 4);
    else if (nc <= 4) FT_NORM(4, 4);
    else FT_NORM(8, 4);
  } else {
    if (nc <= 2) FT_NORM(2, 1);
    else FT_NORM(4, 1);
  }
#undef FT_NORM
  return hipGetLastError();
}

// ------------------------------------------------------------------ backward
// Workgroup g takes rows (or groups of 4 rows) g, g + gridDim, ... and leaves
// its sums of dy n in parts[g][K].
template <int NC, int WPR, bool DW>
__global__ __launch_bounds__(256) void k_rmsnorm_bwd(const uint16_t* dy, const uint16_t* dh,
                                                     const uint16_t* __restrict__ h, const uint16_t* __restrict__ w,
                                                     const float* __restrict__ rstd, int rows, int K, uint16_t* dx,
                                                     float* __restrict__ parts) {
  constexpr int LPR = 64 * WPR, RPI = 4 / WPR;
  __shared__ float part[2][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = threadIdx.x % LPR;
  v4i wv[NC];
  float acc[DW ? NC : 1][8];
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int col = (c * LPR + lr) * 8;
    wv[c] = col < K ? *(const v4i*)(w + col) : v4i{0, 0, 0, 0};
    if constexpr (DW) {
#pragma unroll
      for (int e = 0; e < 8; e++) acc[c][e] = 0.f;
    }
  }
  // The next row's loads go out before this row's sum (up to 4096 columns: wider
  // rows leave no registers for it).
  constexpr bool AHEAD = NC <= 2;
  struct Row { v4i h[NC], g[NC], e[NC]; float r; };
  auto load = [&](int r0, Row& d) {
    const int row = r0 + wave / WPR;
    const bool ok = row < rows;                      // WPR == 4: whole workgroups
    const size_t base = (size_t)row * K;
    d.r = ok ? rstd[row] : 0.f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int col = (c * LPR + lr) * 8;
      d.h[c] = d.g[c] = d.e[c] = v4i{0, 0, 0, 0};
      if (ok && col < K) {
        d.h[c] = *(const v4i*)(h + base + col);
        d.g[c] = *(const v4i*)(dy + base + col);
        if (dh) d.e[c] = *(const v4i*)(dh + base + col);
      }
    }
  };
  int turn = 0;
  Row next;
  if constexpr (AHEAD) load(blockIdx.x * RPI, next);
  for (int r0 = blockIdx.x * RPI; r0 < rows; r0 += gridDim.x * RPI, turn ^= 1) {
    const int row = r0 + wave / WPR;
    const bool ok = row < rows;
    const size_t base = (size_t)row * K;
    Row cur;
    if constexpr (AHEAD) {
      cur = next;
      load(r0 + gridDim.x * RPI, next);
    } else {
      load(r0, cur);
    }
    const float r = cur.r;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
      float a[8], g[8], ww[8];
      unpack_bf16x8(cur.h[c], a);
      unpack_bf16x8(cur.g[c], g);
      unpack_bf16x8(wv[c], ww);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const float n = a[e] * r;
        if constexpr (DW) acc[c][e] = fmaf(g[e], n, acc[c][e]);
        s = fmaf(g[e] * ww[e], n, s);
      }
    }
    s = wave_sum(s);
    if constexpr (WPR > 1) {
      if (lane == 0) part[turn][wave] = s;
      __syncthreads();                               // the other turn's slots are read before the next barrier
      s = (part[turn][0] + part[turn][1]) + (part[turn][2] + part[turn][3]);
    }
    const float m = s / (float)K;
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int col = (c * LPR + lr) * 8;
      float a[8], g[8], ww[8], d[8];
      unpack_bf16x8(cur.h[c], a);
      unpack_bf16x8(cur.g[c], g);
      unpack_bf16x8(wv[c], ww);
      unpack_bf16x8(cur.e[c], d);
#pragma unroll
      for (int e = 0; e < 8; e++) d[e] = fmaf(r, fmaf(-(a[e] * r), m, g[e] * ww[e]), d[e]);
      if (ok && col < K) *(v4i*)(dx + base + col) = pack_bf16x8(d);
    }
  }
  if constexpr (DW) {
    if constexpr (WPR == 1) {
      // the four waves' sums, 512 columns (one chunk) at a time
      __shared__ float sums[4][512];
#pragma unroll
      for (int c = 0; c < NC; c++) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; e++)
          *(v4f*)&sums[wave][lane * 8 + 4 * e] = v4f{acc[c][4 * e], acc[c][4 * e + 1], acc[c][4 * e + 2], acc[c][4 * e + 3]};
        __syncthreads();
        const int j = 2 * threadIdx.x, col = c * 512 + j;
        if (col < K) {
          const v2f a = *(const v2f*)&sums[0][j], b = *(const v2f*)&sums[1][j], d = *(const v2f*)&sums[2][j],
                    f = *(const v2f*)&sums[3][j];
          *(v2f*)(parts + (size_t)blockIdx.x * K + col) = v2f{(a[0] + b[0]) + (d[0] + f[0]), (a[1] + b[1]) + (d[1] + f[1])};
        }
      }
    } else {
#pragma unroll
      for (int c = 0; c < NC; c++) {
        const int col = (c * LPR + lr) * 8;
        if (col < K) {
#pragma unroll
          for (int e = 0; e < 2; e++)
            *(v4f*)(parts + (size_t)blockIdx.x * K + col + 4 * e) =
                v4f{acc[c][4 * e], acc[c][4 * e + 1], acc[c][4 * e + 2], acc[c][4 * e + 3]};
        }
      }
    }
  }
}

// dw[k] = sum over the parts: a workgroup takes 16 columns, its 64 groups of 4
// lanes every 64th part each, all in flight together, and adds the groups in order.
__global__ __launch_bounds__(256) void k_rmsnorm_dw(const float* __restrict__ parts, int n, int K, float* __restrict__ dw) {
  __shared__ float sums[64][17];
  const int g = threadIdx.x >> 2, j = (threadIdx.x & 3) * 4, col = blockIdx.x * 16 + j;   // K % 32 == 0
  v4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = g; p < n; p += 64) s += *(const v4f*)(parts + (size_t)p * K + col);
#pragma unroll
  for (int e = 0; e < 4; e++) sums[g][j + e] = s[e];
  __syncthreads();
  if (threadIdx.x < 64) {                            // 16 groups a lane, then the four lanes of a column
    const int c = threadIdx.x & 15, q = threadIdx.x >> 4;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) t += sums[16 * q + i][c];
    t += __shfl_xor(t, 16, 64);
    t += __shfl_xor(t, 32, 64);
    if (q == 0) dw[blockIdx.x * 16 + c] = t;
  }
}

namespace {
struct BwdPlan { bool wide; int nc, groups; };
// As in the forward; 512 workgroups (two a CU) or fewer, since each leaves a row
// of partial sums.  Both launches, with dh, on inputs that no cache holds: 4608 x
// 4096 34.4 us with 512, 37.1 with 768, 39.8 with 1024; 44.1 on one wave a row, which
// 18432 x 1024 takes in 32.4 against 39.6.
BwdPlan bwd_plan(int rows, int K) {
  const bool wide = K > 2048 || rows < 2048;
  const int units = wide ? rows : (rows + 3) / 4;
  return {wide, (K + (wide ? 2047 : 511)) / (wide ? 2048 : 512), std::min(units, 512)};
}
}  // namespace

size_t rmsnorm_bwd_workspace(int rows, int K) { return (size_t)bwd_plan(rows, K).groups * K * sizeof(float); }

hipError_t launch_rmsnorm_bwd(const uint16_t* dy, const uint16_t* dh, const uint16_t* h, const uint16_t* w,
                              const float* rstd, int rows, int K, uint16_t* dx, float* dw, float* ws, hipStream_t st) {
  const BwdPlan p = bwd_plan(rows, K);
  if (rows == 0) {                                   // a sum over no rows
    if (dw) k_rmsnorm_dw<<<(unsigned)(K / 16), 256, 0, st>>>(ws, 0, K, dw);
    return hipGetLastError();
  }
#define FT_BWD(NC_, WPR_)                                                                                             \
  do {                                                                                                                \
    if (dw) k_rmsnorm_bwd<NC_, WPR_, true><<<p.groups, 256, 0, st>>>(dy, dh, h, w, rstd, rows, K, dx, ws);            \
    else k_rmsnorm_bwd<NC_, WPR_, false><<<p.groups, 256, 0, st>>>(dy, dh, h, w, rstd, rows, K, dx, nullptr);         \
  } while (0)
  if (p.wide) {
    if (p.nc <= 1) FT_BWD(1, 4);
    else if (p.nc <= 2) FT_BWD(2, 4);
    else if (p.nc <= 4) FT_BWD(4, 4);
    else FT_BWD(8, 4);
  } else {
    if (p.nc <= 2) FT_BWD(2, 1);
    else FT_BWD(4, 1);
  }
#undef FT_BWD
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !dw) return e;
  k_rmsnorm_dw<<<(unsigned)(K / 16), 256, 0, st>>>(ws, p.groups, K, dw);
  return hipGetLastError();
}

}  // namespace ft
