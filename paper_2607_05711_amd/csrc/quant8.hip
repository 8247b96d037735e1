// MXFP8 quantization of bf16 rows (gfx950): E4M3 codes [rows, cols] and one
// power-of-two scale per 32 elements, [cols / 128, rows, 4]; optionally of a
// gradient on its way through an activation, src act'(z), which is stored in
// bf16 too.  (With a low-rank projection: the streaming kernel of
// quant_proj.hip.)
//
// Bound by HBM: src (and z) read once, codes, scales (and v) written once.  A
// workgroup takes 16 rows x 512 columns, a wave one row at a time, 8 elements a
// lane, so that all of the workgroup's loads are in flight together and every
// access is a run of 512 bytes or more of a row.  The scale dwords (four
// blocks, 128 columns) of 16 rows meet in LDS and leave as runs of 64 bytes.
// 1111 x 11264 through SiLU' moves 88 MB in 16.9 us, 5.2 TB/s (a 2 GiB copy: 5.0;
// some of this fits the last-level cache).
#include "ft_device.h"
#include "ft_kernels.h"

namespace ft {

namespace {
constexpr int Q8_ROWS = 16, Q8_COLS = 512;
}

template <int ACT, bool Z>
__global__ __launch_bounds__(256) void k_quant8(const uint16_t* src, const uint16_t* __restrict__ z, int rows, int cols,
                                                uint16_t* v, uint8_t* __restrict__ codes, uint32_t* __restrict__ scales) {
  __shared__ uint32_t sc[4][Q8_ROWS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row0 = (blockIdx.x + kGridX * blockIdx.z) * Q8_ROWS, col = blockIdx.y * Q8_COLS + lane * 8;
  constexpr int T = Q8_ROWS / 4;
  v4i x[T], zv[T];
#pragma unroll
  for (int t = 0; t < T; t++) {
    const int row = row0 + 4 * t + wave;
    x[t] = zv[t] = v4i{0, 0, 0, 0};
    if (row < rows && col < cols) {
      x[t] = *(const v4i*)(src + (size_t)row * cols + col);
      if constexpr (Z) zv[t] = *(const v4i*)(z + (size_t)row * cols + col);
    }
  }
#pragma unroll
  for (int t = 0; t < T; t++) {
    const int row = row0 + 4 * t + wave;
    const bool ok = row < rows && col < cols;
    const size_t at = (size_t)row * cols + col;
    float f[8];
    unpack_bf16x8(x[t], f);
    if constexpr (Z) {
      float zf[8];
      unpack_bf16x8(zv[t], zf);
#pragma unroll
      for (int e = 0; e < 8; e++) f[e] *= act_grad<ACT>(zf[e]);
      if (ok && v) *(v4i*)(v + at) = pack_bf16x8(f);
    }
    uint32_t code;
    const v2i q = quad_mxfp8(f, code);
    if (ok) *(v2i*)(codes + at) = q;
    const uint32_t four = row_bytes(col < cols ? code : 127u, lane);
    if ((lane & 15) == 0) sc[lane >> 4][4 * t + wave] = four;
  }
  __syncthreads();
  if (threadIdx.x < 4 * Q8_ROWS) {
    const int g = blockIdx.y * 4 + threadIdx.x / Q8_ROWS, row = row0 + threadIdx.x % Q8_ROWS;
    if (row < rows && g * 128 < cols) scales[(size_t)g * rows + row] = sc[threadIdx.x / Q8_ROWS][threadIdx.x % Q8_ROWS];
  }
}

hipError_t launch_quant8(const uint16_t* src, const uint16_t* z, int act, int rows, int cols, uint16_t* v, uint8_t* codes,
                         uint8_t* scales, hipStream_t st) {
  const RowGrid rg = row_grid((unsigned)(rows + Q8_ROWS - 1) / Q8_ROWS);
  const dim3 grid(rg.x, (cols + Q8_COLS - 1) / Q8_COLS, rg.other);
#define FT_Q8(ACT_, Z_) k_quant8<ACT_, Z_><<<grid, 256, 0, st>>>(src, z, rows, cols, v, codes, (uint32_t*)scales)
  if (!z) FT_Q8(ACT_NONE, false);
  else if (act == ACT_GELU) FT_Q8(ACT_GELU, true);
  else if (act == ACT_SILU) FT_Q8(ACT_SILU, true);
  else FT_Q8(ACT_RELU, true);
#undef FT_Q8
  return hipGetLastError();
}

}  // namespace ft
