// The 8-bit linear's forward over few rows (decoding), gfx950:
//   out[M, N] = act(X W^T + P U + bias) + residual,  M <= 64
// the product of gemm_mx8.hip where the weight's bytes are all that counts.
//
// A workgroup of 8 waves takes 16 columns (16 rows of W) and all rows of X; a
// wave takes every step of 128 reduction elements in its eighth of K, straight
// from memory into the operands of one MFMA per 16 rows of X (v_mfma_scale
// 16x16x128: the weight's rows are operand A, whose 64 bytes a row come as one
// 16-byte load a lane).  No weight byte is used twice, so LDS would only add a
// trip; N / 16 workgroups of 8 waves keep enough loads in flight.  The low-rank
// term P U is split over the waves too (fp32).  X is split at |x| = 2 and
// multiplied in two parts, whose groups of eight products are exact (see
// gemm_mx8.h): the matrix instructions are not what takes the time here.  The eight partial sums meet in
// LDS and are added in order, so results do not depend on timing.
#include "ft_device.h"
#include "ft_kernels.h"

namespace ft {

namespace {
constexpr int RW = 8;                     // waves a workgroup
constexpr int RSTEPS = 4;                 // steps whose loads are in flight together

__device__ __forceinline__ float act_any(int act, float z) {
  switch (act) {
    case ACT_GELU: return act_fn<ACT_GELU>(z);
    case ACT_SILU: return act_fn<ACT_SILU>(z);
    case ACT_RELU: return act_fn<ACT_RELU>(z);
    default: return z;
  }
}
__device__ __forceinline__ uint16_t bf16_bits(float x) {
  const v2f p = {x, x};
  return (uint16_t)__builtin_bit_cast(uint32_t, __builtin_convertvector(p, v2bf));
}
}  // namespace

template <int MT>
__global__ __launch_bounds__(64 * RW) void k_rows_mx8(const uint8_t* __restrict__ X, const uint8_t* __restrict__ Xs,
                                                      const uint8_t* __restrict__ Wq, const uint8_t* __restrict__ Ws,
                                                      int M, int N, int K, const float* __restrict__ P, int R,
                                                      const uint16_t* __restrict__ U, const uint16_t* __restrict__ bias,
                                                      int act, uint16_t* z, const void* res, void* out, int out_f32) {
  __shared__ float sums[RW][MT][16][17];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16, ldw = K >> 1, nkb = K >> 5, nst = (K + 127) >> 7;
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(Wq + (size_t)n0 * ldw, (uint32_t)16 * ldw);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(X, (uint32_t)M * K);
  const __amdgpu_buffer_rsrc_t rxs = make_rsrc(Xs, (uint32_t)nst * M * 4);
  const __amdgpu_buffer_rsrc_t rws = make_rsrc(Ws + (size_t)(n0 >> 5) * nkb, (uint32_t)nkb);
  v4f acc[MT];
#pragma unroll
  for (int i = 0; i < MT; i++) acc[i] = v4f{0.f, 0.f, 0.f, 0.f};

  const int s1 = (wave + 1) * nst / RW;
#pragma unroll 1
  for (int s0 = wave * nst / RW; s0 < s1; s0 += RSTEPS) {
    v4i w[RSTEPS], x[RSTEPS][MT][2];
    int sw[RSTEPS], sx[RSTEPS][MT];
#pragma unroll
    for (int u = 0; u < RSTEPS; u++) {
      const int s = s0 + u;
      const int left = s < s1 ? K - 128 * s : 0;        // reduction elements from this step on
      const bool in = 32 * g < left;
      w[u] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rw, in ? l16 * ldw + 64 * s + 16 * g : (int)kOobOffset, 0, 0));
      sw[u] = __builtin_amdgcn_raw_buffer_load_b8(rws, in ? 4 * s + g : (int)kOobOffset, 0, 0);
#pragma unroll
      for (int i = 0; i < MT; i++) {
        const int m = 16 * i + l16;
#pragma unroll
        for (int e = 0; e < 2; e++)
          x[u][i][e] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(
              rx, 64 * e + 16 * g < left && m < M ? m * K + 128 * s + 64 * e + 16 * g : (int)kOobOffset, 0, 0));
        sx[u][i] = __builtin_amdgcn_raw_buffer_load_b8(rxs, in && m < M ? (s * M + m) * 4 + g : (int)kOobOffset, 0, 0);
      }
    }
#pragma unroll
    for (int u = 0; u < RSTEPS; u++)
#pragma unroll
      for (int i = 0; i < MT; i++) {
        const v8i a = {w[u][0], w[u][1], w[u][2], w[u][3], 0, 0, 0, 0};
        v8i low, b = {x[u][i][0][0], x[u][i][0][1], x[u][i][0][2], x[u][i][0][3],
                       x[u][i][1][0], x[u][i][1][1], x[u][i][1][2], x[u][i][1][3]};
        // (a step or row past the end has zero codes and scales: adds nothing)
        split_e4m3(b, low);
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[i], 4, 0, 0, sw[u], 0, sx[u][i]);
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, low, acc[i], 4, 0, 0, sw[u], 0, sx[u][i]);
      }
  }
  // low-rank columns j = wave, wave + 8, ...: this lane's row m of P, columns 4 g .. 4 g + 3 of U
  for (int j = wave; j < R; j += RW) {
    const v2i uu = *(const v2i*)(U + (size_t)j * N + n0 + 4 * g);
    const float u4[4] = {bf16_to_f32((uint32_t)uu[0] & 0xFFFFu), bf16_to_f32((uint32_t)uu[0] >> 16),
                         bf16_to_f32((uint32_t)uu[1] & 0xFFFFu), bf16_to_f32((uint32_t)uu[1] >> 16)};
#pragma unroll
    for (int i = 0; i < MT; i++) {
      const int m = 16 * i + l16;
      const float p = m < M ? P[(size_t)m * R + j] : 0.f;
#pragma unroll
      for (int e = 0; e < 4; e++) acc[i][e] = fmaf(p, u4[e], acc[i][e]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; i++)
#pragma unroll
    for (int e = 0; e < 4; e++) sums[wave][i][l16][4 * g + e] = acc[i][e];
  __syncthreads();
  for (int o = tid; o < 256 * MT; o += 64 * RW) {
    const int m = o >> 4, c = o & 15, n = n0 + c;
    if (m >= M) break;                                  // rows ascend with o
    float v = bias ? bf16_to_f32(bias[n]) : 0.f;
#pragma unroll
    for (int w = 0; w < RW; w++) v += sums[w][m >> 4][m & 15][c];
    const size_t at = (size_t)m * N + n;
    if (z) z[at] = bf16_bits(v);
    v = act_any(act, v);
    if (out_f32) ((float*)out)[at] = res ? v + ((const float*)res)[at] : v;
    else ((uint16_t*)out)[at] = bf16_bits(res ? v + bf16_to_f32(((const uint16_t*)res)[at]) : v);
  }
}

bool rows_mx8_better(int M, int N, int K) { return M <= kRowsMx8Max; }

hipError_t launch_rows_mx8(const MxArgs& a, int act, bool out_f32, hipStream_t st) {
#define FT_ROWS8(MT_)                                                                                                  \
  k_rows_mx8<MT_><<<a.N / 16, 64 * RW, 0, st>>>(a.x, a.xs, a.wq, a.ws, a.M, a.N, a.K, a.P, a.R, a.lr, a.bias, act, a.z, \
                                                a.res, a.out, out_f32 ? 1 : 0)
  if (a.M <= 16) FT_ROWS8(1);
  else if (a.M <= 32) FT_ROWS8(2);
  else FT_ROWS8(4);
#undef FT_ROWS8
  return hipGetLastError();
}

}  // namespace ft
