// The 8-bit linear's forward over few rows (decoding), gfx950:
//   out[M, N] = act(X W^T + P U + bias) + residual,  M <= 32
// the product of gemm_mx8.hip where the weight's bytes are all that counts.
//
// A workgroup of 8 waves takes 16 to 64 columns (rows of W) and all rows of X; a
// wave takes every step of 128 reduction elements in its eighth of K, straight
// from memory into the operands of one MFMA per 16 rows of X (v_mfma_scale
// 16x16x128: the weight's rows are operand A, whose 64 bytes a row come as one
// 16-byte load a lane).  No weight byte is used twice, so LDS would only add a
// trip; N / 16 workgroups of 8 waves keep enough loads in flight.  The low-rank
// term P U is split over the waves too (fp32).  X is split at |x| = 2 and
// multiplied in two parts, whose groups of eight products are exact (see
// gemm_mx8.h): the matrix instructions are not what takes the time here.  The
// eight partial sums meet in LDS and are added in order, so results do not
// depend on timing.
//
// Bound by the weight's bytes and by one pass of latency: 16 x 4096 -> 16384
// (34 MB of weight) takes 11 us, 3 TB/s; 1 x 4096 -> 4096 (8.5 MB) 5.1.
#include "ft_device.h"
#include "ft_kernels.h"

namespace ft {

namespace {
constexpr int RW = 8;                     // waves a workgroup

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

template <int MT, int NT>
__global__ __launch_bounds__(64 * RW) void k_rows_mx8(const uint8_t* __restrict__ X, const uint8_t* __restrict__ Xs,
                                                      const uint8_t* __restrict__ Wq, const uint8_t* __restrict__ Ws,
                                                      int M, int N, int K, const float* __restrict__ P, int R,
                                                      const uint16_t* __restrict__ U, const uint16_t* __restrict__ bias,
                                                      int act, uint16_t* z, const void* res, void* out, int out_f32) {
  constexpr int RSTEPS = MT == 1 || MT * NT <= 2 ? 4 : 2;   // steps whose loads are in flight together
  constexpr int WN = 16 * NT;                           // columns of the workgroup
  __shared__ float sums[RW][MT * 16][WN + 1];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * WN, ldw = K >> 1, nkb = K >> 5, nst = (K + 127) >> 7;
  const int ncol = min(WN, N - n0);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(Wq + (size_t)n0 * ldw, (uint32_t)ncol * ldw);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(X, (uint32_t)M * K);
  const __amdgpu_buffer_rsrc_t rxs = make_rsrc(Xs, (uint32_t)nst * M * 4);
  const __amdgpu_buffer_rsrc_t rws = make_rsrc(Ws + (size_t)(n0 >> 5) * nkb, (uint32_t)((ncol + 31) >> 5) * nkb);
  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; i++)
#pragma unroll
    for (int j = 0; j < NT; j++) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

  const int s1 = (wave + 1) * nst / RW;
#pragma unroll 1
  for (int s0 = wave * nst / RW; s0 < s1; s0 += RSTEPS) {
    v4i w[RSTEPS][NT], x[RSTEPS][MT][2];
    int sw[RSTEPS][(NT + 1) / 2], sx[RSTEPS][MT];
#pragma unroll
    for (int u = 0; u < RSTEPS; u++) {
      const int s = s0 + u;
      const int left = s < s1 ? K - 128 * s : 0;        // reduction elements from this step on
      const bool in = 32 * g < left;
      // (columns past the last lie past the weight's end and read zeros)
#pragma unroll
      for (int j = 0; j < NT; j++)
        w[u][j] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(
            rw, in ? (16 * j + l16) * ldw + 64 * s + 16 * g : (int)kOobOffset, 0, 0));
#pragma unroll
      for (int j = 0; j < (NT + 1) / 2; j++)            // one scale row per 32 columns
        sw[u][j] = __builtin_amdgcn_raw_buffer_load_b8(rws, in ? j * nkb + 4 * s + g : (int)kOobOffset, 0, 0);
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
        // (a step or row past the end has zero codes and scales: adds nothing)
        v8i low, b = {x[u][i][0][0], x[u][i][0][1], x[u][i][0][2], x[u][i][0][3],
                      x[u][i][1][0], x[u][i][1][1], x[u][i][1][2], x[u][i][1][3]};
        split_e4m3(b, low);
#pragma unroll
        for (int j = 0; j < NT; j++) {
          const v8i a = {w[u][j][0], w[u][j][1], w[u][j][2], w[u][j][3], 0, 0, 0, 0};
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[i][j], 4, 0, 0, sw[u][j / 2], 0, sx[u][i]);
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, low, acc[i][j], 4, 0, 0, sw[u][j / 2], 0, sx[u][i]);
        }
      }
  }
  // low-rank columns r = wave, wave + 8, ...: this lane's rows m of P, columns 16 j + 4 g .. + 3 of U
  for (int r = wave; r < R; r += RW) {
    float p[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) p[i] = 16 * i + l16 < M ? P[(size_t)(16 * i + l16) * R + r] : 0.f;
#pragma unroll
    for (int j = 0; j < NT; j++) {
      const int n = 16 * j + 4 * g;
      v2i uu = {0, 0};
      if (n < ncol) uu = *(const v2i*)(U + (size_t)r * N + n0 + n);
      const float u4[4] = {bf16_to_f32((uint32_t)uu[0] & 0xFFFFu), bf16_to_f32((uint32_t)uu[0] >> 16),
                           bf16_to_f32((uint32_t)uu[1] & 0xFFFFu), bf16_to_f32((uint32_t)uu[1] >> 16)};
#pragma unroll
      for (int i = 0; i < MT; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) acc[i][j][e] = fmaf(p[i], u4[e], acc[i][j][e]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; i++)
#pragma unroll
    for (int j = 0; j < NT; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) sums[wave][16 * i + l16][16 * j + 4 * g + e] = acc[i][j][e];
  __syncthreads();
  for (int o = tid; o < MT * 16 * WN; o += 64 * RW) {
    const int m = o / WN, c = o % WN, n = n0 + c;
    if (m >= M) break;                                  // rows ascend with o
    if (c >= ncol) continue;
    float v = bias ? bf16_to_f32(bias[n]) : 0.f;
#pragma unroll
    for (int w = 0; w < RW; w++) v += sums[w][m][c];
    const size_t at = (size_t)m * N + n;
    if (z) z[at] = bf16_bits(v);
    v = act_any(act, v);
    if (out_f32) ((float*)out)[at] = res ? v + ((const float*)res)[at] : v;
    else ((uint16_t*)out)[at] = bf16_bits(res ? v + bf16_to_f32(((const uint16_t*)res)[at]) : v);
  }
}

// Against the tile kernel (64 x 128 tiles), us a call, M x K -> N: 16 x 4096 -> 16384
// 10.9 against 12.7, 16 x 16384 -> 4096 14 against 29, 32 x 4096 -> 4096 9.4 against
// 11.1; but every workgroup reads X, in rows of 128 bytes a step: 64 x 4096 -> 4096
// took 16 against 11.
bool rows_mx8_better(int M, int N) { return M <= 16 || (M <= kRowsMx8Max && N <= 8192); }

hipError_t launch_rows_mx8(const MxArgs& a, int act, bool out_f32, hipStream_t st) {
  // Columns a workgroup: 16 while that makes no more workgroups than CUs, then
  // 32 and, up to 16 rows, 64, which read X half and a quarter as often (X is read
  // by every one).  More rows come with at most 8192 columns (rows_mx8_better).
  const int wgs = a.N / 16, nt = wgs <= 256 ? 1 : wgs <= 512 ? 2 : 4;
#define FT_ROWS8(MT_, NT_)                                                                                      \
  k_rows_mx8<MT_, NT_><<<(a.N + 16 * NT_ - 1) / (16 * NT_), 64 * RW, 0, st>>>(                                  \
      a.x, a.xs, a.wq, a.ws, a.M, a.N, a.K, a.P, a.R, a.lr, a.bias, act, a.z, a.res, a.out, out_f32 ? 1 : 0)
  if (a.M <= 16) {
    if (nt == 1) FT_ROWS8(1, 1);
    else if (nt == 2) FT_ROWS8(1, 2);
    else FT_ROWS8(1, 4);
  } else {
    if (nt == 1) FT_ROWS8(2, 1);
    else FT_ROWS8(2, 2);
  }
#undef FT_ROWS8
  return hipGetLastError();
}

}  // namespace ft
