// Block-scaled FP8 x FP4 GEMM (gfx950): 8-bit activations or gradients times
// the frozen MXFP4 weight, with the low-rank term, bias, activation and
// residual in the same kernel.
//   forward   out[M, N] = act(X W^T + P U + bias) + residual       (z: act's input)
//   backward  out[M, K] = (G W + Qp D^T) act'(z) + residual
// X, G: E4M3, scales [reduction / 128, M, 4];  W: E2M1 codes [N, K / 2], scales
// per 32 x 32 tile, read in transposed order by the backward.
//
// Workgroup: 4 waves in a 2x2 grid over a TM x TN tile of outputs, computed
// transposed (the weight is MFMA operand A), so that a lane holds runs of four
// columns of one output row.  Stages of 128 reduction elements (X: whole
// 128-byte rows) move through an LDS ring of NS slots by buffer loads that
// write LDS directly; the low-rank term is extra stages of the same ring (bf16
// MFMAs, P split into bf16 terms).  A stage is two MFMA steps of 64: while
// one step's products run, the other's fragments are read, one read per MFMA,
// and the loads of the stage NS further go out behind the second step's.
// The weight's scales of the whole reduction stay in LDS.
//
// Bound by the matrix cores where there are many tiles.  On three cards 18432 x
// 4096 -> 16384 with SiLU takes 950 to 980 us (2.5 to 2.6 PFLOP/s), 4608 rows with
// GELU, z and R = 64 285 to 305 (2.05 to 2.2; on one of them 281 over and over, 252
// bare, 263 with R, 257 with GELU, 251 with z).  These MFMAs from registers alone
// reach 3.8 to 4.0 PFLOP/s on random data, at which the card lowers its clock
// (4.9 on constant data).  A 256 x 256 tile takes 1.28 us
// a stage while all CUs run theirs and 0.98 alone: 3.35 PFLOP/s in the loop.  The
// rest is a tile's start and end, some 10 us, of which little can hide: with
// one wave a SIMD (128 x 128 outputs each, the fewest LDS reads per MFMA that
// the registers allow) no other wave computes meanwhile.  Eight waves a tile or
// two workgroups of 128 x 256 a CU took the same time or longer, and workgroups
// that go on to their next tile with its first stages loaded ahead took 9 % more.
// 192 x 256 tiles serve where they leave fewer CUs idle in the last round.
// Where there are fewer tiles than CUs, latency counts: tiles of 64 x 128, at
// most one a CU, are run by two groups of four waves that share the reduction
// (333 x 3168 -> 2080 in fp32 16.5 us against 18.4; 128 x 4096 -> 4096 10.4
// against 12.5; in turn on one card).  The reduction is shared no further: few
// outputs behind a long one wait for their stages (64 x 16384 -> 256 takes 28 us).
//
// An MFMA with an FP8 operand takes 64 cycles per wave and 32x32x64 products,
// twice the FP4 time.  It adds its products in groups of eight consecutive
// reduction elements, in which it drops what lies below 2^-14 of the largest
// product's power of two; the groups' sums are added in fp32.  On normal values
// that is an error of 5e-6 of the result (2-norm, at 1024 to 16384 reduction
// elements), 2e-5 with 0.5 % of channels x30 beside small values.  As a norm it is a
// hundredth of a bf16 rounding or less; of the single elements, 0.06 % and 0.3 %,
// whose terms nearly cancel, are off by more than half a bf16 step of themselves.
// X's own rounding to E4M3 is a thousand times as large (2.6e-2), so bf16 results
// take it rather than twice the matrix time.  F32 splits X in two at |x| = 2 (bit
// 6 of the code) and makes two products: at or above 2, x's last place is
// 2^-2 or more, so products are multiples of 2^-3, 2^-14 of the largest
// possible, 448 * 6; below 2 they are multiples of 2^-10 and less than 12.  Each
// group of either is then exact.
#pragma once
#include "ft_device.h"
#include "ft_kernels.h"

namespace ft {

namespace {

constexpr int XK = 128;                   // reduction elements per stage
constexpr int XLR = 32;                   // low-rank columns per stage
constexpr int kCuLdsBytes = 160 * 1024;

template <int TM, int TN>
struct MxGeom {
  static constexpr int OFF_W = TM * XK;                 // weight tile, U or D chunk
  static constexpr int OFF_S = OFF_W + TN * (XK / 2);   // scales of the X rows, 4 bytes each
  static constexpr int SLOT = OFF_S + TM * 4;
  static constexpr int XL = TM / 32, WL = TN / 64, LOADS = XL + WL + 1;   // per wave and stage
  static constexpr int WR = TM / 2, WC = TN / 2;        // rows and columns of a wave
  static constexpr int MT = WR / 32, NT = WC / 32;      // 32x32 tiles per wave
  static constexpr int STG = 4 * 2 * 32 * (64 * 4 + 16);   // the epilogue's staging rows (in the ring and the scales)
  static constexpr int NS = TM == 64 ? 4 : 3;           // ring slots
};

template <int V> struct IC8 { static constexpr int value = V; };
template <int N, class F, int I = 0>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(IC8<I>{});
    static_for<N, F, I + 1>(static_cast<F&&>(f));
  }
}

template <int SA, int SB>
__device__ __forceinline__ v16f mfma_w4x8(v4i w, v8i x, v16f c, int sw, int sx) {
  const v8i a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, x, c, 4, 0, SA, sw, SB, sx);
}

// a / b for 0 <= a < 2^30, b > 0: the quotient of the fp32 values is off by at
// most 2^-22 of itself; the remainder says by how much.  (A dozen instructions,
// where the compiler's division takes three dozen, in front of everything else.)
__device__ __forceinline__ int div_small(int a, int b) {
  int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
  int r = a - q * b;
  const int c = (int)((float)r * __builtin_amdgcn_rcpf((float)b));   // what the first quotient missed
  q += c;
  r -= c * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}

// Bytes of LDS that hold the weight's scales: TN / 32 tiles by 4 per stage.
__host__ __device__ inline int mx_slab(int tn, int nst) { return (tn / 32 * 4 * nst + 15) & ~15; }

}  // namespace

// KG groups of four waves take every KG-th stage of the reduction, each with a
// ring and accumulators of its own, which meet in LDS at the end.
template <bool BWD, int TM, int TN, int KG, int ACT, bool F32>
__global__ __launch_bounds__(256 * KG, TM > 128 ? 1 : 2) void k_gemm_mx8(
    const uint8_t* __restrict__ X, const uint8_t* __restrict__ Xs, const uint8_t* __restrict__ Wq,
    const uint8_t* __restrict__ Ws, int M, int N, int K, const float* __restrict__ P, int R,
    const uint16_t* __restrict__ LR, const uint16_t* __restrict__ bias, uint16_t* z, const void* res, void* out,
    int tiles_m, int tiles_n) {
  using G = MxGeom<TM, TN>;
  constexpr int MT = G::MT, NT = G::NT, NS = G::NS;
  extern __shared__ __attribute__((aligned(16))) uint8_t mxlds[];

  // Each XCD takes a contiguous range of tiles, four tile-rows at a time, so
  // that its 32 CUs hold some 4 x 8 tiles whose operands meet in its L2: a byte
  // of X serves 8 of them and a byte of W, half as many, 4.  (Eight tile-rows,
  // in turn on one card: 18432 x 4096 -> 16384 944 us against 925, 4608 rows 283
  // against 280.)
  const int T = tiles_m * tiles_n, per = (T + 7) >> 3;
  const int t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (t >= T || (int)(blockIdx.x >> 3) >= per) return;   // the whole workgroup
  int mt, nt;
  {
    constexpr int GM = 4;
    const int g = div_small(t, GM * tiles_n), first = g * GM, gm = min(GM, tiles_m - first), w = t - g * GM * tiles_n;
    nt = gm == GM ? w / GM : div_small(w, gm);
    mt = first + w - nt * gm;
  }
  const int m0 = mt * TM, n0 = nt * TN;
  const int NO = BWD ? K : N, KR = BWD ? N : K;
  const int nrow = min(TM, M - m0), ncol = min(TN, NO - n0);
  const int ldw = K >> 1, nwkb = K >> 5, nkb = KR >> 5;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), kg = KG == 1 ? 0 : wv >> 2, wave = wv & 3;
  const int r32 = lane & 31, h = lane >> 5, g16 = lane >> 4, t16 = lane & 15;
  const int wm = wave >> 1, wn = wave & 1;

  // Buffers start at the tile: 32-bit offsets hold any number of rows.
  const v4i rx = rsrc_words(X + (size_t)m0 * KR, (uint32_t)nrow * KR);
  const v4i rw = BWD ? rsrc_words(Wq + (n0 >> 1), (uint32_t)N * ldw - (n0 >> 1))
                     : rsrc_words(Wq + (size_t)n0 * ldw, (uint32_t)ncol * ldw);
  const int nst = (KR + XK - 1) / XK, nlr = (R + XLR - 1) / XLR, total = nst + nlr;
  const v4i rxs = rsrc_words(Xs + (size_t)m0 * 4, (uint32_t)(((size_t)(nst - 1) * M + nrow) * 4));
  uint8_t* ring = mxlds + kg * (NS * G::SLOT);
  const uint32_t lds0 = lds_addr(ring);
  const int off_slab = KG * NS * G::SLOT;

  // ---------------- per-lane load offsets within a whole stage
  const int r8 = lane >> 3, c8 = (lane & 7) ^ r8;
  uint32_t x_off[G::XL], w_off[G::WL];
  int w_pos[G::WL];                       // forward: chunk of the stage's row; backward: row of the stage
#pragma unroll
  for (int v = 0; v < G::XL; v++) {
    const int r = (wave * G::XL + v) * 8 + r8;
    x_off[v] = r < nrow ? (uint32_t)r * KR + (c8 ^ (v & 1)) * 16 : kOobOffset;
  }
#pragma unroll
  for (int v = 0; v < G::WL; v++) {
    const int ins = wave * G::WL + v;
    if constexpr (!BWD) {                 // 16 rows of 64 bytes
      const int r = 16 * ins + (lane >> 2), c = (lane & 3) ^ swz64(r);
      w_pos[v] = c;
      w_off[v] = r < ncol ? (uint32_t)r * ldw + c * 16 : kOobOffset;
    } else {                              // rows of TN / 2 bytes: the tile's columns
      constexpr int CH = TN / 32;         // chunks a row
      const int r = ins * (64 / CH) + lane / CH;
      const int c = (lane % CH) ^ (CH == 8 ? (r >> 1) & 7 : swz64(r));
      w_pos[v] = r;
      w_off[v] = c * 32 < ncol ? (uint32_t)r * ldw + c * 16 : kOobOffset;
    }
  }
  const int sseg = wave % (TM / 64);      // every wave loads scales (some the same ones): equal counts
  const uint32_t s_off = sseg * 64 + lane < nrow ? (uint32_t)(sseg * 64 + lane) * 4 : kOobOffset;

  // Load `i` of a whole stage u into the slot at `base`.
  auto load_full = [&](auto ic, int u, uint32_t base) {
    constexpr int i = decltype(ic)::value;
    if constexpr (i < G::XL) {
      dma16(rx, base + (wave * G::XL + i) * 1024, x_off[i], (uint32_t)u * XK);
    } else if constexpr (i < G::XL + G::WL) {
      constexpr int v = i - G::XL;
      dma16(rw, base + G::OFF_W + (wave * G::WL + v) * 1024, w_off[v], BWD ? (uint32_t)u * XK * ldw : (uint32_t)u * (XK / 2));
    } else {
      dma4(rxs, base + G::OFF_S + sseg * 256, s_off, (uint32_t)u * M * 4);
    }
  };
  // Load `i` of any stage: the reduction's last, partial one, a low-rank one, or none (zeros).
  auto load_any = [&](auto ic, int u, uint32_t base) {
    constexpr int i = decltype(ic)::value;
    if (u < nst) {
      if constexpr (i < G::XL) {
        dma16(rx, base + (wave * G::XL + i) * 1024, u * XK + 16 * (c8 ^ (i & 1)) < KR ? x_off[i] : kOobOffset, (uint32_t)u * XK);
      } else if constexpr (i < G::XL + G::WL) {
        constexpr int v = i - G::XL;
        const bool in = u * XK + (BWD ? w_pos[v] : 32 * w_pos[v]) < KR;
        dma16(rw, base + G::OFF_W + (wave * G::WL + v) * 1024, in ? w_off[v] : kOobOffset,
              BWD ? (uint32_t)u * XK * ldw : (uint32_t)u * (XK / 2));
      } else {
        dma4(rxs, base + G::OFF_S + sseg * 256, s_off, (uint32_t)u * M * 4);
      }
    } else {
      const int q = u - nst, left = u < total ? R - q * XLR : 0;   // low-rank columns from this stage on
      if constexpr (i < G::XL) {
        const int r = (wave * G::XL + i) * 8 + r8, c = c8 ^ (i & 1);
        const v4i rp = rsrc_words(P + (size_t)m0 * R, (uint32_t)nrow * R * 4);
        dma16(u < total ? rp : rx, base + (wave * G::XL + i) * 1024, 4 * c < left && r < nrow ? (uint32_t)r * R * 4 + c * 16 : kOobOffset,
              u < total ? (uint32_t)q * 128 : 0u);
      } else if constexpr (i < G::XL + G::WL) {
        const int ins = wave * G::WL + i - G::XL;
        uint32_t off = kOobOffset, so = 0;
        if constexpr (!BWD) {             // [32 j][TN n]
          constexpr int CH = TN / 8;
          const int j = ins * (64 / CH) + lane / CH, c = (lane % CH) ^ (2 * (j & 3));
          if (j < left && c * 8 < ncol) off = (uint32_t)j * NO * 2 + (uint32_t)(n0 + c * 8) * 2;
          so = u < total ? (uint32_t)q * XLR * NO * 2 : 0u;
        } else {                          // [TN k][32 j]
          const int k = 16 * ins + (lane >> 2), c = (lane & 3) ^ swz64(k);
          if (k < ncol && 8 * c < left) off = (uint32_t)k * R * 2 + c * 16;
          so = u < total ? (uint32_t)q * 64 : 0u;
        }
        const v4i rl = BWD ? rsrc_words(LR + (size_t)n0 * R, (uint32_t)ncol * R * 2) : rsrc_words(LR, (uint32_t)NO * R * 2);
        dma16(u < total ? rl : rw, base + G::OFF_W + ins * 1024, off, so);
      } else {
        dma4(rxs, base + G::OFF_S + sseg * 256, kOobOffset, 0);
      }
    }
  };

  // ---------------- the first stages' loads, weight scales into LDS
  // forward [TN / 32 tiles][4 nst blocks], backward [4 nst blocks][TN / 32 tiles]
  constexpr int TB = TN / 32;
  const int nfull = KR / XK;
  auto scale_dword = [&](int i) {                        // rows that are whole dwords
    uint32_t d = 0;
    if constexpr (!BWD) {
      const int j = div_small(i, nst), b = 4 * (i - j * nst), nb = (n0 >> 5) + j;
      if (i < TB * nst && nb < (N >> 5) && b < nwkb) d = *(const uint32_t*)(Ws + (size_t)nb * nwkb + b);
    } else {
      const int b = i / (TB / 4), kb = (n0 >> 5) + 4 * (i % (TB / 4));
      if (b < nkb && kb < nwkb) d = *(const uint32_t*)(Ws + (size_t)b * nwkb + kb);
    }
    return d;
  };
  const bool dwords = (nwkb & 3) == 0;
  const uint32_t first = dwords ? scale_dword(tid) : 0u;   // (in flight behind the loads below)
#pragma unroll 1
  for (int s = 0; s < NS; s++) {
    const int u = KG * s + kg;
    if (u < nfull) static_for<G::LOADS>([&](auto ic) { load_full(ic, u, lds0 + (uint32_t)s * G::SLOT); });
    else static_for<G::LOADS>([&](auto ic) { load_any(ic, u, lds0 + (uint32_t)s * G::SLOT); });
  }
  if (dwords) {
    if (tid < TB * nst) *(uint32_t*)(mxlds + off_slab + 4 * tid) = first;
    for (int i = tid + 256 * KG; i < TB * nst; i += 256 * KG) *(uint32_t*)(mxlds + off_slab + 4 * i) = scale_dword(i);
  } else {                                               // rows that are not 4-byte aligned
    for (int i = tid; i < TB * 4 * nst; i += 256 * KG) {
      const int j = BWD ? i % TB : i / (4 * nst), b = BWD ? i / TB : i - j * 4 * nst;
      const int nb = (n0 >> 5) + j;
      const bool in = b < nkb && nb < (NO >> 5);
      mxlds[off_slab + i] = in ? Ws[BWD ? (size_t)b * nwkb + nb : (size_t)nb * nwkb + b] : (uint8_t)0;
    }
  }
  v16f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; i++)
#pragma unroll
    for (int j = 0; j < NT; j++) acc[i][j] = v16f{};

  // ---------------- fragment reads, one LDS read (two for the backward's weight) an op
  const int sw_r = swz128(r32), sw_w = swz64(r32), sw_t = swz64(t16), sw_t8 = (t16 >> 1) & 7;
  struct Frags { v4i x[MT][2], w[NT]; };
  struct Scales { uint32_t x[MT], w[BWD ? 2 : NT]; };
  auto read_x = [&](auto oc, const uint8_t* base, int kk, Frags& f) {
    constexpr int i = decltype(oc)::value >> 1, e = decltype(oc)::value & 1;
    f.x[i][e] = *(const v4i*)(base + (wm * G::WR + i * 32 + r32) * XK + (((4 * kk + 2 * e + h) ^ sw_r) << 4));
  };
  auto read_w = [&](auto oc, const uint8_t* base, int kk, Frags& f) {
    constexpr int j = decltype(oc)::value;
    if constexpr (!BWD) {
      f.w[j] = *(const v4i*)(base + G::OFF_W + (wn * G::WC + j * 32 + r32) * 64 + (((2 * kk + h) ^ sw_w) << 4));
    } else {
      const int c = (wn * NT + j) ^ (TN == 256 ? sw_t8 : sw_t);
      const uint8_t* p = base + G::OFF_W + (kk * 64 + 32 * h + t16) * (TN / 2) + (c << 4) + 8 * (g16 & 1);
      const v2i lo = lds_read_tr4((const FT_LDS void*)p), hi = lds_read_tr4((const FT_LDS void*)(p + 16 * (TN / 2)));
      f.w[j] = v4i{lo[0], lo[1], hi[0], hi[1]};
    }
  };
  constexpr int XOPS = 2 * MT, FOPS = XOPS + NT, SOPS = FOPS + MT + (BWD ? 2 : NT);
  // in the last stage, bytes past the reduction's end become neutral
  uint32_t keep_last = 0;
#pragma unroll
  for (int b = 0; b < 4; b++)
    if (4 * (nst - 1) + b < nkb) keep_last |= 0xFFu << (8 * b);
  // Scale words of stage s: X and forward W byte 2 kk = block 2 kk + h; backward W[kk] byte j = tile j.
  auto read_s = [&](auto oc, const uint8_t* base, int s, Scales& f) {
    constexpr int o = decltype(oc)::value;
    if constexpr (o < MT) {
      const uint32_t keep = s == nst - 1 ? keep_last : 0xFFFFFFFFu;
      const uint32_t d = *(const uint32_t*)(base + G::OFF_S + (wm * G::WR + o * 32 + r32) * 4);
      f.x[o] = ((d & keep) | (0x7F7F7F7Fu & ~keep)) >> (8 * h);
    } else if constexpr (!BWD) {
      f.w[o - MT] = *(const uint32_t*)(mxlds + off_slab + ((wn * NT + o - MT) * nst + s) * 4) >> (8 * h);
    } else {
      const uint8_t* p = mxlds + off_slab + (4 * s + 2 * (o - MT) + h) * (TN / 32) + wn * NT;
      if constexpr (NT == 4) f.w[o - MT] = *(const uint32_t*)p;
      else f.w[o - MT] = *(const uint16_t*)p;
    }
  };
  auto read_op = [&](auto oc, const uint8_t* base, int kk, int s, Frags& f, Scales& sc) {
    constexpr int o = decltype(oc)::value;
    if constexpr (o < XOPS) read_x(oc, base, kk, f);
    else if constexpr (o < FOPS) read_w(IC8<o - XOPS>{}, base, kk, f);
    else read_s(IC8<o - FOPS>{}, base, s, sc);
  };
  v8i xb, xl;                             // row tile i of X: all of it, or (F32) its parts from 2 up and below
  auto mfma = [&](auto kc, auto tc, const Frags& f, const Scales& sc) {
    constexpr int KK = decltype(kc)::value, i = decltype(tc)::value / NT, j = decltype(tc)::value % NT;
    constexpr int SA = BWD ? j : 2 * KK, SB = 2 * KK;
    const int sw = (int)sc.w[BWD ? KK : j], sx = (int)sc.x[i];
    if constexpr (j == 0) {
      xb = v8i{f.x[i][0][0], f.x[i][0][1], f.x[i][0][2], f.x[i][0][3], f.x[i][1][0], f.x[i][1][1], f.x[i][1][2], f.x[i][1][3]};
      if constexpr (F32) split_e4m3(xb, xl);
    }
    acc[i][j] = mfma_w4x8<SA, SB>(f.w[j], xb, acc[i][j], sw, sx);
    if constexpr (F32) acc[i][j] = mfma_w4x8<SA, SB>(f.w[j], xl, acc[i][j], sw, sx);
  };

  // Stage s + 1 is published in the middle of stage s: by then this wave holds
  // all of stage s in registers, so its slot takes stage s + NS.
  auto publish = [&](auto behind) {       // that many stages may stay in flight
    wait_vm<G::LOADS * decltype(behind)::value>();
    __builtin_amdgcn_s_waitcnt(0xc07f);   // this wave's LDS reads (and writes) are done
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");        // no LDS read moves above the barrier
  };
  publish(IC8<NS - 1>{});
  Frags f0, f1;
  Scales sc;
  static_for<SOPS>([&](auto oc) { read_op(oc, ring, 0, min(kg, nst - 1), f0, sc); });
  int slot = 0;
  constexpr int MF = MT * NT;
  // The group's stages: the reduction's kg, kg + KG, ... of nst, then the low-rank ones.
  const int gfull = (nfull - kg + KG - 1) / KG, gst = (nst - kg + KG - 1) / KG, gtotal = (total - kg + KG - 1) / KG;
  // KIND of stage s + NS: 0 a whole one of X and W, 1 any other, 2 none.
  auto body = [&](int s, auto kindc) {
    const int next = slot + 1 == NS ? 0 : slot + 1;
    const uint8_t* here = ring + slot * G::SLOT;
    const uint8_t* there = ring + next * G::SLOT;
    const uint32_t dst = lds0 + (uint32_t)slot * G::SLOT;
    Scales scn;
    static_for<MF>([&](auto tc) {
      constexpr int t = decltype(tc)::value;
      mfma(IC8<0>{}, tc, f0, sc);
      static_for<(t + 1) * FOPS / MF - t * FOPS / MF>([&](auto e) {
        read_op(IC8<t * FOPS / MF + decltype(e)::value>{}, here, 1, s, f1, scn);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    constexpr int KIND = decltype(kindc)::value;
    publish(IC8<KIND == 2 ? 0 : NS - 2>{});
    const int un = min(KG * (s + 1) + kg, nst - 1);   // unused when stage s + 1 is a low-rank one
    static_for<MF>([&](auto tc) {
      constexpr int t = decltype(tc)::value;
      mfma(IC8<1>{}, tc, f1, sc);
      static_for<(t + 1) * SOPS / MF - t * SOPS / MF>([&](auto e) {
        read_op(IC8<t * SOPS / MF + decltype(e)::value>{}, there, 0, un, f0, scn);
      });
      if constexpr (KIND != 2)
        static_for<(t + 1) * G::LOADS / MF - t * G::LOADS / MF>([&](auto e) {
          constexpr int i = t * G::LOADS / MF + decltype(e)::value;
          if constexpr (KIND == 0) load_full(IC8<i>{}, KG * (s + NS) + kg, dst);
          else load_any(IC8<i>{}, KG * (s + NS) + kg, dst);
        });
      __builtin_amdgcn_sched_barrier(0);
    });
    sc = scn;
    slot = next;
  };
  int s = 0;
#pragma unroll 1
  for (; s + NS < gfull; s++) body(s, IC8<0>{});
#pragma unroll 1
  for (; s < gst && s + NS < gtotal; s++) body(s, IC8<1>{});
#pragma unroll 1
  for (; s < gst; s++) body(s, IC8<2>{});

  // ---------------- low-rank stages: 16 columns at a time, P in two bf16 terms (F32: three)
  const int jj = t16 >> 2, qq = t16 & 3;
  auto lr_half = [&](const uint8_t* base, int c) {
    v8bf b[NT];
#pragma unroll
    for (int j = 0; j < NT; j++) {
      if constexpr (!BWD) {
        const int n = wn * G::WC + j * 32 + 16 * (g16 & 1) + 4 * qq, row = 16 * c + 8 * h + jj;
        const int ch = (n >> 3) ^ (2 * (row & 3));   // row + 4 has the same swizzle
        const uint8_t* p = base + G::OFF_W + row * (TN * 2) + (ch << 4) + ((n >> 2) & 1) * 8;
        b[j] = make_v8bf(lds_read_tr16((const FT_LDS void*)p), lds_read_tr16((const FT_LDS void*)(p + 4 * TN * 2)));
      } else {
        b[j] = __builtin_bit_cast(v8bf, *(const v4i*)(base + G::OFF_W + (wn * G::WC + j * 32 + r32) * 64 + (((2 * c + h) ^ sw_w) << 4)));
      }
    }
#pragma unroll
    for (int i = 0; i < MT; i++) {
      v4f x[2];
      v4i part[F32 ? 3 : 2];              // terms of P: 16 significant bits, or 24
#pragma unroll
      for (int e = 0; e < 2; e++)
        x[e] = *(const v4f*)(base + (wm * G::WR + i * 32 + r32) * 128 + (((4 * c + 2 * h + e) ^ sw_r) << 4));
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float a = x[e >> 1][2 * (e & 1)], d = x[e >> 1][2 * (e & 1) + 1];
        uint32_t hi, lo;
        split_bf16x2(a, d, hi, lo);
        part[0][e] = (int)hi;
        part[1][e] = (int)lo;
        if constexpr (F32) {
          const v2f left = {a - __uint_as_float(hi << 16) - __uint_as_float(lo << 16),
                            d - __uint_as_float(hi & 0xFFFF0000u) - __uint_as_float(lo & 0xFFFF0000u)};
          part[2][e] = (int)__builtin_bit_cast(uint32_t, __builtin_convertvector(left, v2bf));
        }
      }
#pragma unroll
      for (int p = 0; p < (F32 ? 3 : 2); p++)
#pragma unroll
        for (int j = 0; j < NT; j++) acc[i][j] = mfma_bf16_32x32x16(b[j], __builtin_bit_cast(v8bf, part[p]), acc[i][j]);
    }
  };
#pragma unroll 1
  for (; s < gtotal; s++) {
    const uint8_t* base = ring + slot * G::SLOT;
    const int u = KG * s + kg;
    lr_half(base, 0);
    if (R - (u - nst) * XLR > 16) lr_half(base, 1);
    publish(IC8<0>{});
    if (s + NS < gtotal) static_for<G::LOADS>([&](auto ic) { load_any(ic, KG * (s + NS) + kg, lds0 + (uint32_t)slot * G::SLOT); });
    slot = slot + 1 == NS ? 0 : slot + 1;
  }
  if (KG > 1 && gtotal < (total + KG - 1) / KG) publish(IC8<0>{});   // (as many barriers in every group)
  wait_vm<0>();   // zeros of stages past the end must not land in the epilogue's LDS
  __syncthreads();
  if constexpr (KG == 2) {
    float* sums = (float*)(mxlds + G::STG) + (wave * (MT * NT * 16)) * 64 + lane;
    if (kg == 1) {
#pragma unroll
      for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++)
#pragma unroll
          for (int e = 0; e < 16; e++) sums[((i * NT + j) * 16 + e) * 64] = acc[i][j][e];
    }
    __syncthreads();
    if (kg == 1) return;
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
      for (int j = 0; j < NT; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[i][j][e] += sums[((i * NT + j) * 16 + e) * 64];
  }

  // ---------------- epilogue: 32 rows x 64 columns at a time through the wave's own LDS
  // Eight lanes hold 64 columns of a row, eight each, so that every global
  // access is a whole 128-byte line of a row (256 bytes in fp32).  Everything
  // is fp32 until the one rounding of each output.  Two staging buffers: a
  // pass's accumulators are written while the one before is on its way out, and
  // what a pass reads from memory is loaded in front of the stores of the pass
  // before (the counter that loads wait on counts stores too).  One pass's code
  // for all of them, the accumulators chosen by a switch: run once per tile,
  // unrolled code would be fetched from memory.
  constexpr int SROW = 64 * 4 + 16, PASSES = MT * NT / 2, JP = NT / 2;
  constexpr bool ZIN = BWD && ACT != ACT_NONE;
  constexpr int es = F32 ? 4 : 2;
  uint8_t* stg = mxlds + wave * (2 * 32 * SROW);
  const size_t tile0 = (size_t)m0 * NO + n0;
  const uint32_t span = (uint32_t)(nrow - 1) * NO + ncol;   // elements from the tile's first to its last
  const __amdgpu_buffer_rsrc_t ro = make_rsrc((uint8_t*)out + tile0 * es, span * es);
  const __amdgpu_buffer_rsrc_t rr = make_rsrc(res ? (const uint8_t*)res + tile0 * es : nullptr, res ? span * es : 0u);
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(bias, !BWD && bias ? (uint32_t)N * 2 : 0u);   // (no bias reads zeros)
  const __amdgpu_buffer_rsrc_t rz = make_rsrc(z ? z + tile0 : nullptr, z ? span * 2 : 0u);
  // Element offset of this lane's eight columns in the wave's first row; rows
  // past the tile's lie past the buffers' ends, columns past it are marked.
  const int lrow = lane >> 3, lcol = wn * G::WC + (lane & 7) * 8;
  auto at = [&](int pass, int it) {
    const int c = lcol + 64 * (pass % JP), r = wm * G::WR + 32 * (pass / JP) + 8 * it;
    return c < ncol ? (uint32_t)(r + lrow) * NO + c : kOobOffset;
  };
  struct Pass { v4i z[ZIN ? 4 : 1], r[4][F32 ? 2 : 1]; };
  auto load_pass = [&](int pass, Pass& d) {
    if constexpr (ZIN) {
#pragma unroll
      for (int it = 0; it < 4; it++) {
        const uint32_t a = at(pass, it);
        d.z[it] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rz, a == kOobOffset ? a : a * 2, 0, 0));
      }
    }
    if (res) {
#pragma unroll
      for (int it = 0; it < 4; it++) {
        const uint32_t a = at(pass, it), o = a == kOobOffset ? a : a * es;
        d.r[it][0] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rr, o, 0, 0));
        if constexpr (F32) d.r[it][1] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rr, o, 16, 0));
      }
    }
  };
  auto stage = [&](int pass) {
    uint8_t* to = stg + (pass & 1) * (32 * SROW) + r32 * SROW + 16 * h;
    static_for<PASSES>([&](auto pc) {
      constexpr int p = decltype(pc)::value;
      if (pass == p) {
#pragma unroll
        for (int jh = 0; jh < 2; jh++)
#pragma unroll
          for (int q = 0; q < 4; q++) {
            const v16f& a = acc[p / JP][2 * (p % JP) + jh];
            *(v4f*)(to + (32 * jh + 8 * q) * 4) = v4f{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
          }
        asm volatile("; pass %0" ::"n"(p));
      }
    });
  };
  float bf[JP][8];
#pragma unroll
  for (int jp = 0; jp < JP; jp++)
    if constexpr (!BWD)
      unpack_bf16x8(__builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rb, (n0 + lcol + 64 * jp) * 2, 0, 0)), bf[jp]);
  Pass cur, nxt;
  load_pass(0, cur);
  stage(0);
  auto run_pass = [&](int pass, auto jc) {
    __builtin_amdgcn_s_waitcnt(0xc07f);                 // the wave reads back only its own rows
    asm volatile("" ::: "memory");
    const uint8_t* from = stg + (pass & 1) * (32 * SROW) + lrow * SROW + (lane & 7) * 32;
    v4f v[4][2];
#pragma unroll
    for (int it = 0; it < 4; it++) {
      v[it][0] = *(const v4f*)(from + it * 8 * SROW);
      v[it][1] = *(const v4f*)(from + it * 8 * SROW + 16);
    }
    if (pass + 1 < PASSES) {
      load_pass(pass + 1, nxt);
      stage(pass + 1);
    }
#pragma unroll
    for (int it = 0; it < 4; it++) {
      float f[8] = {v[it][0][0], v[it][0][1], v[it][0][2], v[it][0][3], v[it][1][0], v[it][1][1], v[it][1][2], v[it][1][3]};
      const uint32_t a = at(pass, it);
      if constexpr (!BWD) {
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] += bf[decltype(jc)::value][e];
        if (z) __builtin_amdgcn_raw_buffer_store_b128(pack_bf16x8(f), rz, a == kOobOffset ? a : a * 2, 0, 0);
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] = act_fn<ACT>(f[e]);
      } else if constexpr (ZIN) {
        float zf[8];
        unpack_bf16x8(cur.z[it], zf);
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] *= act_grad<ACT>(zf[e]);
      }
      if (res) {
        float rf[8];
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 8; e++) rf[e] = __int_as_float(cur.r[it][e >> 2][e & 3]);
        } else {
          unpack_bf16x8(cur.r[it][0], rf);
        }
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] += rf[e];
      }
      const uint32_t o = a == kOobOffset ? a : a * es;
      if constexpr (F32) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, v4f{f[0], f[1], f[2], f[3]}), ro, o, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, v4f{f[4], f[5], f[6], f[7]}), ro, o, 16, 0);
      } else {
        __builtin_amdgcn_raw_buffer_store_b128(pack_bf16x8(f), ro, o, 0, 0);
      }
    }
    cur = nxt;
  };
#pragma unroll 1
  for (int i = 0; i < MT; i++) static_for<JP>([&](auto jc) { run_pass(i * JP + decltype(jc)::value, jc); });
}

template <bool F32>
hipError_t launch_gemm_mx8_t(bool bwd, int tm, const MxArgs& a, int act, hipStream_t st) {
  const int NO = bwd ? a.K : a.N, nst = ((bwd ? a.N : a.K) + XK - 1) / XK;
  const int tn = tm > 128 ? 256 : 128;
  const int tiles_m = (a.M + tm - 1) / tm, tiles_n = (NO + tn - 1) / tn;
  const unsigned grid = (unsigned)(((long)tiles_m * tiles_n + 7) / 8 * 8);
#define FT_MX(BW, TM_, TN_, KG_, ACT_)                                                                              \
  do {                                                                                                              \
    using G = MxGeom<TM_, TN_>;                                                                                     \
    const size_t sums = KG_ == 1 ? 0 : (size_t)TM_ * TN_ * 4;                                                       \
    const size_t lds = std::max((size_t)KG_ * G::NS * G::SLOT + mx_slab(TN_, nst), (size_t)G::STG + sums);          \
    k_gemm_mx8<BW, TM_, TN_, KG_, ACT_, F32><<<grid, 256 * KG_, lds, st>>>(                                         \
        a.x, a.xs, a.wq, a.ws, a.M, a.N, a.K, a.P, a.R, a.lr, a.bias, a.z, a.res, a.out, tiles_m, tiles_n);         \
  } while (0)
#define FT_MX_ACT(BW, TM_, TN_, KG_)                                   \
  do {                                                                 \
    if (act == ACT_GELU) FT_MX(BW, TM_, TN_, KG_, ACT_GELU);           \
    else if (act == ACT_SILU) FT_MX(BW, TM_, TN_, KG_, ACT_SILU);      \
    else if (act == ACT_RELU) FT_MX(BW, TM_, TN_, KG_, ACT_RELU);      \
    else FT_MX(BW, TM_, TN_, KG_, ACT_NONE);                           \
  } while (0)
  if (tm == 256) { if (!bwd) FT_MX_ACT(false, 256, 256, 1); else FT_MX_ACT(true, 256, 256, 1); }
  else if (tm == 192) { if (!bwd) FT_MX_ACT(false, 192, 256, 1); else FT_MX_ACT(true, 192, 256, 1); }
  else if (tm == 128) { if (!bwd) FT_MX_ACT(false, 128, 128, 1); else FT_MX_ACT(true, 128, 128, 1); }
  else if (tiles_m * tiles_n > 256) { if (!bwd) FT_MX_ACT(false, 64, 128, 1); else FT_MX_ACT(true, 64, 128, 1); }
  else { if (!bwd) FT_MX_ACT(false, 64, 128, 2); else FT_MX_ACT(true, 64, 128, 2); }
#undef FT_MX_ACT
#undef FT_MX
  return hipGetLastError();
}

}  // namespace ft
