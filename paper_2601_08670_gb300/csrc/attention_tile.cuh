// attention_tile.cuh -- the math of one warp on a 64-key tile of K and V, and the
// merge of a CTA's eight warps: shared by the kernels of slab and of paged caches.
#pragma once
#include <math.h>

#include "attention.cuh"

namespace pced {

template <int D>
struct AttCfg {
  static constexpr int BOXES = D / 64;                  // 64-element TMA boxes per row
  static constexpr int BOX_BYTES = ATT_BLOCK_N * 128;   // 64 rows x 128 B
  static constexpr int TILE_BYTES = BOXES * BOX_BYTES;  // K (or V) part of a stage
  static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
  static constexpr int STAGES = D == 128 ? 5 : 7;       // odd: consecutive uses of a stage alternate warpgroups
  static constexpr int KSTEPS = D / 16;
  static constexpr int MTILES = D / 16;
  static constexpr int OROW = D + 4;                    // padded row (one head of one warp) of a piece's partials
  static constexpr int PARTIALS = 2 * ATT_CONSUMERS * ATT_MAX_G + ATT_CONSUMERS * ATT_MAX_G * OROW;  // floats, G = 8
  static constexpr size_t BARS = (2 * STAGES + 2) * 8;
  // one-layer kernel: stages, barriers, partials, pre[S+1], lens / row0 / cap [S]
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE_BYTES + BARS + (size_t)PARTIALS * 4 +
                                 (ATT_MAX_S + 1) * 8 + 3 * ATT_MAX_S * 4 + 128;
};

// ------------------------------------------------------------ consumer math
// Online-softmax state of one consumer warp over its keys of a piece.
template <int D>
struct WarpAcc {
  float m0, m1, l0, l1;  // heads 2tq and 2tq+1 of this thread
  float o[D / 16][4];    // O^T fragments: dims 16i + g (+8), heads 2tq, 2tq+1
};

template <int D>
__device__ __forceinline__ void acc_reset(WarpAcc<D>& A) {
  A.m0 = A.m1 = -INFINITY;
  A.l0 = A.l1 = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) A.o[i][0] = A.o[i][1] = A.o[i][2] = A.o[i][3] = 0.f;
}

// This warp's 16 keys [kb, kb+16) of the 64-key K/V tiles at sk / sv (TMA
// 128-byte swizzle, D/64 boxes of 64 rows x 128 B); keys at or past nvalid
// are masked.  qf: B operand of S^T = K Q^T (dims x heads).
//
// P enters the P V product as bf16 hi + lo parts.  With PK (at most four
// heads) both parts share one MMA: accumulator columns 0-3 take the hi parts
// of heads 0-3 and columns 4-7 the lo parts of the same heads (qf repeats
// heads 0-3 in columns 4-7, so the threads owning those columns, tq >= 2,
// hold the same scores as lane ^ 2), and o of head h is column h plus column
// h + 4 (summed once per piece, see pack_fold).  With P3 a third part follows, in an
// MMA of its own, so P keeps the 24 bits it was computed with, and a tile's sums
// are added to o in fp32, rounded to nearest (the MMA's own accumulation cuts
// off): error of the output against 64 bits 2.4e-6 without, 1.7e-7 with it, the time
// of memory-bound calls the same.
template <int D, bool PK = false, bool P3 = false>
__device__ __forceinline__ void tile_math(WarpAcc<D>& A, const uint32_t (&qf)[D / 16][2], uint32_t sk, uint32_t sv,
                                          int kb, int nvalid, float scale_log2, int lane) {
  using C = AttCfg<D>;
  const int g = lane >> 2, tq = lane & 3, mat = lane >> 3, mr = lane & 7;
  // ---- scores S^T (16 keys x 8 heads), four independent accumulation chains
  float sc4[4][4] = {};
  {
    const int key = kb + (mat & 1) * 8 + mr;
    const uint32_t rowa = sk + key * 128;
    const uint32_t sw = key & 7;
#pragma unroll
    for (int j = 0; j < C::KSTEPS; ++j) {
      const int chunk = 2 * j + (mat >> 1);
      const uint32_t addr = rowa + (chunk >> 3) * C::BOX_BYTES + (((chunk & 7) ^ sw) << 4);
      uint32_t a0, a1, a2, a3;
      ldsm_x4(addr, a0, a1, a2, a3);
      mma_bf16(sc4[j & 3], a0, a1, a2, a3, qf[j][0], qf[j][1]);
    }
  }
  const bool v0 = kb + g < nvalid, v1 = kb + g + 8 < nvalid;
  const float s0 = v0 ? ((sc4[0][0] + sc4[1][0]) + (sc4[2][0] + sc4[3][0])) * scale_log2 : -INFINITY;
  const float s1 = v0 ? ((sc4[0][1] + sc4[1][1]) + (sc4[2][1] + sc4[3][1])) * scale_log2 : -INFINITY;
  const float s2 = v1 ? ((sc4[0][2] + sc4[1][2]) + (sc4[2][2] + sc4[3][2])) * scale_log2 : -INFINITY;
  const float s3 = v1 ? ((sc4[0][3] + sc4[1][3]) + (sc4[2][3] + sc4[3][3])) * scale_log2 : -INFINITY;
  // The reference max only moves when a score exceeds it by more than
  // ATT_RESCALE_SLACK (log2 units): exp2 of the others stays below
  // 2^ATT_RESCALE_SLACK, and the rescale of o, l (and the max reduction across
  // the warp) is skipped for most tiles.  Any reference gives the same o / l.
  float x0 = fmaxf(s0, s2), x1 = fmaxf(s1, s3);
  if (__any_sync(0xffffffffu, x0 > A.m0 + ATT_RESCALE_SLACK || x1 > A.m1 + ATT_RESCALE_SLACK)) {
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) {
      x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, off));
      x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, off));
    }
    const float n0 = fmaxf(A.m0, x0), n1 = fmaxf(A.m1, x1);
    const float al0 = A.m0 == -INFINITY ? 0.f : exp2f(A.m0 - n0);
    const float al1 = A.m1 == -INFINITY ? 0.f : exp2f(A.m1 - n1);
    A.l0 *= al0;
    A.l1 *= al1;
#pragma unroll
    for (int i = 0; i < C::MTILES; ++i) {
      A.o[i][0] *= al0;
      A.o[i][2] *= al0;
      A.o[i][1] *= al1;
      A.o[i][3] *= al1;
    }
    A.m0 = n0;
    A.m1 = n1;
  }
  const float u0 = A.m0 == -INFINITY ? 0.f : A.m0, u1 = A.m1 == -INFINITY ? 0.f : A.m1;
  const float p0 = exp2f(s0 - u0), p1 = exp2f(s1 - u1), p2 = exp2f(s2 - u0), p3 = exp2f(s3 - u1);
  A.l0 += p0 + p2;
  A.l1 += p1 + p3;
  // ---- P^T as the B operand (keys x heads), split into bf16 hi + lo
  const uint32_t h01 = pack_bf16(p0, p1), h23 = pack_bf16(p2, p3);
  const uint32_t q01 = pack_bf16(p0 - bf16_lo(h01), p1 - bf16_hi(h01));
  const uint32_t q23 = pack_bf16(p2 - bf16_lo(h23), p3 - bf16_hi(h23));
  const bool lo_cols = PK && tq >= 2;
  const uint32_t bh0 = movmatrix_t(lo_cols ? q01 : h01), bh1 = movmatrix_t(lo_cols ? q23 : h23);
  const uint32_t bl0 = PK ? 0u : movmatrix_t(q01), bl1 = PK ? 0u : movmatrix_t(q23);
  uint32_t bt0 = 0u, bt1 = 0u;
  if (P3) {
    const uint32_t t01 = pack_bf16((p0 - bf16_lo(h01)) - bf16_lo(q01), (p1 - bf16_hi(h01)) - bf16_hi(q01));
    const uint32_t t23 = pack_bf16((p2 - bf16_lo(h23)) - bf16_lo(q23), (p3 - bf16_hi(h23)) - bf16_hi(q23));
    bt0 = movmatrix_t(lo_cols ? 0u : t01);
    bt1 = movmatrix_t(lo_cols ? 0u : t23);
  }
  // ---- O^T += V^T P^T; rows of V past the live length are zeroed
  const bool partial = kb + 16 > nvalid;
  const int klo = kb + 2 * tq, khi = klo + 8;
  const int key = kb + (mat >> 1) * 8 + mr;
  const uint32_t rowa = sv + key * 128;
  const uint32_t sw = key & 7;
#pragma unroll
  for (int i = 0; i < C::MTILES; ++i) {
    const int chunk = 2 * i + (mat & 1);
    const uint32_t addr = rowa + (chunk >> 3) * C::BOX_BYTES + (((chunk & 7) ^ sw) << 4);
    uint32_t a0, a1, a2, a3;
    ldsm_x4_t(addr, a0, a1, a2, a3);
    if (partial) {
      const uint32_t mlo = (klo < nvalid ? 0xFFFFu : 0u) | (klo + 1 < nvalid ? 0xFFFF0000u : 0u);
      const uint32_t mhi = (khi < nvalid ? 0xFFFFu : 0u) | (khi + 1 < nvalid ? 0xFFFF0000u : 0u);
      a0 &= mlo;
      a1 &= mlo;
      a2 &= mhi;
      a3 &= mhi;
    }
    if (P3) {
      float t[4] = {};
      mma_bf16(t, a0, a1, a2, a3, bt0, bt1);
      if (!PK) mma_bf16(t, a0, a1, a2, a3, bl0, bl1);
      mma_bf16(t, a0, a1, a2, a3, bh0, bh1);
#pragma unroll
      for (int j = 0; j < 4; ++j) A.o[i][j] += t[j];
    } else {
      mma_bf16(A.o[i], a0, a1, a2, a3, bh0, bh1);
      if (!PK) mma_bf16(A.o[i], a0, a1, a2, a3, bl0, bl1);
    }
  }
}

// After tile_math<D, true>: o of heads 2tq, 2tq+1 in the threads with tq < 2
// (hi columns plus the lo columns held by lane ^ 2).
template <int D>
__device__ __forceinline__ void pack_fold(WarpAcc<D>& A) {
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) A.o[i][j] += __shfl_xor_sync(0xffffffffu, A.o[i][j], 2);
}

// This warp's partial of a piece (o, running max, sum) into shared memory:
// ms, ls [ATT_MAX_G][8 warps], os [8 warps][G][D + 4].
template <int D>
__device__ __forceinline__ void store_partial(const WarpAcc<D>& A, float* ms, float* ls, float* os, int G, int warp,
                                              int lane) {
  using C = AttCfg<D>;
  const int g = lane >> 2, tq = lane & 3;
  float l0 = A.l0, l1 = A.l1;
#pragma unroll
  for (int off = 4; off < 32; off <<= 1) {
    l0 += __shfl_xor_sync(0xffffffffu, l0, off);
    l1 += __shfl_xor_sync(0xffffffffu, l1, off);
  }
  if (g == 0) {
    ms[(2 * tq) * ATT_CONSUMERS + warp] = A.m0;
    ms[(2 * tq + 1) * ATT_CONSUMERS + warp] = A.m1;
    ls[(2 * tq) * ATT_CONSUMERS + warp] = l0;
    ls[(2 * tq + 1) * ATT_CONSUMERS + warp] = l1;
  }
  float* ow = os + warp * G * C::OROW;
  const bool h0 = 2 * tq < G, h1 = 2 * tq + 1 < G;
#pragma unroll
  for (int i = 0; i < C::MTILES; ++i) {
    const int d0 = 16 * i + g, d1 = d0 + 8;
    if (h0) {
      ow[(2 * tq) * C::OROW + d0] = A.o[i][0];
      ow[(2 * tq) * C::OROW + d1] = A.o[i][2];
    }
    if (h1) {
      ow[(2 * tq + 1) * C::OROW + d0] = A.o[i][1];
      ow[(2 * tq + 1) * C::OROW + d1] = A.o[i][3];
    }
  }
}

// The eight warps' partials combined for outputs idx0 .. idx0 + 3 (head hh):
// running max mx (log2 units), sum lsum and unnormalised output acc.
template <int D>
__device__ __forceinline__ void load_merged(const float* ms, const float* ls, const float* os, int G, int hh, int idx0,
                                            float& mx, float& lsum, float (&acc)[4]) {
  using C = AttCfg<D>;
  float mw[ATT_CONSUMERS], lw[ATT_CONSUMERS];
  const float4* m4 = reinterpret_cast<const float4*>(ms + hh * ATT_CONSUMERS);
  const float4* l4 = reinterpret_cast<const float4*>(ls + hh * ATT_CONSUMERS);
  *reinterpret_cast<float4*>(mw) = m4[0];
  *reinterpret_cast<float4*>(mw + 4) = m4[1];
  *reinterpret_cast<float4*>(lw) = l4[0];
  *reinterpret_cast<float4*>(lw + 4) = l4[1];
  float M = mw[0];
#pragma unroll
  for (int w = 1; w < ATT_CONSUMERS; ++w) M = fmaxf(M, mw[w]);
  const float* oc = os + hh * C::OROW + (idx0 - hh * D);
#pragma unroll
  for (int w = 0; w < ATT_CONSUMERS; ++w) {
    if (mw[w] == -INFINITY) continue;  // a warp without live keys in this piece
    const float e = exp2f(mw[w] - M);
    const float4 o4 = *reinterpret_cast<const float4*>(oc + w * G * C::OROW);
    acc[0] += o4.x * e;
    acc[1] += o4.y * e;
    acc[2] += o4.z * e;
    acc[3] += o4.w * e;
    lsum += lw[w] * e;
  }
  mx = M;
}

}  // namespace pced
