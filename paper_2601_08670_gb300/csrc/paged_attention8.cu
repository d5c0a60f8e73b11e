// paged_attention8.cu -- one layer of decode attention over a paged cache of e4m3
// numbers with scales (pced_paged_attention8; the kernel is in paged_attention.cuh).
//
//   x_r = (scale log2(e) s_k) q.b_r,  o = sum_r 2^(x_r - m) s_v b_r / sum_r 2^(x_r - m)
//
// A warp's 16 rows lie in one block, so the scale of the keys joins the factor of the
// scores and the scale of the values the factor with which the warp's sums are added.
// The bytes become fp16 in registers, which holds every e4m3 number, and the products
// run as fp16 mma.sync.  fp16's range is met by powers of two: a head's query is scaled
// so that its largest part lies in [2^14, 2^15) (a part below 2^-31 of it loses bits,
// which the sum does not keep either), probabilities are counted from 2^7 at the
// reference (at most 2^15 until it moves), their first 11 bits in one part, the rest, times
// 2^11, in the other: 23 bits, as a sum in fp32 keeps.  The values' sums are kept 2^-15 down, so that
// they overflow no sooner than with probabilities up to 1 (scales below 2^-111 lose bits by it).
//
// What bounds it (one GB300, GPU time in a graph): 272 ragged sequences of 32/8 heads of
// 128, 665 MB in 128 us (5.2 TB/s, 77 % of the copy rate; the bf16 operator needs 193 for
// twice the bytes): a byte costs the eight consumer warps as many instructions as two of bf16
// (a conversion to fp16, and two products with the probabilities' parts), so that they are
// about as long as the copies.  The small calls are bound by the chain from the lengths to
// the merge, as the bf16 operator's: 9 x 2081 rows 13.6 us for 5.7 of streaming, 3 x 257 rows of
// 8/2 heads of 64 5.8 us.  One sequence of 131,104 rows in 16-row blocks, 34 MB in 18.5: eight
// copies of 1 KB a tile, each with a look at the table.
#include "paged_attention.cuh"

namespace pced {

constexpr float P8_RAISE = 7.f;   // log2 of a probability at the reference
constexpr float P8_SLACK = 15.f;  // log2 of the largest one
constexpr float P8_LOW = 2048.f;  // factor of a probability's second part
constexpr float P8_UP = 32768.f;  // 2^P8_SLACK, by which the sums of the values are kept down

template <int D_, bool PK>
struct TileE4m3 {
  static constexpr int D = D_, TILE_BYTES = ATT_BLOCK_N * D;
  static constexpr int COLS = 1, ROW_BYTES = D;
  static constexpr bool SCALED = true;
  // (small: eight copies a tile are more than one warp issues in time, 131,104 rows of 8 x 128
  // in 16-row blocks 60 us with one, 48 with three.  Whole tiles: nine stages for seven, or three
  // warps, make 9 x 2081 rows 14.0 and 14.3 us for 13.6, as copies in flight share the
  // bandwidth and the first tile comes late; 272 ragged sequences gain 0.3 and 3 %)
  static constexpr int stages(bool small) { return D == 128 ? (small ? 9 : 7) : (small ? 15 : 9); }
  static constexpr int producers(bool small) { return small ? 3 : 1; }
  // The B operand of S^T = K Q^T, head g (with PK columns 4-7 repeat heads 0-3).  Of the
  // 32 channels that an ldmatrix of bytes brings, a thread has 4tq ... 4tq + 3 and the
  // same 16 further: the order of a sum's channels is free, so those are its k indexes.
  uint32_t qf[D / 32][4];
  float f0, f1;  // factors of heads 2tq, 2tq + 1, which undo the query's scaling
  __device__ __forceinline__ void load_q(const PagedAttArgs& a, int s, int h, int lane) {
    const int g = lane >> 2, tq = lane & 3;
    const int qh = PK ? (g & 3) : g;
    const bool hv = qh < a.G;
    const uint2* qrow = reinterpret_cast<const uint2*>(a.q + s * a.q_stride + ((int64_t)h * a.G + (hv ? qh : 0)) * D);
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint2 w = hv ? qrow[8 * j + 4 * i + tq] : make_uint2(0u, 0u);
        qf[j][2 * i] = w.x, qf[j][2 * i + 1] = w.y;
        // (exponent fields: the largest, and those of not-a-number)
        top = max(max(top, max(w.x & 0x7F80u, w.x >> 16 & 0x7F80u)), max(w.y & 0x7F80u, w.y >> 16 & 0x7F80u));
      }
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(max((int)(top >> 7) - 127, -100), 127);
    const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23), down = __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) qf[j][i] = pack_f16(bf16_lo(qf[j][i]) * up, bf16_hi(qf[j][i]) * up);
    f0 = __shfl_sync(0xffffffffu, down, 8 * tq) * a.scale_log2;
    f1 = __shfl_sync(0xffffffffu, down, 8 * tq + 4) * a.scale_log2;
  }

  // 16-byte part c of row r of a tile
  static __device__ __forceinline__ uint32_t part(uint32_t tile, int r, int c) {
    return tile + r * D + ((c ^ (D == 128 ? r & 7 : r >> 1 & 3)) << 4);
  }

  // This warp's 16 rows [kb, kb + 16) of the tiles at sk, sv; rows >= nvalid are masked.
  __device__ __forceinline__ void math(WarpAcc<D>& A, uint32_t sk, uint32_t sv, int kb, int nvalid, float2 scales,
                                       float, int lane) const {
    constexpr int N = D / 32;
    const int g = lane >> 2, tq = lane & 3, mat = lane >> 3, mr = lane & 7;
    const int row = kb + (mat & 1) * 8 + mr;
    // (the loads all at once, those of V ahead of the softmax, and every sum taken up an MMA
    // later: the instructions are issued in this order, so what waits holds up all that follows)
    uint32_t rk[N][4], rv[N][4];
#pragma unroll
    for (int j = 0; j < N; ++j) ldsm_x4(part(sk, row, 2 * j + (mat >> 1)), rk[j][0], rk[j][1], rk[j][2], rk[j][3]);
    // ---- scores S^T (16 rows x 8 heads), four independent accumulation chains
    float sc4[4][4];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      uint32_t a[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) e4m3_to_f16(rk[j][i], a[2 * i], a[2 * i + 1]);
      if (j < 2) {
        mma_f16_first(sc4[2 * j], a[0], a[2], a[1], a[3], qf[j][0], qf[j][1]);
        mma_f16_first(sc4[2 * j + 1], a[4], a[6], a[5], a[7], qf[j][2], qf[j][3]);
      } else {
        mma_f16(sc4[2 * j & 3], a[0], a[2], a[1], a[3], qf[j][0], qf[j][1]);
        mma_f16(sc4[(2 * j + 1) & 3], a[4], a[6], a[5], a[7], qf[j][2], qf[j][3]);
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) ldsm_x4_t(part(sv, row, 2 * j + (mat >> 1)), rv[j][0], rv[j][1], rv[j][2], rv[j][3]);
    const bool v0 = kb + g < nvalid, v1 = kb + g + 8 < nvalid;
    const float k0 = f0 * scales.x, k1 = f1 * scales.x;
    const float s0 = v0 ? ((sc4[0][0] + sc4[1][0]) + (sc4[2][0] + sc4[3][0])) * k0 : -INFINITY;
    const float s1 = v0 ? ((sc4[0][1] + sc4[1][1]) + (sc4[2][1] + sc4[3][1])) * k1 : -INFINITY;
    const float s2 = v1 ? ((sc4[0][2] + sc4[1][2]) + (sc4[2][2] + sc4[3][2])) * k0 : -INFINITY;
    const float s3 = v1 ? ((sc4[0][3] + sc4[1][3]) + (sc4[2][3] + sc4[3][3])) * k1 : -INFINITY;
    // The reference only moves when a score exceeds it by more than P8_SLACK
    float x0 = fmaxf(s0, s2), x1 = fmaxf(s1, s3);
    if (__any_sync(0xffffffffu, x0 > A.m0 + P8_SLACK || x1 > A.m1 + P8_SLACK)) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) {
        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, off));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, off));
      }
      const float n0 = fmaxf(A.m0, x0 - P8_RAISE), n1 = fmaxf(A.m1, x1 - P8_RAISE);
      const float al0 = A.m0 == -INFINITY ? 0.f : exp2f(A.m0 - n0);
      const float al1 = A.m1 == -INFINITY ? 0.f : exp2f(A.m1 - n1);
      A.l0 *= al0;
      A.l1 *= al1;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        A.o[i][0] *= al0;
        A.o[i][2] *= al0;
        A.o[i][1] *= al1;
        A.o[i][3] *= al1;
      }
      A.m0 = n0;
      A.m1 = n1;
    }
    const float u0 = A.m0 == -INFINITY ? 0.f : A.m0, u1 = A.m1 == -INFINITY ? 0.f : A.m1;
    const float p0 = exp2_ftz(s0 - u0), p1 = exp2_ftz(s1 - u1), p2 = exp2_ftz(s2 - u0), p3 = exp2_ftz(s3 - u1);
    A.l0 += p0 + p2;
    A.l1 += p1 + p3;
    // ---- P^T as the B operand (rows x heads), in two parts
    const uint32_t h01 = pack_f16(p0, p1), h23 = pack_f16(p2, p3);
    const float2 w01 = unpack_f16(h01), w23 = unpack_f16(h23);
    const uint32_t q01 = pack_f16((p0 - w01.x) * P8_LOW, (p1 - w01.y) * P8_LOW);
    const uint32_t q23 = pack_f16((p2 - w23.x) * P8_LOW, (p3 - w23.y) * P8_LOW);
    const bool lo_cols = PK && tq >= 2;
    const uint32_t bh0 = movmatrix_t(lo_cols ? q01 : h01), bh1 = movmatrix_t(lo_cols ? q23 : h23);
    const uint32_t bl0 = PK ? 0u : movmatrix_t(q01), bl1 = PK ? 0u : movmatrix_t(q23);
    // ---- O^T += s_v V^T P^T.  A transposing ldmatrix of bytes brings pairs of channels
    // (2g, 2g + 1) of a thread's two rows; sorted by channel they are rows g and g + 8 of V^T.
    const bool partial = kb + 16 > nvalid;
    const int klo = kb + 2 * tq, khi = klo + 8;
    const uint32_t mlo = (klo < nvalid ? 0xFFFFu : 0u) | (klo + 1 < nvalid ? 0xFFFF0000u : 0u);
    const uint32_t mhi = (khi < nvalid ? 0xFFFFu : 0u) | (khi + 1 < nvalid ? 0xFFFF0000u : 0u);
    const float high = scales.y * (1.f / P8_UP), low = high * (1.f / P8_LOW);
    float t[2][2][4], u[2][2][4];
    const auto take_up = [&](int j) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          A.o[2 * j + i][e] = fmaf(t[j & 1][i][e], high, A.o[2 * j + i][e]);
          if (!PK) A.o[2 * j + i][e] = fmaf(u[j & 1][i][e], low, A.o[2 * j + i][e]);
        }
    };
#pragma unroll
    for (int j = 0; j < N; ++j) {
      uint32_t a[8];
      if (partial) rv[j][0] &= mlo, rv[j][1] &= mhi, rv[j][2] &= mlo, rv[j][3] &= mhi;
#pragma unroll
      for (int i = 0; i < 4; ++i) e4m3_to_f16(__byte_perm(rv[j][i], 0u, 0x3120), a[2 * i], a[2 * i + 1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // channels 32j + 16i ...
        mma_f16_first(t[j & 1][i], a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3], bh0, bh1);
        if (!PK) mma_f16_first(u[j & 1][i], a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3], bl0, bl1);
      }
      if (j > 0) take_up(j - 1);
    }
    take_up(N - 1);
  }
  // the second parts' sums, in columns 4-7, to the first parts'
  static __device__ __forceinline__ void fold(WarpAcc<D>& A) {
    if constexpr (PK) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          A.o[i][e] = fmaf(__shfl_xor_sync(0xffffffffu, A.o[i][e], 2), 1.f / P8_LOW, A.o[i][e]);
    }
  }
  // (store_partial with this tile's order of channels: 16i + 2g and 16i + 2g + 1)
  static __device__ __forceinline__ void store(const WarpAcc<D>& A, float* ms, float* ls, float* os, int G, int warp,
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
    float* ow = os + warp * G * C::OROW + 2 * g;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      if (2 * tq < G) *reinterpret_cast<float2*>(ow + (2 * tq) * C::OROW + 16 * i) = make_float2(A.o[i][0], A.o[i][2]);
      if (2 * tq + 1 < G)
        *reinterpret_cast<float2*>(ow + (2 * tq + 1) * C::OROW + 16 * i) = make_float2(A.o[i][1], A.o[i][3]);
    }
  }
};

}  // namespace pced

using namespace pced;
using namespace pced_host;

extern "C" pced_status pced_paged_attention8(const pced_paged_cache8* cache, const void* q, int64_t q_stride,
                                             int32_t Hq, const int32_t* sel, int32_t n_sel, int64_t total_rows,
                                             float scale, void* out, int32_t out_type, float* lse, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  const char* fn = "pced_paged_attention8";
  if (cache && !cache->scale) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (cache && !aligned(cache->scale, 8)) return fail(PCED_ERR_INVALID_ARG, "%s: misaligned cache pointer", fn);
  PagedAttArgs a;
  int ctas;
  pced_status st = paged_attention_args(cache ? &cache->pages : nullptr, q, q_stride, Hq, sel, n_sel, total_rows, scale,
                                        out, out_type, lse, workspace, workspace_bytes, fn, a, ctas);
  if (st != PCED_OK) return st;
  const pced_paged_cache& c = a.c;
  a.scale = reinterpret_cast<const float2*>(cache->scale);
  a.up = P8_UP;
  const uint64_t rows = (uint64_t)c.num_blocks * c.Hkv * c.block_rows;
  CUtensorMap maps[4];
  const void* pools[2] = {c.k, c.v};
  for (int i = 0; i < 4 && st == PCED_OK; ++i)
    st = make_tmap_bytes(&maps[i], pools[i & 1], rows, c.D, i < 2 ? ATT_BLOCK_N : PATT_GRAN);
  if (st != PCED_OK) return st;
  const cudaError_t e = c.D == 128 ? launch_paged_d<TileE4m3, 128>(maps, a, ctas, (cudaStream_t)stream)
                                   : launch_paged_d<TileE4m3, 64>(maps, a, ctas, (cudaStream_t)stream);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "paged_attention8 launch");
}
