// paged_attention.cu -- one layer of decode attention over a paged bf16 cache, over
// all blocks or the selected ones (pced_paged_attention; the kernel is in
// paged_attention.cuh).
//
// The math on a tile is that of the slab
// kernels (attention_tile.cuh): mma.sync, whose rate is no bound here (at most
// eight heads share a row: 8 operations a byte, against 280 that the GPU has).
//
// What bounds it (one GB300, GPU time in a graph): HBM for long calls (272 ragged
// sequences, 1.32 GB in 193 us: the measured copy rate), for short ones the chain
// before the first tile (launch, lengths, plan, table: 2.4 us) and after the last
// (partials, record, count, merge: 3 us): 9 x 2081 rows, 77 MB, 17 us, of which 11
// stream; three sequences of 257 rows 5.5 us.  A CTA has one tile at least: with
// four these took 10 us, as a tile's own chain is longer than a record's merge.
// Tiles prefetched into L2 ahead of the ring made every case slower (17 x 64 blocks
// of 64 rows by 15-24 %); a ring of three tiles costs 1-3 %.
#include "paged_attention.cuh"

namespace pced {

// 64 rows of bf16 keys and values, as D/64 boxes of 64 columns
template <int D_, bool PK>
struct TileBf16 {
  static constexpr int D = D_, TILE_BYTES = AttCfg<D>::TILE_BYTES;
  static constexpr int COLS = AttCfg<D>::BOXES, ROW_BYTES = 128;
  static constexpr bool SCALED = false;
  static constexpr int stages(bool) { return AttCfg<D>::STAGES; }
  static constexpr int producers(bool) { return 1; }
  // B column g of S^T = K Q^T is head g; with PK columns 4-7 repeat heads 0-3
  uint32_t qf[D / 16][2];
  __device__ __forceinline__ void load_q(const PagedAttArgs& a, int s, int h, int lane) {
    const int g = lane >> 2, tq = lane & 3;
    const int qh = PK ? (g & 3) : g;
    const bool hv = qh < a.G;
    const uint32_t* qrow =
        reinterpret_cast<const uint32_t*>(a.q + s * a.q_stride + ((int64_t)h * a.G + (hv ? qh : 0)) * D);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      qf[j][0] = hv ? qrow[8 * j + tq] : 0u;
      qf[j][1] = hv ? qrow[8 * j + 4 + tq] : 0u;
    }
  }
  __device__ __forceinline__ void math(WarpAcc<D>& A, uint32_t sk, uint32_t sv, int kb, int nvalid, float2,
                                       float scale_log2, int lane) const {
    tile_math<D, PK, true>(A, qf, sk, sv, kb, nvalid, scale_log2, lane);
  }
  static __device__ __forceinline__ void fold(WarpAcc<D>& A) {
    if (PK) pack_fold<D>(A);
  }
  static __device__ __forceinline__ void store(const WarpAcc<D>& A, float* ms, float* ls, float* os, int G, int warp,
                                               int lane) {
    store_partial<D>(A, ms, ls, os, G, warp, lane);
  }
};

}  // namespace pced

using namespace pced;
using namespace pced_host;

extern "C" size_t pced_paged_attention_workspace_size(int32_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  if (S < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || D < 1) return 0;
  return place_records(nullptr, nullptr, Hq / Hkv, D);
}

extern "C" pced_status pced_paged_attention(const pced_paged_cache* cache, const void* q, int64_t q_stride, int32_t Hq,
                                            const int32_t* sel, int32_t n_sel, int64_t total_rows, float scale,
                                            void* out, int32_t out_type, float* lse, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  PagedAttArgs a;
  int ctas;
  pced_status st = paged_attention_args(cache, q, q_stride, Hq, sel, n_sel, total_rows, scale, out, out_type, lse,
                                        workspace, workspace_bytes, "pced_paged_attention", a, ctas);
  if (st != PCED_OK) return st;
  // the pool as rows of D elements: whole tiles, and 16 rows of 64 columns
  const pced_paged_cache& c = a.c;
  const uint64_t rows = (uint64_t)c.num_blocks * c.Hkv * c.block_rows;
  CUtensorMap maps[4];
  const void* pools[2] = {c.k, c.v};
  for (int i = 0; i < 4 && st == PCED_OK; ++i)
    st = make_tmap_kv_part(&maps[i], pools[i & 1], rows, c.D, i < 2 ? ATT_BLOCK_N : PATT_GRAN, i < 2 ? c.D / 64 : 1);
  if (st != PCED_OK) return st;
  const cudaError_t e = c.D == 128 ? launch_paged_d<TileBf16, 128>(maps, a, ctas, (cudaStream_t)stream)
                                   : launch_paged_d<TileBf16, 64>(maps, a, ctas, (cudaStream_t)stream);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "paged_attention launch");
}
