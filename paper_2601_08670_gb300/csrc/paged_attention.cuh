// paged_attention.cuh -- one layer of decode attention over a paged cache: the kernel
// that paged_attention.cu (bf16 pools) and paged_attention8.cu (e4m3 pools) instantiate.
//
//   o = sum_r exp2(x_r - m) v_r / sum_r exp2(x_r - m),  x_r = scale log2(e) q.k_r
//
// Split over the rows: every (sequence, kv-head) is a segment of 64-row tiles,
// the tiles of all segments are cut into equal contiguous ranges, one per CTA,
// and the parts of a segment that several CTAs hold meet through records in
// the workspace, merged by the CTA that comes last (in the order of the CTAs,
// so that the result does not depend on who that is).  A producer warp brings
// the tiles with TMA: 32 tiles at a time, each lane finds one tile's segment,
// its place in the selection and its pool block, so the dependent loads of the
// lookups are paid once per 32 tiles.  Where a tile is not 64 live rows of one
// block (a block of another size, a sequence's end) it is put together from
// 16-row boxes, the rows that one consumer warp takes, and rows past the live
// ones are neither brought nor used.
#pragma once
#include "attention_tile.cuh"
#include "paged.cuh"

namespace pced {

constexpr int PATT_MAX_CTAS = 256;  // sizes the records and counters of the workspace
constexpr int PATT_GRAN = 16;       // rows of a consumer warp, and of a small box
constexpr int PATT_EPI = 4;         // epilogue warps

struct PagedAttArgs {
  pced_paged_cache c;
  const __nv_bfloat16* q;
  int64_t q_stride;
  int32_t Hq, G;
  const int32_t* sel;
  int32_t n_sel;
  float scale_log2;
  float up;  // what the sums of the values have to be multiplied by (1, or what Tile::math keeps them down by)
  void* out;
  int32_t out_bf16;
  float* lse;
  float* rec_o;     // [2 * CTAs][G][D] unnormalised partial outputs
  float2* rec_ml;   // [2 * CTAs][G] (running max in log2 units, sum of exp2)
  const float2* scale;  // [num_blocks][Hkv] of the keys and values (8-bit caches)
  int32_t* parts;   // [CTAs] records written of the segment that begins in a CTA and goes on past it (0 between calls)
  int* status;
};

// The tiles [t0, t1) of segment (s, h) that a CTA holds; nt tiles in all.
struct PagedPiece {
  int32_t s, h, t0, t1, nt;
};
// Positions: sequence s begins at base[s]; its heads follow one another, tiles[s] each.
struct PagedPlan {
  const int32_t* base;   // [S + 1]
  const int32_t* tiles;  // [S]
  int32_t S, Hkv;
  __device__ __forceinline__ PagedPiece at(int32_t p, int32_t end) const {
    int32_t lo = 0, hi = S - 1;
    while (lo < hi) {  // the last sequence that begins at or before p (one without tiles begins where the next does)
      const int32_t mid = (lo + hi + 1) >> 1;
      if (base[mid] <= p) lo = mid;
      else hi = mid - 1;
    }
    PagedPiece pc;
    pc.s = lo;
    pc.nt = tiles[lo];
    const uint32_t off = p - base[lo];
    pc.h = off / (uint32_t)pc.nt;
    pc.t0 = off - pc.h * pc.nt;
    pc.t1 = min(pc.nt, pc.t0 + (end - p));
    return pc;
  }
  // the piece after one that ended at its segment's end, at position p < end
  __device__ __forceinline__ PagedPiece after(PagedPiece pc, int32_t p, int32_t end) const {
    if (++pc.h == Hkv) {
      pc.h = 0;
      do ++pc.s;
      while (tiles[pc.s] == 0);
      pc.nt = tiles[pc.s];
    }
    pc.t0 = 0;
    pc.t1 = min(pc.nt, end - p);
    return pc;
  }
};

// Barrier of the epilogue's warps (bounded); `phase` is the caller's phase bit.
__device__ __forceinline__ bool bar_sync_warps(uint32_t bar, uint32_t& phase, int lane, int* status) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
  const bool ok = mbar_wait(bar, phase, status);
  phase ^= 1u;
  return ok;
}

// Shared memory of a CTA over the tiles of `Tile`, which says what the pools hold and
// does the math on it (TileBf16 in paged_attention.cu, TileE4m3 in paged_attention8.cu):
//   D, PK                 head dim; whether the two parts of P share an MMA
//   TILE_BYTES            of K (or V) in a stage
//   COLS, ROW_BYTES       boxes side by side in a tile's rows, bytes of a box's row
//   SCALED                whether a part's two scales come with it
//   stages, producers     of the ring; warps that fill it, which take the CTA's tiles by turns
//                         (small: every tile in boxes of 16 rows)
//   load_q, math, fold, store   a consumer warp's queries, its part of a tile, its partials
constexpr size_t align16(size_t x) { return (x + 15) / 16 * 16; }
template <class Tile, bool SMALL>
struct PagedCfg {
  static constexpr int D = Tile::D;
  static constexpr int STAGES = Tile::stages(SMALL);  // odd: consecutive uses of a stage alternate warpgroups
  static constexpr int STAGE_BYTES = 2 * Tile::TILE_BYTES;
  static constexpr int PARTIALS = AttCfg<D>::PARTIALS;
  static constexpr int PRODUCERS = Tile::producers(SMALL);
  static constexpr int SCALES_OF = SMALL ? ATT_BLOCK_N / PATT_GRAN : 1;  // blocks of a tile
  static constexpr int THREADS = (ATT_CONSUMERS + PRODUCERS + PATT_EPI) * 32;
  static constexpr size_t BARS = (2 * STAGES + 4) * 8;
  static constexpr size_t DESC = (size_t)STAGES * 4;
  static constexpr size_t SCALES = Tile::SCALED ? align16((size_t)STAGES * SCALES_OF * 8) : 0;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE_BYTES + BARS + SCALES + (size_t)PARTIALS * 4 +
                                 (3 * PAGED_MAX_S + 1) * 4 + DESC + 64;
  static_assert(STAGES % 2 == 1 && (BARS + SCALES) % 16 == 0, "the partials are read as float4");
  static_assert(SMEM <= 227 * 1024, "what a CTA can have");
};

// Writes four outputs of a finished segment, normalised.
__device__ __forceinline__ void write_out(const PagedAttArgs& a, int s, int h, int D, int hh, int idx0, float mx,
                                          float lsum, const float (&acc)[4]) {
  const float w = mx == -INFINITY ? 0.f : a.up / lsum;
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = mx == -INFINITY ? 0.f : acc[j] * w;
  const int64_t at = ((int64_t)s * a.Hq + (int64_t)h * a.G) * D + idx0;
  if (a.out_bf16)
    *reinterpret_cast<uint2*>((__nv_bfloat16*)a.out + at) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
  else
    *reinterpret_cast<float4*>((float*)a.out + at) = make_float4(y[0], y[1], y[2], y[3]);
  if (a.lse && idx0 % D == 0)
    a.lse[(int64_t)s * a.Hq + h * a.G + hh] = mx == -INFINITY ? -INFINITY : (mx + log2f(lsum)) * 0.6931471805599453f;
}

// (mx, lsum, acc) joined with another part's
__device__ __forceinline__ void join(float& mx, float& lsum, float (&acc)[4], float mx2, float lsum2,
                                     const float (&acc2)[4]) {
  const float M = fmaxf(mx, mx2);
  const float f = mx == -INFINITY ? 0.f : exp2f(mx - M), g = mx2 == -INFINITY ? 0.f : exp2f(mx2 - M);
  lsum = lsum * f + lsum2 * g;
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = acc[j] * f + acc2[j] * g;
  mx = M;
}

// Records [r0, n) of the segment that begins in CTA c merged into (mx, lsum, acc):
// slots 2c + 1, 2(c + 1), 2(c + 2), ...
__device__ __forceinline__ void merge_records(const PagedAttArgs& a, int c, int r0, int n, int D, int hh, int idx0,
                                              float& mx, float& lsum, float (&acc)[4]) {
  constexpr int BATCH = 8;  // records in flight
  const int GD = a.G * D;
  for (int i0 = r0; i0 < n; i0 += BATCH) {
    float2 ml[BATCH];
    float4 o[BATCH];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const int i = i0 + q;
      ml[q] = make_float2(-INFINITY, 0.f);
      o[q] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i >= n) continue;
      const int64_t slot = i == 0 ? 2 * (int64_t)c + 1 : 2 * ((int64_t)c + i);
      ml[q] = __ldcg(a.rec_ml + slot * a.G + hh);
      o[q] = __ldcg(reinterpret_cast<const float4*>(a.rec_o + slot * GD + idx0));
    }
    float M = mx;
#pragma unroll
    for (int q = 0; q < BATCH; ++q) M = fmaxf(M, ml[q].x);
    const float f = mx == -INFINITY ? 0.f : exp2f(mx - M);
    lsum *= f;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] *= f;
#pragma unroll
    for (int q = 0; q < BATCH; ++q) {
      const float e = ml[q].x == -INFINITY ? 0.f : exp2f(ml[q].x - M);
      acc[0] += o[q].x * e;
      acc[1] += o[q].y * e;
      acc[2] += o[q].z * e;
      acc[3] += o[q].w * e;
      lsum += ml[q].y * e;
    }
    mx = M;
  }
}

// The eight warps' partials (store_partial) merged for outputs idx0 ... idx0 + 3 of
// head hh: load_merged without its branches, so that all warps' values
// are in flight (a piece took the epilogue 1.2 us with them; a warp without rows has
// a sum and an o of zero).
template <int D>
__device__ __forceinline__ void merge_partials(const float* ms, const float* ls, const float* os, int G, int hh,
                                               int idx0, float& mx, float& lsum, float (&acc)[4]) {
  constexpr int W = ATT_CONSUMERS;
  float m[W], l[W];
  float4 o[W];
#pragma unroll
  for (int w = 0; w < W; w += 4) {
    *reinterpret_cast<float4*>(m + w) = *reinterpret_cast<const float4*>(ms + hh * W + w);
    *reinterpret_cast<float4*>(l + w) = *reinterpret_cast<const float4*>(ls + hh * W + w);
  }
#pragma unroll
  for (int w = 0; w < W; ++w)
    o[w] = *reinterpret_cast<const float4*>(os + (w * G + hh) * AttCfg<D>::OROW + (idx0 - hh * D));
  mx = m[0];
#pragma unroll
  for (int w = 1; w < W; ++w) mx = fmaxf(mx, m[w]);
  const float M = mx == -INFINITY ? 0.f : mx;
  lsum = acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float e = exp2f(m[w] - M);
    acc[0] += o[w].x * e;
    acc[1] += o[w].y * e;
    acc[2] += o[w].z * e;
    acc[3] += o[w].w * e;
    lsum += l[w] * e;
  }
}

// A piece's partials, merged, into the output (a whole segment) or into a record,
// and the segment's records into the output where this was the last of them to
// come.  NT threads, whole warps, with a barrier of their own; seq0: the position at
// which the piece's sequence begins; bar_read: told when the partials have been
// read (0: nobody waits).
template <int D, int NT>
__device__ __forceinline__ bool finish_piece(const PagedAttArgs& a, const PagedPiece& pc, int32_t seq0, int32_t per,
                                             const float* ms, const float* ls, float* os, int et, uint32_t bar,
                                             uint32_t& phase, uint32_t bar_read, int32_t* last_here) {
  const int G = a.G, GD = G * D, lane = et & 31;
  const bool whole = pc.t0 == 0 && pc.t1 == pc.nt;
  // a part of a segment: record 2c of CTA c when it began in an earlier CTA,
  // 2c + 1 when it begins here
  const int64_t slot = 2 * (int64_t)blockIdx.x + (pc.t0 == 0 ? 1 : 0);
  if (!PCED_IN_BOUNDS(pc.s >= 0 && pc.s < a.c.S && pc.h >= 0 && pc.h < a.c.Hkv && slot < 2 * PATT_MAX_CTAS, a.status))
    return false;
  for (int i = et; i < GD / 4; i += NT) {
    const int hh = i / (D / 4), idx0 = 4 * i;
    float mx, lsum, acc[4];
    merge_partials<D>(ms, ls, os, G, hh, idx0, mx, lsum, acc);
    if (whole) {
      write_out(a, pc.s, pc.h, D, hh, idx0, mx, lsum, acc);
    } else {
      *reinterpret_cast<float4*>(a.rec_o + slot * GD + idx0) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      if (idx0 % D == 0) a.rec_ml[slot * G + hh] = make_float2(mx, lsum);
    }
  }
  __syncwarp();
  if (bar_read && lane == 0) mbar_arrive(bar_read);
  if (whole) return true;
  const int32_t seg0 = seq0 + pc.h * pc.nt;  // the segment's first position
  const int first = (uint32_t)seg0 / (uint32_t)per;
  const int n = (int)((uint32_t)(seg0 + pc.nt - 1) / (uint32_t)per) - first + 1;
  if (!PCED_IN_BOUNDS(first >= 0 && n >= 2 && first + n <= (int)gridDim.x, a.status)) return false;
  if (!bar_sync_warps(bar, phase, lane, a.status)) return false;  // all of this CTA's record is written
  // (its release and acquire at gpu scope carry what the barriers order for the other threads)
  if (et == 0) *last_here = atom_acq_rel_gpu_add(a.parts + first, 1) == n - 1;
  if (!bar_sync_warps(bar, phase, lane, a.status)) return false;
  if (!*last_here) return true;
  // Many records are merged in shares, which are joined in order.  At the CTA's end,
  // where the partials' memory is free, the threads that are more than the outputs take
  // a share each (one sequence of 39,382 rows, two kv-heads of 64, 70 records each:
  // 14.8 us, with four shares side by side 10.9); the epilogue takes them one after the
  // other: the same arithmetic, whoever comes last.
  const int shares = n <= 8 ? 1 : ATT_CT / (GD / 4), per_share = (n + shares - 1) / shares;
  if (shares > 1 && !bar_read) {
    const int share = et / (GD / 4), i = et - share * (GD / 4);
    float mx = -INFINITY, lsum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    if (share < shares)
      merge_records(a, first, share * per_share, min(n, (share + 1) * per_share), D, i / (D / 4), 4 * i, mx, lsum, acc);
    float* mine = os + 6 * et;  // (6 floats a thread: less than the partials' memory)
    mine[0] = mx, mine[1] = lsum, mine[2] = acc[0], mine[3] = acc[1], mine[4] = acc[2], mine[5] = acc[3];
    if (!bar_sync_warps(bar, phase, lane, a.status)) return false;
    if (share == 0) {
      for (int k = 1; k < shares; ++k) {
        const float* o = os + 6 * (et + k * (GD / 4));
        const float acc2[4] = {o[2], o[3], o[4], o[5]};
        join(mx, lsum, acc, o[0], o[1], acc2);
      }
      write_out(a, pc.s, pc.h, D, i / (D / 4), 4 * i, mx, lsum, acc);
    }
  } else {
    for (int i = et; i < GD / 4; i += NT) {
      float mx = -INFINITY, lsum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
      merge_records(a, first, 0, min(n, per_share), D, i / (D / 4), 4 * i, mx, lsum, acc);
      for (int k = 1; k < shares; ++k) {
        float mx2 = -INFINITY, lsum2 = 0.f, acc2[4] = {0.f, 0.f, 0.f, 0.f};
        merge_records(a, first, k * per_share, min(n, (k + 1) * per_share), D, i / (D / 4), 4 * i, mx2, lsum2, acc2);
        join(mx, lsum, acc, mx2, lsum2, acc2);
      }
      write_out(a, pc.s, pc.h, D, i / (D / 4), 4 * i, mx, lsum, acc);
    }
  }
  if (et == 0) a.parts[first] = 0;
  return true;
}

// Roles: eight consumer warps (the math, and each piece's partials into shared
// memory), a producer warp (lookups and TMA) and PATT_EPI warps that finish the
// pieces, so that the consumers go on with the next piece at once: while they
// finished pieces themselves, a CTA with a segment's end in its range took 2.5 us
// longer than one without (17.0 and 14.5 us of the 9 x 2081 rows' 19).
//
// (Only a CTA's last piece is the consumers' own matter: they are more, and idle.)
// A warpgroup that finished segments of one tile alone, while the other one took the
// next, brought 2176 segments of 16 to 64 rows from 24.3 to 22.3 us, but every other
// call 1 to 4 % more time, the more the colder the code (a layer of 9 sequences and
// 16 selected blocks between matrix products: 39.2 us against 37.5).
//
// SMALL: block_rows is no multiple of 64, so every tile comes in 16-row boxes,
// each of its own block.
template <class Tile, bool SMALL>
__global__ void __launch_bounds__(PagedCfg<Tile, SMALL>::THREADS, 1)
    paged_attention_kernel(const __grid_constant__ CUtensorMap ktile, const __grid_constant__ CUtensorMap vtile,
                           const __grid_constant__ CUtensorMap kbox, const __grid_constant__ CUtensorMap vbox,
                           PagedAttArgs a) {
  using C = PagedCfg<Tile, SMALL>;
  constexpr int D = Tile::D;
  constexpr int NG = ATT_BLOCK_N / PATT_GRAN;  // small boxes of a tile
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t smem0 = (raw + 1023u) & ~1023u;
  uint8_t* gbase = smem_raw + (smem0 - raw);
  // layout: stages | full[STAGES] | empty[STAGES] | partials full | partials empty | epilogue | last piece | scales | partials | tables
  const uint32_t bar_full = smem0 + C::STAGES * C::STAGE_BYTES;
  const uint32_t bar_empty = bar_full + C::STAGES * 8;
  const uint32_t bar_pfull = bar_empty + C::STAGES * 8, bar_pempty = bar_pfull + 8;
  const uint32_t bar_epi = bar_pempty + 8, bar_last = bar_epi + 8;
  float2* scales = reinterpret_cast<float2*>(gbase + C::STAGES * C::STAGE_BYTES + C::BARS);  // [STAGES][SCALES_OF]
  float* ms = reinterpret_cast<float*>(gbase + C::STAGES * C::STAGE_BYTES + C::BARS + C::SCALES);
  float* ls = ms + ATT_CONSUMERS * ATT_MAX_G;
  float* os = ls + ATT_CONSUMERS * ATT_MAX_G;
  int32_t* base = reinterpret_cast<int32_t*>(ms + C::PARTIALS);  // [S + 1]
  int32_t* tiles = base + PAGED_MAX_S + 1;
  int32_t* lens = tiles + PAGED_MAX_S;
  uint32_t* desc = reinterpret_cast<uint32_t*>(lens + PAGED_MAX_S);  // [STAGES] live rows of a tile's 16-row parts, a byte each
  int32_t* last_here = reinterpret_cast<int32_t*>(desc + C::STAGES);

  const int tid = threadIdx.x, warp = uniform_warp(), lane = tid & 31;
  const int32_t S = a.c.S, Hkv = a.c.Hkv, G = a.G, P = a.c.block_rows;

  if (tid == 0) {
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(bar_full + 8 * i, Tile::SCALED ? 1 + C::SCALES_OF : 1);
      mbar_init(bar_empty + 8 * i, 4);  // the four warps of the consuming warpgroup
    }
    mbar_init(bar_pfull, ATT_CONSUMERS);
    mbar_init(bar_pempty, PATT_EPI);
    mbar_init(bar_epi, PATT_EPI);
    mbar_init(bar_last, ATT_CONSUMERS);
    mbar_fence_init();
  }
  if (warp == ATT_CONSUMERS && lane == 0) {
    tma_prefetch_desc(&ktile);
    tma_prefetch_desc(&vtile);
    tma_prefetch_desc(&kbox);
    tma_prefetch_desc(&vbox);
  }
  pdl_wait();
  for (int i = tid; i < S; i += C::THREADS) {
    const int32_t n = paged_len(a.c, i, a.status);
    uint32_t rows = n;
    if (a.sel) rows = min((uint32_t)a.n_sel, (rows + P - 1) / P) * P;
    lens[i] = n;
    tiles[i] = (rows + ATT_BLOCK_N - 1) / ATT_BLOCK_N;
  }
  __syncthreads();
  if (warp == 0) {  // prefix of the tiles of all heads
    const int chunk = (S + 31) / 32, b0 = min(S, lane * chunk), b1 = min(S, b0 + chunk);
    int32_t own = 0;
    for (int i = b0; i < b1; ++i) own += tiles[i] * Hkv;
    int32_t incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    int32_t run = incl - own;
    for (int i = b0; i < b1; ++i) {
      base[i] = run;
      run += tiles[i] * Hkv;
    }
    if (lane == 31) base[S] = incl;
  }
  __syncthreads();
  const PagedPlan plan = {base, tiles, S, Hkv};
  const int32_t total = base[S];
  const int32_t per = (int32_t)((uint32_t)(total + gridDim.x - 1) / gridDim.x);  // tiles of a CTA
  const int32_t r_begin = (int32_t)min((int64_t)total, (int64_t)blockIdx.x * per);
  const int32_t r_end = min(total - r_begin, per) + r_begin;

  if (warp >= ATT_CONSUMERS && warp < ATT_CONSUMERS + C::PRODUCERS) {
    // ------------------------------------------------------------ producer
    constexpr int NP = C::PRODUCERS;
    // (A stage has one producer: it waits for every release of the stage in turn, so that the parity
    // tells which; with two, one could take the release before the last for the last.)
    static_assert(C::STAGES % NP == 0, "a stage is always the same producer's");
    const uint64_t pol = policy_evict_first();
    uint32_t st = warp - ATT_CONSUMERS, ph = 0, it = st;
    bool ok = true;
    for (int32_t p0 = r_begin + (int32_t)it; p0 < r_end && ok; p0 += 32 * NP) {
      // this lane's tile: pool row of each of its parts, live rows of the parts, their pages
      int32_t row[SMALL ? NG : 1], page[Tile::SCALED ? (SMALL ? NG : 1) : 1];
      uint32_t live4 = 0;
      row[0] = page[0] = 0;
      const int nt = min(32, (r_end - p0 + NP - 1) / NP);
      if (lane < nt) {
        const PagedPiece pc = plan.at(p0 + NP * lane, r_end);
        const int32_t n = lens[pc.s];
        const int32_t nb = (int32_t)((uint32_t)(n + P - 1) / (uint32_t)P);
        const int32_t* sel = a.sel ? a.sel + ((int64_t)pc.s * Hkv + pc.h) * a.n_sel : nullptr;
        const int32_t places = sel ? min(a.n_sel, nb) : nb;
#pragma unroll
        for (int i = 0; i < (SMALL ? NG : 1); ++i) {
          const uint32_t r = (uint32_t)pc.t0 * ATT_BLOCK_N + i * PATT_GRAN;  // row of the list
          const int32_t place = (int32_t)(r / (uint32_t)P), at = (int32_t)(r - (uint32_t)place * P);
          row[i] = 0;
          if (Tile::SCALED) page[i] = 0;
          if (place >= places) continue;
          const int32_t j = sel ? sel[place] : place;
          if (j < 0 || j >= nb) {
            if (j != -1) dev_flag(a.status, PCED_DEV_BAD_BLOCK);
            continue;
          }
          const int32_t blk = paged_block(a.c, pc.s, j, a.status);
          if (blk < 0) continue;
          if (!PCED_IN_BOUNDS(in_pool(a.c, (int64_t)blk * Hkv + pc.h, at), a.status)) continue;
          row[i] = (blk * Hkv + pc.h) * P + at;
          if (Tile::SCALED) page[i] = blk * Hkv + pc.h;
          const int32_t left = n - j * P - at;  // live rows from here on
          if (SMALL) {
            live4 |= (uint32_t)max(0, min(left, PATT_GRAN)) << (8 * i);
          } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) live4 |= (uint32_t)max(0, min(left - g * PATT_GRAN, PATT_GRAN)) << (8 * g);
          }
        }
      }
      for (int t = 0; t < nt; ++t, it += NP) {
        if (!mbar_wait_warp(bar_empty + 8 * st, ph ^ 1u, a.status)) {
          ok = false;
          break;
        }
        const uint32_t fb = bar_full + 8 * st, sk = smem0 + st * C::STAGE_BYTES, sv = sk + Tile::TILE_BYTES;
        const uint32_t lv = __shfl_sync(0xffffffffu, live4, t);
        const int32_t r0 = __shfl_sync(0xffffffffu, row[0], t);
        const uint32_t on = elect_one();
        if (on) desc[st] = lv;
        if constexpr (Tile::SCALED) {  // they come as the rows do: a load that waits would hold the copies up
          int32_t pg = __shfl_sync(0xffffffffu, page[0], t);
          if (SMALL) {
#pragma unroll
            for (int i = 1; i < NG; ++i) {
              const int32_t x = __shfl_sync(0xffffffffu, page[i], t);
              if (i == lane) pg = x;
            }
          }
          if (lane < C::SCALES_OF) {
            if (lv >> (8 * lane) & 0xFFu) copy_async_8(smem_u32(scales + st * C::SCALES_OF + lane), a.scale + pg);
            mbar_arrive_copies(fb);
          }
        }
        // (more than 48 live rows of one block: the whole tile at once)
        if (!SMALL && lv >> 24) {
          mbar_arrive_expect_tx_if(on, fb, C::STAGE_BYTES);
          if (on) {
            tma_load_3d(sk, &ktile, fb, 0, r0, 0, pol);
            tma_load_3d(sv, &vtile, fb, 0, r0, 0, pol);
          }
        } else {
          // parts with live rows; a lane for each box of K and V
          const int boxes = ((lv & 0xFFu) != 0) + ((lv & 0xFF00u) != 0) + ((lv & 0xFF0000u) != 0) + (lv >> 24 != 0);
          mbar_arrive_expect_tx_if(on, fb, boxes * (2 * Tile::COLS * Tile::ROW_BYTES * PATT_GRAN));
          __syncwarp();
          const int g = lane / (2 * Tile::COLS) % NG, col = lane % Tile::COLS, v = lane / Tile::COLS & 1;
          int32_t rg = r0 + g * PATT_GRAN;
          if (SMALL) {
#pragma unroll
            for (int i = 0; i < NG; ++i) {
              const int32_t x = __shfl_sync(0xffffffffu, row[i], t);
              if (i == g) rg = x;
            }
          }
          if (lane < 2 * Tile::COLS * NG && (lv >> (8 * g) & 0xFFu))
            tma_load_3d((v ? sv : sk) + (col * ATT_BLOCK_N + g * PATT_GRAN) * Tile::ROW_BYTES, v ? &vbox : &kbox, fb, 0,
                        rg, col, pol);
        }
        st += NP;
        if (st >= C::STAGES) {
          st -= C::STAGES;
          ph ^= 1u;
        }
      }
    }
    if (!ok) {
      // let this warp's copies in flight land before the CTA exits: those of its tiles before `it`
      // whose stage it has not waited for again
      for (uint32_t j = it; j >= NP && it - (j - NP) <= C::STAGES; j -= NP)
        mbar_wait(bar_full + 8 * ((j - NP) % C::STAGES), ((j - NP) / C::STAGES) & 1u, a.status);
    }
    return;
  }

  if (warp >= ATT_CONSUMERS + C::PRODUCERS) {
    // ------------------------------------------------------------ epilogue
    const int et = tid - (ATT_CONSUMERS + C::PRODUCERS) * 32;
    // sequences without rows
    for (int s = blockIdx.x; s < S; s += gridDim.x)
      if (tiles[s] == 0) {
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i = et; i < a.Hq * (D / 4); i += PATT_EPI * 32)
          write_out(a, s, 0, D, i / (D / 4), 4 * i, -INFINITY, 0.f, zero);
      }
    if (r_begin >= r_end) return;
    PagedPiece pc = plan.at(r_begin, r_end);
    uint32_t phase = 0;
    for (int32_t p = r_begin + pc.t1 - pc.t0, np = 0; p < r_end; p += pc.t1 - pc.t0, ++np) {
      if (!mbar_wait(bar_pfull, np & 1u, a.status)) return;
      if (!finish_piece<D, PATT_EPI * 32>(a, pc, base[pc.s], per, ms, ls, os, et, bar_epi, phase, bar_pempty,
                                          last_here))
        return;
      pc = plan.after(pc, p, r_end);
    }
    return;
  }

  // -------------------------------------------------------------- consumers
  if (r_begin >= r_end) return;
  const int wg = warp >> 2, kb = PATT_GRAN * (warp & 3);
  Tile tile;
  PagedPiece pc = plan.at(r_begin, r_end);
  tile.load_q(a, pc.s, pc.h, lane);
  uint32_t it = 0, st = 0, use = 0, np = 0;  // tile counter, its stage and use of the stage; shared pieces done
  for (int32_t p = r_begin;; ++np) {
    p += pc.t1 - pc.t0;
    WarpAcc<D> A;
    acc_reset(A);
    for (int32_t t = pc.t0; t < pc.t1; ++t, ++it, st = st + 1 == C::STAGES ? (++use, 0u) : st + 1) {
      if ((int)(it & 1u) != wg) continue;
      // (the release of the stage's previous use, by the other warpgroup, comes
      // first: the parity below then means this tile's phase)
      if ((use > 0 && !mbar_wait(bar_empty + 8 * st, (use - 1u) & 1u, a.status)) ||
          !mbar_wait(bar_full + 8 * st, use & 1u, a.status))
        return;
      const int live = desc[st] >> (8 * (warp & 3)) & 0xFFu;
      if (live) {
        const uint32_t sk = smem0 + st * C::STAGE_BYTES;
        tile.math(A, sk, sk + Tile::TILE_BYTES, kb, kb + live,
                  Tile::SCALED ? scales[st * C::SCALES_OF + (SMALL ? warp & 3 : 0)] : make_float2(1.f, 1.f), a.scale_log2, lane);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * st);
    }
    const bool more = p < r_end;
    const PagedPiece last = pc;
    if (more) {  // the next piece's queries come while this one's partials go
      pc = plan.after(pc, p, r_end);
      tile.load_q(a, pc.s, pc.h, lane);
    }
    // scores that are all not numbers moved no maximum: their sum shall not be dropped with it
    if (__any_sync(0xffffffffu, (A.m0 == -INFINITY && A.l0 != A.l0) || (A.m1 == -INFINITY && A.l1 != A.l1))) {
      A.m0 = A.m0 == -INFINITY ? 0.f : A.m0;
      A.m1 = A.m1 == -INFINITY ? 0.f : A.m1;
    }
    Tile::fold(A);
    // the previous piece's partials have been read
    if (np > 0 && !mbar_wait(bar_pempty, (np - 1u) & 1u, a.status)) return;
    Tile::store(A, ms, ls, os, G, warp, lane);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_pfull);
    if (more) continue;
    // the CTA's last piece
    uint32_t phase = 0;
    if (mbar_wait(bar_pfull, np & 1u, a.status))
      finish_piece<D, ATT_CT>(a, last, base[last.s], per, ms, ls, os, tid, bar_last, phase, 0, last_here + 1);
    return;
  }
}


// ----------------------------------------------------------------------- host
// records and counters in the workspace, after its status word
inline size_t place_records(PagedAttArgs* a, void* ws, int32_t G, int32_t D) {
  pced_host::Carver cv(ws ? (char*)ws + 256 : nullptr);
  int32_t* parts = cv.take<int32_t>(PATT_MAX_CTAS);
  float* rec_o = cv.take<float>((size_t)2 * PATT_MAX_CTAS * G * D);
  float2* rec_ml = cv.take<float2>((size_t)2 * PATT_MAX_CTAS * G);
  if (a) a->parts = parts, a->rec_o = rec_o, a->rec_ml = rec_ml;
  return 256 + cv.used();
}

template <class Tile, bool SMALL>
cudaError_t launch_paged(const CUtensorMap (&maps)[4], const PagedAttArgs& a, int ctas, cudaStream_t stream) {
  const auto kernel = paged_attention_kernel<Tile, SMALL>;
  static std::atomic<bool> done[64];
  const cudaError_t e = pced_host::allow_smem(kernel, PagedCfg<Tile, SMALL>::SMEM, done);
  if (e != cudaSuccess) return e;
  return pced_host::launch_pdl(kernel, dim3(ctas), PagedCfg<Tile, SMALL>::THREADS, PagedCfg<Tile, SMALL>::SMEM, stream, maps[0], maps[1],
                               maps[2], maps[3], a);
}
// Tile<D, PK>: PK where at most four heads share a row (hi and lo parts of P in one MMA)
template <template <int, bool> class Tile, int D>
cudaError_t launch_paged_d(const CUtensorMap (&maps)[4], const PagedAttArgs& a, int ctas, cudaStream_t stream) {
  const bool pk = a.G <= 4, small = a.c.block_rows % ATT_BLOCK_N != 0;
  return pk ? (small ? launch_paged<Tile<D, true>, true>(maps, a, ctas, stream)
                     : launch_paged<Tile<D, true>, false>(maps, a, ctas, stream))
            : (small ? launch_paged<Tile<D, false>, true>(maps, a, ctas, stream)
                     : launch_paged<Tile<D, false>, false>(maps, a, ctas, stream));
}

// The checks and arguments of a call that do not depend on what the pools hold;
// ctas: the grid.
inline pced_status paged_attention_args(const pced_paged_cache* cache, const void* q, int64_t q_stride, int32_t Hq,
                                        const int32_t* sel, int32_t n_sel, int64_t total_rows, float scale, void* out,
                                        int32_t out_type, float* lse, void* workspace, size_t workspace_bytes,
                                        const char* fn, PagedAttArgs& a, int& ctas) {
  using namespace pced_host;
  pced_status st = check_paged_cache(cache, fn);
  if (st == PCED_OK) st = check_paged_heads(cache, Hq, fn);
  if (st != PCED_OK) return st;
  const pced_paged_cache& c = *cache;
  if (!c.k || !c.v || !q || !out || !workspace) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (out_type != PCED_OUT_F32 && out_type != PCED_OUT_BF16)
    return fail(PCED_ERR_INVALID_ARG, "%s: no such output type", fn);
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(sel, 4))
    return fail(PCED_ERR_INVALID_ARG, "%s: misaligned pointer", fn);
  if (q_stride % 8 || q_stride < (int64_t)Hq * c.D)
    return fail(PCED_ERR_INVALID_ARG, "%s: q_stride no multiple of 8 or below a token's heads", fn);
  if (sel ? n_sel < 1 : n_sel != 0) return fail(PCED_ERR_INVALID_ARG, "%s: n_sel without sel, or below 1", fn);
  // (positions of tiles are 32-bit numbers)
  if (((int64_t)c.max_blocks * c.block_rows / ATT_BLOCK_N + 2) * c.S * c.Hkv > INT32_MAX)
    return fail(PCED_ERR_UNSUPPORTED, "%s: tables of 2^31 tiles or more", fn);
  if (!isfinite(scale) || total_rows < 0) return fail(PCED_ERR_INVALID_ARG, "%s: scale or total_rows", fn);
  if (!aligned(workspace, 256) || workspace_bytes < pced_paged_attention_workspace_size(c.S, Hq, c.Hkv, c.D))
    return fail(PCED_ERR_WORKSPACE, "%s: workspace too small or misaligned", fn);
  const int sms = num_sms();
  if (sms <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  a.c = c;
  a.q = (const __nv_bfloat16*)q;
  a.q_stride = q_stride;
  a.Hq = Hq, a.G = Hq / c.Hkv;
  a.sel = sel, a.n_sel = n_sel;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.up = 1.f;
  a.out = out, a.out_bf16 = out_type == PCED_OUT_BF16;
  a.lse = lse;
  a.scale = nullptr;
  a.status = (int*)workspace;
  place_records(&a, workspace, a.G, c.D);
  // a CTA for every SM, fewer where the caller's bound of the rows needs no more
  int64_t n = sms < PATT_MAX_CTAS ? sms : PATT_MAX_CTAS;
  if (total_rows > 0) {
    const int64_t tiles = total_rows / ATT_BLOCK_N + c.S;  // of a kv-head
    if (tiles < n) n = min(n, tiles * c.Hkv);
  }
  ctas = (int)n;
  return PCED_OK;
}

}  // namespace pced
