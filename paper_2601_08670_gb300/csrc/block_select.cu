// block_select.cu -- the blocks of a paged cache that a new token attends to
// (pced_block_select).
//
// The score of a block is the dot product of the group's pooled query (its
// positive and its negative parts, in 127 steps) with the block's largest and
// smallest keys: 2D products of 8-bit numbers, four a dp4a, exact in 32 bits.  The
// lowest chosen score of a row is found by a radix select, eight bits a pass; the
// blocks above it and, of those at it, the lowest are written in ascending order.
//
// What bounds it (one GB300, GPU time in a graph): for long rows the gather of 256
// bytes a block from anywhere in the pool (33 sequences of 1025 to 2049 blocks,
// 8 kv-heads, 103 MB in 27 us: about 18 of scoring at 5.6 TB/s, 2.5 before it, 5 for
// the selection and the rows' unequal ends), for many short ones the instructions
// (2176 rows of 129 blocks 24 us), for few short ones latency (72 rows of 129
// blocks 4.0 us).  Tried for long rows: clusters that share 4 or 8 heads, so that a
// block's summaries are read side by side, 34 and 50 us (clusters of eight CTAs
// start and end together); four CTAs a row 31 us, one 36 us.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace pced {

namespace cg = cooperative_groups;

constexpr int BSEL_THREADS = 256;       // (also the values of a digit)
constexpr int BSEL_BATCH = 4;           // blocks of a group of lanes in flight
constexpr int BSEL_CLUSTER = 8;         // most CTAs of a row
constexpr int BSEL_MIN_PART = 128;      // blocks that a CTA of a shared row has at least
constexpr int BSEL_MAX_BLOCKS = 32768;  // scores of a row lie in shared memory
constexpr int32_t BSEL_WORST = -(1 << 22);  // of a bad block: below -2 * 128 * 127 * 127

struct SelectArgs {
  pced_paged_cache c;
  const __nv_bfloat16* q;
  int64_t q_stride;
  int32_t G, n_sel, n_first, n_last;
  int32_t* sel;
  int* status;
};

// Exclusive prefix over the CTA's threads of x (all threads; wsum: a word per warp).
__device__ __forceinline__ uint32_t cta_prefix(uint32_t x, uint32_t* wsum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) wsum[warp] = incl;
  __syncthreads();
  uint32_t before = incl - x;
#pragma unroll
  for (int w = 0; w < BSEL_THREADS / 32 - 1; ++w) before += w < warp ? wsum[w] : 0u;
  return before;
}

// Scores of the BSEL_BATCH * 32 / LANES blocks whose pool numbers lie in the
// lanes from `first` on (-1: none): LANES lanes share a block, BSEL_BATCH blocks
// of theirs are in flight.  With LANES >= BSEL_BATCH the sums cross the lanes in
// halves, so that in the end LANES / BSEL_BATCH lanes hold each block's.
template <int D>
struct Scorer {
  static constexpr int LANES = 2 * D / 16, SIDE = 32 / LANES;  // lanes of a block, blocks side by side
  int4 w[BSEL_BATCH];
  __device__ __forceinline__ void load(const int8_t* summary, int64_t page, int entry, int first, int lane) {
#pragma unroll
    for (int u = 0; u < BSEL_BATCH; ++u) {
      const int blk = __shfl_sync(0xffffffffu, entry, first + u * SIDE + lane / LANES);
      w[u] = make_int4(0, 0, 0, 0);
      if (blk >= 0) w[u] = reinterpret_cast<const int4*>(summary + blk * page)[lane % LANES];
    }
  }
  // the score of block first + slot() * SIDE + lane / LANES
  __device__ __forceinline__ int sum(int4 pq, int lane) const {
    int v[BSEL_BATCH];
#pragma unroll
    for (int u = 0; u < BSEL_BATCH; ++u)
      v[u] = __dp4a(w[u].x, pq.x, __dp4a(w[u].y, pq.y, __dp4a(w[u].z, pq.z, __dp4a(w[u].w, pq.w, 0))));
    int o = LANES / 2;
#pragma unroll
    for (int half = BSEL_BATCH / 2; half > 0; half /= 2, o /= 2) {
      const bool upper = lane & o;
#pragma unroll
      for (int u = 0; u < half; ++u) {
        const int give = upper ? v[u] : v[u + half], keep = upper ? v[u + half] : v[u];
        v[u] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
    for (; o > 0; o /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
  }
  static __device__ __forceinline__ int slot(int lane) { return lane % LANES / (LANES / BSEL_BATCH); }
  static __device__ __forceinline__ bool writes(int lane) { return lane % (LANES / BSEL_BATCH) == 0; }
};

// A cluster of CTAs shares a row: their warps take turns at 32 blocks and put the
// scores into the first CTA's shared memory, which selects alone.
template <int D>
__global__ void __launch_bounds__(BSEL_THREADS, 5) block_select_kernel(SelectArgs a) {
  extern __shared__ int32_t scores[];  // [blocks of the sequence]
  __shared__ __align__(16) int8_t pooled[2 * D];
  __shared__ float wmax[BSEL_THREADS / 32];
  __shared__ int2 wrange[BSEL_THREADS / 32];
  __shared__ __align__(16) uint32_t hist[BSEL_THREADS];
  __shared__ uint32_t found[3];  // digit of the threshold, entries wanted at it, entries there are
  __shared__ uint32_t wsum[BSEL_THREADS / 32];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const int s = blockIdx.y, h = blockIdx.x / ctas;
  if (ctas > 1) cluster.barrier_arrive();  // (the first CTA runs before its memory is written)
  pdl_wait();
  // the length, this thread's part of the queries and its first table entry arrive together
  const int32_t* table = a.c.block_table + (int64_t)s * a.c.max_blocks;
  const int stride = ctas * BSEL_THREADS;
  int j = (warp * ctas + rank) * 32 + lane;
  int entry = j < a.c.max_blocks ? table[j] : -1;
  float x[PAGED_MAX_G];
  const __nv_bfloat16* q = a.q + s * a.q_stride + (int64_t)h * a.G * D + tid % D;
#pragma unroll
  for (int g = 0; g < PAGED_MAX_G; ++g) x[g] = g < a.G ? __bfloat162float(q[g * D]) : 0.f;
  const int n = paged_len(a.c, s, a.status);
  const int nb = (n + a.c.block_rows - 1) / a.c.block_rows;
  if (nb <= a.n_sel) {  // all of them
    if (rank == 0) {
      int32_t* sel = a.sel + ((int64_t)s * a.c.Hkv + h) * a.n_sel;
      for (int i = tid; i < a.n_sel; i += BSEL_THREADS) sel[i] = i < nb ? i : -1;
    }
    if (ctas > 1) cluster.barrier_wait();
    return;
  }
  const int64_t page = (int64_t)a.c.Hkv * 2 * D;  // bytes of a block's summaries
  const int8_t* summary = a.c.summary + h * 2 * D;
  Scorer<D> sc;
  const auto check = [&](int j) {  // the lane's entry, -1 where there is no such block
    if (j >= nb) {
      entry = -1;
    } else if (entry < 0 || entry >= a.c.num_blocks) {
      dev_flag(a.status, PCED_DEV_BAD_BLOCK);
      entry = -1;
    }
  };
  check(j);
  sc.load(summary, page, entry, 0, lane);  // the first blocks come while the queries are pooled
  // ---- the pooled query
  float p = 0.f;  // part tid: D positive ones, then D negative ones (and with D = 64 these again)
#pragma unroll
  for (int g = 0; g < PAGED_MAX_G; ++g) {
    if (g >= a.G) break;
    p = __fadd_rn(p, tid < D ? (x[g] > 0.f ? x[g] : 0.f) : (x[g] < 0.f ? x[g] : 0.f));
    if (x[g] != x[g]) p = x[g];
  }
  float m = warp_max(p != p ? INFINITY : fabsf(p));
  if (lane == 0) wmax[warp] = m;
  __syncthreads();
  m = wmax[0];
#pragma unroll
  for (int w = 1; w < BSEL_THREADS / 32; ++w) m = fmaxf(m, wmax[w]);
  const float per_one = __fdiv_rn(127.f, m);  // (infinite where m is zero or next to it)
  if (tid < 2 * D)
    pooled[tid] = per_one < INFINITY && m < INFINITY ? (int8_t)(int)rintf(__fmul_rn(p, per_one)) : (int8_t)0;
  __syncthreads();
  if (ctas > 1) cluster.barrier_wait();
  // ---- scores
  constexpr int LANES = Scorer<D>::LANES, SIDE = Scorer<D>::SIDE;
  int32_t* out = ctas > 1 ? cluster.map_shared_rank(scores, 0) : scores;
  const int4 pq = reinterpret_cast<const int4*>(pooled)[lane % LANES];
  for (int jw = j - lane; jw < nb; jw += stride) {  // 32 blocks of this warp
    const int next = jw + stride + lane < nb ? table[jw + stride + lane] : -1;
#pragma unroll
    for (int first = 0; first < 32; first += BSEL_BATCH * SIDE) {
      if (jw + first >= nb) break;
      if (first > 0 || jw != j - lane) sc.load(summary, page, entry, first, lane);
      const int mine = first + Scorer<D>::slot(lane) * SIDE + lane / LANES;
      const int blk = __shfl_sync(0xffffffffu, entry, mine);
      const int v = sc.sum(pq, lane);
      if (Scorer<D>::writes(lane) && jw + mine < nb) out[jw + mine] = blk < 0 ? BSEL_WORST : v;
    }
    entry = next;
    check(jw + stride + lane);
  }
  if (ctas > 1) cluster.sync();
  else __syncthreads();
  if (rank > 0) return;

  int32_t* sel = a.sel + ((int64_t)s * a.c.Hkv + h) * a.n_sel;
  const auto choose = [&](uint32_t at, int j) {
    if (PCED_IN_BOUNDS(at < (uint32_t)a.n_sel && j < nb, a.status)) sel[at] = j;
  };
  if (nb <= BSEL_THREADS) {
    // ---- few blocks, one a thread: chosen where fewer than `want` others come before it
    const bool forced = tid < a.n_first || tid >= nb - a.n_last;
    // (scores fall with the number within equal ones, so that no two keys are the same)
    const uint32_t key = (uint32_t)((tid < nb ? scores[tid] : BSEL_WORST) - BSEL_WORST) << 8 | (255u - tid);
    hist[tid] = forced || tid >= nb ? 0u : key;
    __syncthreads();
    uint32_t before = 0;
    const int n4 = 32 * warp < nb ? (nb + 3) / 4 : 0;  // (a warp without blocks has nothing to count)
    for (int i = 0; i < n4; ++i) {
      const uint4 k = reinterpret_cast<const uint4*>(hist)[i];
      before += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
    }
    const bool chosen = tid < nb && (forced || before < (uint32_t)(a.n_sel - a.n_first - a.n_last));
    const uint32_t at = cta_prefix(chosen, wsum);
    if (chosen) choose(at, tid);
    return;
  }
  // ---- the lowest score chosen among the blocks [lo, hi) between the first and the last ones
  const int lo = min(a.n_first, nb), hi = max(lo, nb - a.n_last);
  uint32_t want = a.n_sel - (a.n_first + a.n_last);  // of them; fewer than there are, as nb > n_sel
  int2 range = make_int2(INT32_MAX, INT32_MIN);
  for (int j = lo + tid; j < hi; j += BSEL_THREADS) {
    range.x = min(range.x, scores[j]);
    range.y = max(range.y, scores[j]);
  }
  range.x = __reduce_min_sync(0xffffffffu, range.x);
  range.y = __reduce_max_sync(0xffffffffu, range.y);
  if (lane == 0) wrange[warp] = range;
  hist[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < BSEL_THREADS / 32; ++w) {
    range.x = min(range.x, wrange[w].x);
    range.y = max(range.y, wrange[w].y);
  }
  // Scores as distances from the lowest, eight bits a pass from the highest bit
  // that any of them has; the search ends early where a digit's entries are all wanted.
  uint32_t floor = 0;  // distance of the threshold
  if (want > 0) {
    int shift = max(0, 32 - __clz(range.y - range.x) - 8), bits = 32;  // bits: of the distance not fixed yet
    while (true) {
      for (int j = lo + tid; j < hi; j += BSEL_THREADS) {
        const uint32_t d = (uint32_t)(scores[j] - range.x);
        if (bits == 32 || (d ^ floor) >> bits == 0) atomicAdd(&hist[d >> shift & 255u], 1u);
      }
      __syncthreads();
      // the digit that holds the want-th from above: a thread each, suffix sums
      const uint32_t own = hist[tid];
      uint32_t above = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_down_sync(0xffffffffu, above, o);
        if (lane + o < 32) above += v;
      }
      if (lane == 0) wsum[warp] = above;
      __syncthreads();
      above -= own;
#pragma unroll
      for (int w = 1; w < BSEL_THREADS / 32; ++w) above += w > warp ? wsum[w] : 0u;
      if (above < want && want <= above + own) found[0] = tid, found[1] = want - above, found[2] = own;
      __syncthreads();
      floor |= found[0] << shift;
      want = found[1];
      if (shift == 0 || want == found[2]) break;  // (then all from `floor` on are chosen)
      bits = shift;
      shift = max(0, shift - 8);
      hist[tid] = 0;
      __syncthreads();
    }
    if (want == found[2]) want = UINT32_MAX;  // of those at the threshold, or in its digit, all
  }
  // ---- the chosen, in order; each thread takes consecutive blocks
  const bool none = a.n_sel == a.n_first + a.n_last;
  const int per = (nb + BSEL_THREADS - 1) / BSEL_THREADS, j0 = min(nb, tid * per), j1 = min(nb, j0 + per);
  // (2: chosen, 1: at the threshold)
  auto rate = [&](int j) -> uint32_t {
    if (j < lo || j >= hi) return 2;
    if (none) return 0;
    const uint32_t d = (uint32_t)(scores[j] - range.x);
    if (want == UINT32_MAX) return d >= floor ? 2 : 0;
    return d > floor ? 2 : d == floor;
  };
  uint32_t above = 0, ties = 0;
  uint64_t rates = 0;  // of the first 32 of them, two bits each
  for (int j = j0; j < j1; ++j) {
    const uint32_t r = rate(j);
    if (j - j0 < 32) rates |= (uint64_t)r << (2 * (j - j0));
    above += r >> 1;
    ties += r & 1u;
  }
  const uint32_t before = cta_prefix(above << 16 | ties, wsum);
  above = before >> 16, ties = before & 0xFFFFu;
  for (int j = j0; j < j1; ++j) {
    const uint32_t r = j - j0 < 32 ? (uint32_t)(rates >> (2 * (j - j0))) & 3u : rate(j);
    if (r == 2 || (r == 1 && ties < want)) choose(above + min(ties, want), j);
    above += r >> 1;
    ties += r & 1u;
  }
}

}  // namespace pced

using namespace pced;
using namespace pced_host;

extern "C" pced_status pced_block_select(const pced_paged_cache* cache, const void* q, int64_t q_stride, int32_t Hq,
                                         int32_t n_sel, int32_t n_first, int32_t n_last, int32_t* sel,
                                         int32_t* status, void* stream) {
  const char* fn = "pced_block_select";
  pced_status st = check_paged_cache(cache, fn);
  if (st == PCED_OK) st = check_paged_heads(cache, Hq, fn);
  if (st != PCED_OK) return st;
  const pced_paged_cache& c = *cache;
  if (!c.summary || !q || !sel) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (!aligned(q, 16) || !aligned(sel, 4) || !aligned(status, 4))
    return fail(PCED_ERR_INVALID_ARG, "%s: misaligned pointer", fn);
  if (q_stride % 8 || q_stride < (int64_t)Hq * c.D)
    return fail(PCED_ERR_INVALID_ARG, "%s: q_stride no multiple of 8 or below a token's heads", fn);
  if (n_sel < 1 || n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > n_sel)
    return fail(PCED_ERR_INVALID_ARG, "%s: n_first + n_last above n_sel, or a count out of range", fn);
  if (c.max_blocks > BSEL_MAX_BLOCKS)
    return fail(PCED_ERR_UNSUPPORTED, "%s: max_blocks above %d", fn, BSEL_MAX_BLOCKS);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  SelectArgs a;
  a.c = c;
  a.q = (const __nv_bfloat16*)q;
  a.q_stride = q_stride;
  a.G = Hq / c.Hkv;
  a.n_sel = n_sel, a.n_first = n_first, a.n_last = n_last;
  a.sel = sel;
  a.status = status;
  const auto kernel = c.D == 128 ? block_select_kernel<128> : block_select_kernel<64>;
  const size_t smem = (size_t)c.max_blocks * 4;
  static std::atomic<bool> done[2][64];
  cudaError_t e = allow_smem(kernel, BSEL_MAX_BLOCKS * 4, done[c.D == 128]);
  if (e != cudaSuccess) return cuda_status(e, "block_select shared memory");
  // CTAs of a row: more while there are fewer than two for every SM and the blocks
  // are many (four sequences of up to 2049 blocks 8.7 us; one CTA a row 19)
  int ctas = 1;
  while (ctas < BSEL_CLUSTER && (int64_t)c.Hkv * c.S * ctas < 2 * (int64_t)num_sms() &&
         c.max_blocks >= 2 * ctas * BSEL_MIN_PART)
    ctas *= 2;
  e = launch_cluster(kernel, dim3(c.Hkv * ctas, c.S), ctas, BSEL_THREADS, smem, (cudaStream_t)stream, true, a);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "block_select launch");
}
