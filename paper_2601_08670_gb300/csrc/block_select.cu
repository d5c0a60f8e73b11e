// block_select.cu -- the blocks of a paged cache that a new token attends to
// (pced_block_select).
//
// The score of a block is the dot product of the group's pooled query (its
// positive and its negative parts, in 127 steps) with the block's largest and
// smallest keys: 2D products of 8-bit numbers, four a dp4a, exact in 32 bits.  The
// n_sel-th highest of a row's scores is found by a radix select over 24-bit
// keys, eight bits a pass; one more pass writes the blocks above it and, of
// those at it, the lowest, in ascending order.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace pced {

namespace cg = cooperative_groups;

constexpr int BSEL_THREADS = 256;
constexpr int BSEL_BATCH = 8;    // blocks of a half-warp in flight
constexpr int BSEL_CLUSTER = 8;  // most CTAs of a row
constexpr int BSEL_MIN_PART = 128;  // blocks that a CTA of a shared row has at least
constexpr int BSEL_MAX_BLOCKS = 32768;   // scores of a row lie in shared memory
constexpr uint32_t BSEL_ZERO = 1u << 22;         // key of score 0: |score| <= 2 * 128 * 127 * 127 < 2^22
constexpr uint32_t BSEL_FORCED = (1u << 24) - 1;  // key of a block that is chosen whatever its score

struct SelectArgs {
  pced_paged_cache c;
  const __nv_bfloat16* q;
  int64_t q_stride;
  int32_t G, n_sel, n_first, n_last;
  int32_t* sel;
  int* status;
};

// A cluster of CTAs shares a row: each scores its part of the blocks, BSEL_BATCH
// of them in flight per half-warp, and puts the keys into the first CTA's shared
// memory, which selects alone.
template <int D>
__global__ void __launch_bounds__(BSEL_THREADS) block_select_kernel(SelectArgs a) {
  extern __shared__ uint32_t keys[];  // [blocks of the sequence]; in the part being scored the pool blocks first
  __shared__ __align__(16) int8_t pooled[2 * D];
  __shared__ float wmax[BSEL_THREADS / 32];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];  // bin of the threshold's digit, entries wanted from it
  __shared__ uint32_t wcnt[BSEL_THREADS / 32];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank();
  const int s = blockIdx.y, h = blockIdx.x / ctas;
  if (ctas > 1) cluster.barrier_arrive();  // (the first CTA runs before its memory is written)
  pdl_wait();
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
  const int part = (nb + ctas - 1) / ctas, j_lo = min(nb, rank * part), j_hi = min(nb, j_lo + part);
  for (int j = j_lo + tid; j < j_hi; j += BSEL_THREADS) keys[j] = (uint32_t)paged_block(a.c, s, j, a.status);
  // ---- the pooled query
  float p = 0.f, m = 0.f;
  if (tid < 2 * D) {
    const __nv_bfloat16* q = a.q + s * a.q_stride + (int64_t)h * a.G * D + tid % D;
    float x[PAGED_MAX_G];
#pragma unroll
    for (int g = 0; g < PAGED_MAX_G; ++g) x[g] = g < a.G ? __bfloat162float(q[g * D]) : 0.f;
#pragma unroll
    for (int g = 0; g < PAGED_MAX_G; ++g) {
      p = __fadd_rn(p, tid < D ? (x[g] > 0.f ? x[g] : 0.f) : (x[g] < 0.f ? x[g] : 0.f));
      if (x[g] != x[g]) p = x[g];
    }
    m = p != p ? INFINITY : fabsf(p);
  }
  m = warp_max(m);
  if (lane == 0) wmax[warp] = m;
  __syncthreads();
  m = wmax[0];
  for (int w = 1; w < BSEL_THREADS / 32; ++w) m = fmaxf(m, wmax[w]);
  if (tid < 2 * D)
    pooled[tid] = m > 0.f && m < INFINITY ? (int8_t)(int)rintf(__fmul_rn(p, __fdiv_rn(127.f, m))) : (int8_t)0;
  __syncthreads();
  if (ctas > 1) cluster.barrier_wait();
  // ---- scores: 2D / 16 lanes a block
  constexpr int LANES = 2 * D / 16, STRIDE = BSEL_THREADS / LANES;
  uint32_t* out = ctas > 1 ? cluster.map_shared_rank(keys, 0) : keys;
  const int l = tid % LANES;
  const int4 pq = reinterpret_cast<const int4*>(pooled)[l];
  for (int j0 = j_lo + tid / LANES; j0 - tid / LANES < j_hi; j0 += BSEL_BATCH * STRIDE) {
    int4 w[BSEL_BATCH];
    int blk[BSEL_BATCH];
#pragma unroll
    for (int u = 0; u < BSEL_BATCH; ++u) {
      const int j = j0 + u * STRIDE;
      blk[u] = j < j_hi ? (int)keys[j] : -1;
      w[u] = make_int4(0, 0, 0, 0);
      if (blk[u] >= 0)
        w[u] = reinterpret_cast<const int4*>(a.c.summary + ((int64_t)blk[u] * a.c.Hkv + h) * 2 * D)[l];
    }
#pragma unroll
    for (int u = 0; u < BSEL_BATCH; ++u) {
      const int j = j0 + u * STRIDE;
      int sc = __dp4a(w[u].x, pq.x, __dp4a(w[u].y, pq.y, __dp4a(w[u].z, pq.z, __dp4a(w[u].w, pq.w, 0))));
#pragma unroll
      for (int o = 1; o < LANES; o <<= 1) sc += __shfl_xor_sync(0xffffffffu, sc, o);
      if (l == 0 && j < j_hi)
        out[j] = j < a.n_first || j >= nb - a.n_last ? BSEL_FORCED : (blk[u] < 0 ? 0u : BSEL_ZERO + (uint32_t)sc);
    }
  }
  if (ctas > 1) cluster.sync();
  else __syncthreads();
  if (rank > 0) return;
  int32_t* sel = a.sel + ((int64_t)s * a.c.Hkv + h) * a.n_sel;
  // ---- threshold: the n_sel-th highest key
  uint32_t prefix = 0, want = a.n_sel;  // digits found so far; entries wanted among the keys that share them
  for (int shift = 16; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < nb; j += BSEL_THREADS)
      if (shift == 16 || keys[j] >> (shift + 8) == prefix) atomicAdd(&hist[keys[j] >> shift & 255u], 1u);
    __syncthreads();
    if (warp == 0) {  // the bin that holds the want-th from above
      uint32_t own = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) own += hist[8 * lane + i];
      uint32_t above = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_down_sync(0xffffffffu, above, o);
        if (lane + o < 32) above += v;
      }
      above -= own;
      if (above < want && want <= above + own) {
        int b = 8 * lane + 7;
        while (above + hist[b] < want) above += hist[b--];
        found[0] = b;
        found[1] = want - above;
      }
    }
    __syncthreads();
    prefix = prefix << 8 | found[0];
    want = found[1];
    __syncthreads();
  }
  // ---- the chosen, in order; of those at the threshold the first `want`
  uint32_t above0 = 0, ties0 = 0;  // before this round's blocks
  for (int j0 = 0; j0 < nb; j0 += BSEL_THREADS) {
    const int j = j0 + tid;
    const uint32_t key = j < nb ? keys[j] : 0u;
    const bool above = j < nb && key > prefix, tie = j < nb && key == prefix;
    const uint32_t ba = __ballot_sync(0xffffffffu, above), bt = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) wcnt[warp] = __popc(ba) | __popc(bt) << 16;
    __syncthreads();
    const uint32_t below = (1u << lane) - 1u;
    uint32_t na = above0 + __popc(ba & below), nt = ties0 + __popc(bt & below);
    for (int w = 0; w < BSEL_THREADS / 32; ++w) {
      const uint32_t x = wcnt[w];
      above0 += x & 0xFFFFu;
      ties0 += x >> 16;
      if (w < warp) {
        na += x & 0xFFFFu;
        nt += x >> 16;
      }
    }
    if (above || (tie && nt < want)) sel[na + min(nt, want)] = j;
    __syncthreads();
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
  static bool done[2][64];
  cudaError_t e = allow_smem(kernel, BSEL_MAX_BLOCKS * 4, done[c.D == 128]);
  if (e != cudaSuccess) return cuda_status(e, "block_select shared memory");
  int ctas = 1;
  while (ctas < BSEL_CLUSTER && (int64_t)c.Hkv * c.S * ctas < 4 * (int64_t)num_sms() &&
         c.max_blocks >= 2 * ctas * BSEL_MIN_PART)
    ctas *= 2;
  e = launch_cluster(kernel, dim3(c.Hkv * ctas, c.S), ctas, BSEL_THREADS, smem, (cudaStream_t)stream, true, a);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "block_select launch");
}
