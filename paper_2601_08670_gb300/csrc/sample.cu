// sample.cu -- a token for every row of logits from a given random number, by
// temperature, top-k, top-p and min-p (pced_sample).
//
// With m the row's largest logit, w_v = exp((x_v - m) / t).  Ordered by logit, then by
// token, a cut keeps the first tokens: the top k, the shortest prefix of them that holds
// p of their weight, those of weight min_p or more.  The token is the first kept one, in
// the order of the vocabulary, up to which the kept weights sum to more than u of all.
//
// A sum over a vocabulary decides at which token u falls, so it must not depend on its
// order, and its error counts 150,000 times (every border of two tokens is a place to be
// wrong): with weights of 24 bits, one row in some thousands gets another token than in 64
// bits.  So weights are whole numbers of 2^-44, exact to about 2^-32 of themselves (see
// Weight), and summed as such.
//
// A cluster of CTAs holds a row in shared memory, read once.  A cut is found by counting
// (or weighing) the tokens in 1024 equal ranges of x below m, then the border range's
// tokens one by one if they are few, else in 1024 equal ranges of their (logit, token)
// pairs, as 64-bit numbers, again and again: pairs are distinct, so that ends.
#include <cooperative_groups.h>

#include "paged.cuh"

namespace pced {

namespace cg = cooperative_groups;

struct SampleArgs {
  const void* x;
  int64_t stride;
  int32_t V, per;  // tokens; of a CTA of the row's cluster
  const float* u;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* token;
  float* logprob;
  int* status;
};

constexpr int SMP_THREADS = 512;
constexpr int SMP_WARPS = SMP_THREADS / 32;
constexpr int SMP_BINS = 1024;
constexpr int SMP_FEW = 512;          // tokens of a border range that are ranked one by one
constexpr int SMP_EACH = 8;           // tokens of a lane in a tile
constexpr int SMP_TILE = 32 * SMP_EACH;
constexpr int SMP_MAX_V = 393216;     // a cluster's shared memory (and 2^44 V < 2^63)
constexpr int SMP_MAX_BYTES = 192 * 1024;  // of a CTA's part of a row
constexpr int SMP_MAX_TILES = SMP_MAX_BYTES / 2 / SMP_TILE;
constexpr float SMP_LEAST = -45.f;    // log2 of weights that are nothing in steps of 2^-44
constexpr uint64_t SMP_ONE = (uint64_t)1 << 44;

// 2^(j / 32) in steps of 2^-31
__device__ const uint32_t kExp2Table[32] = {
    2147483648u, 2194507417u, 2242560872u, 2291666561u, 2341847524u, 2393127307u, 2445529972u, 2499080105u,
    2553802834u, 2609723834u, 2666869345u, 2725266179u, 2784941738u, 2845924021u, 2908241642u, 2971923842u,
    3037000500u, 3103502151u, 3171459999u, 3240905930u, 3311872529u, 3384393094u, 3458501653u, 3534232978u,
    3611622603u, 3690706840u, 3771522796u, 3854108391u, 3938502376u, 4024744348u, 4112874773u, 4202935003u};

// Weights of a row's logits.  y = (x - m) log2(e) / t is held in two fp32 numbers (x - m
// exactly, by the two-sum; the factor in two parts): y = q / 32 + r, q whole, |r| <= 1/64.
// 2^(q / 32) comes from the table, 2^r - 1 from its series to r^4 (the next term is below
// 2^-39), both in whole steps of 2^-31, so that their product is one of two 32-bit numbers.
struct Weight {
  float m, ch, cl;  // ch + cl = log2(e) / t
  uint32_t table;   // entry `lane`
  __device__ __forceinline__ void set(float m_, float t, int lane) {
    m = m_;
    ch = cl = 0.f;
    if (t < 1e30f) {  // (above, all weights are the same)
      const float lh = 1.44269502f, ll = 1.92596303e-08f;
      ch = __fdiv_rn(lh, t);
      cl = __fdiv_rn(fmaf(-ch, t, lh) + ll, t);
    }
    table = kExp2Table[lane];
  }
  // whether a weight can be more than nothing
  __device__ __forceinline__ bool some(float x) const { return x == m || (x - m) * ch > SMP_LEAST; }
  // All lanes of a warp.
  __device__ __forceinline__ uint64_t of(float x) const {
    const float s = __fsub_rn(x, m), b = __fsub_rn(s, x);
    const float e = __fadd_rn(__fsub_rn(x, __fsub_rn(s, b)), __fsub_rn(-m, b));
    const float p = __fmul_rn(s, ch);
    const float low = fmaf(e, ch, fmaf(s, cl, fmaf(s, ch, -p)));
    constexpr float MAGIC = 393216.f;  // 1.5 2^18: sums with it are rounded to 32nds
    const float shifted = __fadd_rn(p, MAGIC);
    const float r = __fadd_rn(__fsub_rn(p, __fsub_rn(shifted, MAGIC)), low);
    const int q = __float_as_int(shifted) - __float_as_int(MAGIC);
    const float g = r * fmaf(r, fmaf(r, fmaf(r, 20654774.98f, 119194165.75f), 515882495.51f), 1488522235.91f);
    const uint32_t f = 0x80000000u + (uint32_t)__float2int_rn(g);
    const uint32_t t = __shfl_sync(0xffffffffu, table, q & 31);
    const uint64_t w = (uint64_t)t * f >> ((18 - (q >> 5)) & 63);
    return x == m ? SMP_ONE : p > SMP_LEAST ? w : 0;
  }
};

// Order of (logit, token) pairs: larger logits first, then lower tokens
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t pair_of(float x, int v) { return (uint64_t)order_key(x) << 32 | (uint32_t)~v; }

__device__ __forceinline__ float load_logit(const float* p) { return *p; }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }

__device__ __forceinline__ uint64_t warp_sum64(uint64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The first range that brings the sum to the target, and what lies before it.
struct Border {
  uint32_t found, bin, count, n;  // count: tokens before it, n: in it
  uint64_t mass;                  // weight before it
};

struct SampleShared {
  uint32_t hist[4][SMP_BINS];  // tokens of a range; their weights' 15-bit parts
  uint64_t cand[SMP_FEW], cand_w[SMP_FEW];
  uint64_t tile_mass[SMP_MAX_TILES];
  uint32_t n_cand;
  uint32_t wcount[SMP_WARPS];
  uint64_t wmass[SMP_WARPS], wmin[SMP_WARPS], wmax[SMP_WARPS];
  float fmax[SMP_WARPS], fmin[SMP_WARPS];
  // what the cluster's CTAs tell one another: two of each, by turns, with a barrier of
  // the cluster between a write and its reads, so that the next write to one comes after them
  struct Told {
    float mx, mn;
    uint32_t count;
    uint64_t mass, lo, hi, cut;
    Border border;
  } told[2];
  uint64_t target, seek;
  float threshold;
};

template <typename T>
struct Row {
  const SampleArgs& a;
  SampleShared& s;
  cg::cluster_group cluster;
  const T* data;  // this CTA's part of the row
  int first, n;   // its first token, their number
  int ctas, rank, tid, lane, warp, turn;
  Weight w;
  uint64_t cut;  // pairs below it are not kept

  __device__ __forceinline__ SampleShared::Told& mine() { return s.told[turn & 1]; }
  __device__ __forceinline__ const SampleShared::Told& theirs(int r) { return cluster.map_shared_rank(&s, r)->told[turn & 1]; }
  // all have told; read with theirs(), then call next()
  __device__ __forceinline__ void meet() { cluster.sync(); }
  __device__ __forceinline__ void next() { ++turn; }

  __device__ __forceinline__ float logit(int i) const {  // (-0 is 0, what is not a number: -inf)
    return i < n ? fmaxf(load_logit(data + i), -INFINITY) + 0.f : -INFINITY;
  }
  // f(token of the part, logit) for all lanes and tiles; tokens past the end are -inf
  template <typename F>
  __device__ __forceinline__ void each_tile(F f) {
    for (int t = warp; t * SMP_TILE < n; t += SMP_WARPS) f(t);
  }
  __device__ __forceinline__ bool keeps(float x, int i) const { return w.some(x) && pair_of(x, first + i) >= cut; }

  // Weight of all kept tokens, tile by tile into tile_mass; the CTA's sum to all threads.
  __device__ __forceinline__ uint64_t weigh() {
    uint64_t sum = 0;
    each_tile([&](int t) {
      uint64_t mass = 0;
#pragma unroll
      for (int e = 0; e < SMP_EACH; ++e) {
        const int i = t * SMP_TILE + e * 32 + lane;
        const float x = logit(i);
        const bool k = keeps(x, i);
        if (cut == 0 || __any_sync(0xffffffffu, k)) {
          const uint64_t v = w.of(x);
          mass += k ? v : 0;
        }
      }
      mass = warp_sum64(mass);
      if (lane == 0) s.tile_mass[t] = mass;
      sum += mass;
    });
    __syncthreads();
    if (lane == 0) s.wmass[warp] = sum;
    __syncthreads();
    sum = 0;
    for (int i = 0; i < SMP_WARPS; ++i) sum += s.wmass[i];
    return sum;
  }

  // Border of the histogram, which the cluster's CTAs bring together, a part of the
  // ranges each; `share` > 0: the target is that share of the weight, at least 1.
  __device__ __forceinline__ Border border(bool by_mass, uint64_t target, double share) {
    meet();  // all histograms are complete
    const int slice = SMP_BINS / ctas, each = (slice + SMP_THREADS - 1) / SMP_THREADS;  // of a CTA, of a thread
    const int b0 = rank * slice + tid * each, mine_n = tid * each < slice ? each : 0;
    uint32_t count[2] = {0, 0};
    uint64_t mass[2] = {0, 0};
    uint32_t c = 0;
    uint64_t ms = 0;
    for (int j = 0; j < mine_n; ++j) {
      for (int r = 0; r < ctas; ++r) {
        const SampleShared& o = *cluster.map_shared_rank(&s, r);
        count[j] += o.hist[0][b0 + j];
        if (by_mass)
          mass[j] += o.hist[1][b0 + j] + ((uint64_t)o.hist[2][b0 + j] << 15) + ((uint64_t)o.hist[3][b0 + j] << 30);
      }
      c += count[j];
      ms += mass[j];
    }
    // sums up to this thread
    uint32_t ci = c;
    uint64_t mi = ms;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, ci, o);
      const uint64_t y = __shfl_up_sync(0xffffffffu, mi, o);
      if (lane >= o) ci += x, mi += y;
    }
    __syncthreads();
    if (lane == 31) s.wcount[warp] = ci, s.wmass[warp] = mi;
    __syncthreads();
    for (int i = 0; i < warp; ++i) ci += s.wcount[i], mi += s.wmass[i];
    if (tid == SMP_THREADS - 1) mine().count = ci, mine().mass = mi;
    meet();
    uint64_t all = 0;
    uint32_t before_c = 0;
    uint64_t before_m = 0;
    for (int r = 0; r < ctas; ++r) {
      all += theirs(r).mass;
      if (r < rank) before_c += theirs(r).count, before_m += theirs(r).mass;
    }
    next();
    if (share > 0) {
      const double want = ceil(share * (double)all);
      target = want < 1.0 ? 1 : (uint64_t)want;
    }
    if (tid == 0) mine().border.found = 0;
    __syncthreads();
    uint32_t at_c = before_c + ci - c;
    uint64_t at_m = before_m + mi - ms;
    for (int j = 0; j < mine_n; ++j) {
      const uint64_t from = by_mass ? at_m : at_c, to = from + (by_mass ? mass[j] : count[j]);
      if (from < target && to >= target) {
        Border b;
        b.found = 1, b.bin = b0 + j, b.count = at_c, b.n = count[j], b.mass = at_m;
        mine().border = b;
      }
      at_c += count[j], at_m += mass[j];
    }
    s.target = target;
    meet();
    Border b;
    b.found = 0;
    for (int r = 0; r < ctas; ++r)
      if (theirs(r).border.found) b = theirs(r).border;
    next();
    return b;
  }

  // Cuts off what lies behind the first `target` tokens (by_mass: behind the first that
  // hold `share` of the kept weight).
  __device__ __forceinline__ void search(bool by_mass, uint64_t target, double share, float per_range) {
    uint64_t lo = cut, hi = ~0ull;
    int shift = -1;  // -1: equal ranges of x
    for (int level = 0; level < 10; ++level) {
      const auto range_of = [&](float x, uint64_t pair) -> int {
        if (shift >= 0) return (int)((hi - pair) >> shift);
        return x == w.m ? 0 : (int)fminf((w.m - x) * per_range, (float)(SMP_BINS - 1));
      };
      __syncthreads();
      for (int i = tid; i < 4 * SMP_BINS; i += SMP_THREADS) s.hist[0][i] = 0;
      if (tid == 0) s.n_cand = 0;
      __syncthreads();
      each_tile([&](int t) {
#pragma unroll
        for (int e = 0; e < SMP_EACH; ++e) {
          const int i = t * SMP_TILE + e * 32 + lane;
          const float x = logit(i);
          const uint64_t pair = pair_of(x, first + i);
          const bool in = w.some(x) && pair >= lo && pair <= hi;
          if (!__any_sync(0xffffffffu, in)) continue;
          const int b = in ? range_of(x, pair) : 0;
          if (in) atomicAdd(&s.hist[0][b], 1u);
          if (by_mass) {
            const uint64_t v = w.of(x);
            if (in) {
              atomicAdd(&s.hist[1][b], (uint32_t)v & 0x7FFFu);
              atomicAdd(&s.hist[2][b], (uint32_t)(v >> 15) & 0x7FFFu);
              atomicAdd(&s.hist[3][b], (uint32_t)(v >> 30));
            }
          }
        }
      });
      const Border b = border(by_mass, target, share);
      if (!b.found) return;  // all are kept
      // the next level counts from what lies before this range on
      target = s.target - (by_mass ? b.mass : b.count);
      share = 0.0;
      const bool few = b.n <= SMP_FEW;
      uint64_t least = ~0ull, most = 0;
      if (few || shift < 0) {
        each_tile([&](int t) {
#pragma unroll
          for (int e = 0; e < SMP_EACH; ++e) {
            const int i = t * SMP_TILE + e * 32 + lane;
            const float x = logit(i);
            const uint64_t pair = pair_of(x, first + i);
            const bool in = w.some(x) && pair >= lo && pair <= hi && range_of(x, pair) == (int)b.bin;
            if (!__any_sync(0xffffffffu, in)) continue;
            const uint64_t v = by_mass && few ? w.of(x) : 0;
            if (!in) continue;
            least = min(least, pair), most = max(most, pair);
            if (few) {
              const uint32_t at = atomicAdd(&s.n_cand, 1u);
              s.cand[at] = pair, s.cand_w[at] = v;
            }
          }
        });
      }
      if (few) {
        rank_few(by_mass, target);
        return;
      }
      if (shift < 0) {  // the pairs that the range holds
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
          most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        }
        if (lane == 0) s.wmin[warp] = least, s.wmax[warp] = most;
        __syncthreads();
        if (tid == 0) {
          for (int i = 1; i < SMP_WARPS; ++i) least = min(least, s.wmin[i]), most = max(most, s.wmax[i]);
          mine().lo = least, mine().hi = most;
        }
        meet();
        lo = ~0ull, hi = 0;
        for (int r = 0; r < ctas; ++r) lo = min(lo, theirs(r).lo), hi = max(hi, theirs(r).hi);
        next();
      } else {
        const uint64_t top = hi - ((uint64_t)b.bin << shift);
        const uint64_t bottom = top - (((uint64_t)1 << shift) - 1);
        lo = bottom > lo ? bottom : lo;
        hi = top;
      }
      shift = max(0, 64 - __clzll((long long)(hi - lo)) - 10);
    }
  }

  // The cluster's candidates, at most SMP_FEW, ranked by CTA 0: the cut is the one that
  // brings the sum to the target.
  __device__ __forceinline__ void rank_few(bool by_mass, uint64_t target) {
    __syncthreads();
    if (tid == 0) mine().count = s.n_cand;
    meet();
    if (rank == 0) {
      int total = s.n_cand;
      for (int r = 1; r < ctas; ++r) {
        const SampleShared& o = *cluster.map_shared_rank(&s, r);
        const int k = theirs(r).count;
        for (int i = tid; i < k; i += SMP_THREADS)
          if (PCED_IN_BOUNDS(total + i < SMP_FEW, a.status)) s.cand[total + i] = o.cand[i], s.cand_w[total + i] = o.cand_w[i];
        total += k;
      }
      if (tid == 0) mine().cut = cut;
      __syncthreads();
      if (tid < total) {
        const uint64_t own = s.cand[tid], ow = by_mass ? s.cand_w[tid] : 1;
        uint64_t before = 0;
        for (int i = 0; i < total; ++i)
          if (s.cand[i] > own) before += by_mass ? s.cand_w[i] : 1;
        if (before < target && before + ow >= target) mine().cut = own;
      }
      __syncthreads();
    }
    next();
    if (rank == 0 && tid == 0) mine().cut = s.told[(turn - 1) & 1].cut;
    meet();
    cut = theirs(0).cut;
    next();
  }
};

template <typename T>
__global__ void __launch_bounds__(SMP_THREADS, 2) sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ SampleShared s;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank(), tid = threadIdx.x;
  const int64_t row = blockIdx.x / ctas;
  Row<T> R = {a, s, cluster, nullptr, rank * a.per, 0, ctas, rank, tid, tid & 31, tid >> 5, 0, {}, 0};
  R.n = max(0, min(a.per, a.V - R.first));
  pdl_wait();
  // ---- the row into shared memory, at the offset in 16 bytes that it has in memory
  const T* src = (const T*)a.x + row * a.stride + R.first;
  constexpr int W = 16 / sizeof(T);
  const int phase = (int)((uintptr_t)src / sizeof(T) % W);
  T* data = reinterpret_cast<T*>(smem_raw) + phase;
  R.data = data;
  float mx = -INFINITY, mn = INFINITY;
  const auto take = [&](float x) {
    mx = fmaxf(mx, x);
    mn = x > -INFINITY ? fminf(mn, x) : mn;
  };
  const int head = min(R.n, (W - phase) % W), words = (R.n - head) / W;
  {
    const uint4* from = reinterpret_cast<const uint4*>(src + head);
    uint4* to = reinterpret_cast<uint4*>(data + head);
    constexpr int BATCH = 8;
    for (int i0 = tid; i0 < words; i0 += BATCH * SMP_THREADS) {
      uint4 v[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k)
        if (i0 + k * SMP_THREADS < words) v[k] = from[i0 + k * SMP_THREADS];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (i0 + k * SMP_THREADS >= words) break;
        to[i0 + k * SMP_THREADS] = v[k];
        const T* p = reinterpret_cast<const T*>(&v[k]);
#pragma unroll
        for (int e = 0; e < W; ++e) take(load_logit(p + e));
      }
    }
    const int edges = head + (R.n - head) % W;
    for (int i = tid; i < edges; i += SMP_THREADS) {
      const int at = i < head ? i : head + words * W + i - head;
      data[at] = src[at];
      take(load_logit(src + at));
    }
  }
  // ---- its largest and smallest logit
  mx = warp_max(mx), mn = -warp_max(-mn);
  if (R.lane == 0) s.fmax[R.warp] = mx, s.fmin[R.warp] = mn;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < SMP_WARPS; ++i) mx = fmaxf(mx, s.fmax[i]), mn = fminf(mn, s.fmin[i]);
    R.mine().mx = mx, R.mine().mn = mn;
  }
  R.meet();
  for (int r = 0; r < ctas; ++r) mx = fmaxf(mx, R.theirs(r).mx), mn = fminf(mn, R.theirs(r).mn);
  R.next();
  mx += 0.f;
  // ---- what the row asks for
  const float t = a.temperature ? a.temperature[row] : 1.f, u = a.u[row];
  const float p = a.top_p ? a.top_p[row] : 1.f, least = a.min_p ? a.min_p[row] : 0.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const bool bad = !(t >= 0.f) || !(u >= 0.f && u <= 1.f) || p != p || least != least;
  if (bad || mx == -INFINITY) {  // a request out of range, or a row without a token
    if (rank == 0 && tid == 0) {
      if (bad) dev_flag(a.status, PCED_DEV_BAD_PARAM);
      a.token[row] = -1;
      if (a.logprob) a.logprob[row] = -INFINITY;
    }
    cluster.sync();
    return;
  }
  if (t == 0.f || k == 1 || p <= 0.f || least > 1.f) {  // the first of the largest
    uint32_t at = UINT32_MAX;
    for (int i = tid; i < R.n; i += SMP_THREADS)
      if (R.logit(i) == mx) at = min(at, (uint32_t)i);
    at = __reduce_min_sync(0xffffffffu, at);
    if (R.lane == 0) s.wcount[R.warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < SMP_WARPS; ++i) at = min(at, s.wcount[i]);
      R.mine().count = at == UINT32_MAX ? at : R.first + at;
    }
    R.meet();
    if (rank == 0 && tid == 0) {
      for (int r = 0; r < ctas; ++r) at = min(r == 0 ? UINT32_MAX : at, R.theirs(r).count);
      a.token[row] = (int32_t)at;
      if (a.logprob) a.logprob[row] = 0.f;
    }
    cluster.sync();
    return;
  }
  R.w.set(mx, t, R.lane);
  // ---- cuts
  const float per_range = (float)(SMP_BINS - 1) / fminf(32.f * t, mx - mn);
  if (k > 1 && k < a.V) R.search(false, (uint64_t)k, 0.0, per_range);
  if (p < 1.f) R.search(true, 0, (double)p, per_range);
  if (least > 0.f) {
    if (tid == 0)
      s.threshold = __double2float_ru((double)mx + (double)t * log((double)least));
    __syncthreads();
    const uint64_t from = (uint64_t)order_key(s.threshold + 0.f) << 32;
    R.cut = from > R.cut ? from : R.cut;
  }
  // ---- the kept weights, and where u falls
  const uint64_t own = R.weigh();
  if (tid == 0) R.mine().mass = own;
  R.meet();
  uint64_t total = 0, before = 0;
  for (int r = 0; r < ctas; ++r) {
    const uint64_t m = R.theirs(r).mass;
    total += m;
    if (r < rank) before += m;
  }
  R.next();
  if (R.warp == 0) {
    // (both factors are exact, and total is below 2^63)
    const uint64_t seek = min((uint64_t)((double)u * (double)total), total - 1);
    if (seek >= before && seek < before + own) {
      uint64_t left = seek - before;
      // its tile: each lane some of them in a row
      const int tiles = (R.n + SMP_TILE - 1) / SMP_TILE, each = (tiles + 31) / 32;
      uint64_t sum = 0;
      for (int i = R.lane * each; i < min(tiles, (R.lane + 1) * each); ++i) sum += s.tile_mass[i];
      uint64_t to = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, to, o);
        if (R.lane >= o) to += y;
      }
      const int who = __ffs(__ballot_sync(0xffffffffu, to > left)) - 1;
      left -= __shfl_sync(0xffffffffu, to - sum, who);
      int tile = who * each;
      while (left >= s.tile_mass[tile]) left -= s.tile_mass[tile++];
      // its token: 32 at a time
      for (int e = 0; e < SMP_EACH; ++e) {
        const int i = tile * SMP_TILE + e * 32 + R.lane;
        const float x = R.logit(i);
        const uint64_t v = R.w.of(x);
        uint64_t run = R.keeps(x, i) ? v : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint64_t y = __shfl_up_sync(0xffffffffu, run, o);
          if (R.lane >= o) run += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, run > left);
        if (past) {
          if (R.lane == __ffs(past) - 1) {
            a.token[row] = R.first + i;
            if (a.logprob) {
              const double z = x == mx ? 0.0 : ((double)x - (double)mx) / (double)t;
              a.logprob[row] = (float)(z - log((double)total * (1.0 / (double)SMP_ONE)));
            }
          }
          break;
        }
        left -= __shfl_sync(0xffffffffu, run, 31);
      }
    }
  }
  cluster.sync();  // (a CTA's memory stays until the others have read it)
}

}  // namespace pced

using namespace pced;
using namespace pced_host;

template <typename T>
static cudaError_t launch_sample(SampleArgs a, int32_t rows, cudaStream_t stream) {
  static bool done[64];
  const auto kernel = sample_kernel<T>;
  cudaError_t e = allow_smem(kernel, SMP_MAX_BYTES + 16, done);
  if (e != cudaSuccess) return e;
  const auto part = [&](int ctas) { return ((int64_t)a.V + ctas - 1) / ctas; };
  int ctas = 1;
  // two CTAs an SM; and more while there are SMs without a row and a part is more than a
  // few tokens a thread
  constexpr int64_t HALF = 80 * 1024 / sizeof(T), FEW = 4 * SMP_THREADS;
  while (ctas < ROW_CLUSTER && (part(ctas) > HALF || (2 * ctas * (int64_t)rows <= 2 * num_sms() && part(ctas) > FEW)))
    ctas *= 2;
  a.per = (int32_t)part(ctas);
  const size_t smem = align_up((size_t)a.per * sizeof(T) + 16, 16);
  return launch_cluster(kernel, dim3((unsigned)(rows * ctas)), ctas, SMP_THREADS, smem, stream, true, a);
}

extern "C" pced_status pced_sample(const void* x, int32_t type, int64_t stride, int32_t rows, int32_t V, const float* u,
                                   const float* temperature, const int32_t* top_k, const float* top_p,
                                   const float* min_p, int32_t* token, float* logprob, int32_t* status, void* stream) {
  const char* fn = "pced_sample";
  if (rows < 0 || V < 1 || stride < V) return fail(PCED_ERR_INVALID_ARG, "%s: sizes", fn);
  if (type != PCED_IN_F32 && type != PCED_IN_BF16) return fail(PCED_ERR_INVALID_ARG, "%s: no such type", fn);
  if (rows == 0) return PCED_OK;
  if (!x || !u || !token) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (!aligned(x, type == PCED_IN_F32 ? 4 : 2) || !aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
      !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(token, 4) || !aligned(logprob, 4) || !aligned(status, 4))
    return fail(PCED_ERR_INVALID_ARG, "%s: misaligned pointer", fn);
  if (V > SMP_MAX_V) return fail(PCED_ERR_UNSUPPORTED, "%s: V above %d", fn, SMP_MAX_V);
  if ((int64_t)rows * ROW_CLUSTER > INT32_MAX) return fail(PCED_ERR_UNSUPPORTED, "%s: too many rows", fn);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  const SampleArgs a = {x, stride, V, 0, u, temperature, top_k, top_p, min_p, token, logprob, status};
  const cudaError_t e = type == PCED_IN_F32 ? launch_sample<float>(a, rows, (cudaStream_t)stream)
                                             : launch_sample<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "sample launch");
}
