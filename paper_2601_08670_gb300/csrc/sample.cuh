// sample.cuh -- a token for every row of logits from a given random number, by
// temperature, top-k, top-p and min-p (pced_sample).
//
// With m the row's largest logit, w_v = exp((x_v - m) / t).  Ordered by logit, then by
// token, a cut keeps the first tokens: the top k, the shortest prefix of them that holds
// p of their weight, those of weight min_p or more.  The token is the first kept one, in
// the order of the vocabulary, up to which the kept weights sum to more than u of all.
//
// A sum over a vocabulary decides at which token u falls, and its error counts 150,000
// times (every border of two tokens is a place to be wrong): with weights of 24 bits one row
// in some thousands gets another token than in 64 bits.  So weights are exact to 2^-30
// of themselves, and are added with 2^-42 lost in sixteen (see Sum).
//
// A cluster of CTAs reads a row two to four times, from L2 after the first: for its largest logit,
// for its weights, for what a cut leaves.  A cut is found by counting the tokens in equal
// ranges of the weights' logarithm.  For the top k a bound comes from the threads' largest logits,
// and the tokens above it are listed; for the top p the counts bound the weights to half a percent, so
// that a few ranges are left, whose tokens are listed and weighed.  What a list holds goes into
// finer ranges, of which one is ranked token by token.  Ranges with too many tokens (of equal
// logits, say) are split by (logit, token) pairs as 64-bit numbers, again and again: pairs are
// distinct, so that ends.  Few tokens that are left go to one CTA, which ends alone.
//
// What bounds it (one GB300, GPU time in a graph).  Many rows: 272 of 151936 fp32 logits 48 us for
// the largest logit alone (3.4 TB/s, half of the copy rate: a warp has one group's loads in flight),
// without a cut 84 (a weight and its sum take about 24 instructions a token), top 50 79 (the same
// first pass and one that lists), p = 0.9 190 (a count and a second weight, and about 45,000 cycles a
// CTA of small steps between barriers), mixed cuts 142 to 154 of a floor of 24.5; the warps issue
// in 35 to 60 % of the slots, so loads and barriers are waited for as well.  Few rows:
// those steps.  A row of 128256 5.0 us at t = 0, 9.4 without a cut, 12.7 for the top 50, 29 for
// p = 0.9; a barrier of a cluster costs 900 cycles, what its CTAs read of one another 10 bytes a clock.
#pragma once

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
constexpr int SMP_BINS = 1024;        // ranges
constexpr int SMP_COARSE = 2 * SMP_BINS;  // ranges of all weights, a 64th of their log2 each
constexpr int SMP_FEW = 512;          // tokens of a range that are ranked one by one
constexpr int SMP_EACH = 16;          // tokens of a lane in a group, whose weight is kept
constexpr int SMP_GROUP = 32 * SMP_EACH;
constexpr int SMP_FINE = 256;         // ranges that a cluster weighs (what its CTAs read of one another is slow)
constexpr int SMP_LIST = 4608;        // tokens that a CTA's list takes
constexpr int SMP_SOLO = 4096;        // tokens of a row that one CTA goes on with alone
constexpr int SMP_QUEUE = 32 * 8 + 32;  // tokens of a warp on their way to whole warps: half a group and a rest
constexpr int SMP_RANK = 128;         // tokens that are ranked at once
constexpr int SMP_LONG = 65536;       // tokens of a row that two CTAs share where rows wait
constexpr int SMP_MAX_V = 393216;     // (sets the groups)
constexpr int SMP_MAX_GROUPS = SMP_MAX_V / SMP_GROUP + 1;
constexpr int SMP_UNIT = 42;          // weights are counted in steps of 2^-42
constexpr int SMP_PART = 14;          // bits of a weight that are added up in one number of 32
constexpr int SMP_MAX_PER = (1 << 18) - 1;  // tokens of a CTA: as many such parts as fit, also of the uppermost
constexpr float SMP_ALIVE = 44.f;     // -log2 of weights that no cut asks about
constexpr float SMP_LOWEST = 100.f;   // ... and that are nothing

// {2^(j / 64) as fp32, log2 of what it has to be multiplied by}
struct Exp2Entry {
  uint32_t bits;
  float rest;
};
constexpr int SMP_EXP2 = 64;
__device__ const Exp2Entry kExp2Table[SMP_EXP2] = {
    {0x3F800000u, 0.f}, {0x3F8164D2u, -8.15134182e-09f}, {0x3F82CD87u, -6.79286885e-08f}, {0x3F843A29u, -3.92309936e-08f},
    {0x3F85AAC3u, 6.67758187e-08f}, {0x3F871F62u, -6.70637164e-08f}, {0x3F88980Fu, -8.02199409e-08f}, {0x3F8A14D5u, 7.30413632e-08f},
    {0x3F8B95C2u, -1.73010264e-08f}, {0x3F8D1ADFu, 5.57574609e-08f}, {0x3F8EA43Au, -7.03689835e-08f}, {0x3F9031DCu, 4.00033358e-08f},
    {0x3F91C3D3u, 6.82363321e-08f}, {0x3F935A2Bu, 2.74734742e-08f}, {0x3F94F4F0u, -5.02265998e-08f}, {0x3F96942Du, 3.14805497e-08f},
    {0x3F9837F0u, 4.60712819e-08f}, {0x3F99E046u, -6.0841586e-08f}, {0x3F9B8D3Au, -3.87892598e-08f}, {0x3F9D3EDAu, -4.85744387e-08f},
    {0x3F9EF532u, 5.22408143e-08f}, {0x3FA0B051u, 8.41478265e-09f}, {0x3FA27043u, 1.61354052e-09f}, {0x3FA43516u, -4.29211156e-08f},
    {0x3FA5FED7u, -4.47101591e-08f}, {0x3FA7CD94u, -3.84792926e-08f}, {0x3FA9A15Bu, -3.80626375e-08f}, {0x3FAB7A3Au, -3.72789515e-08f},
    {0x3FAD583Fu, -1.07844533e-08f}, {0x3FAF3B79u, -4.05290344e-08f}, {0x3FB123F6u, -6.12515763e-08f}, {0x3FB311C4u, 8.96096175e-09f},
    {0x3FB504F3u, 2.46906744e-08f}, {0x3FB6FD92u, -1.35528202e-08f}, {0x3FB8FBAFu, 3.3184822e-08f}, {0x3FBAFF5Bu, -3.58339562e-08f},
    {0x3FBD08A4u, -4.39687788e-08f}, {0x3FBF179Au, -3.30846959e-08f}, {0x3FC12C4Du, -2.38600659e-08f}, {0x3FC346CDu, -1.6670608e-08f},
    {0x3FC5672Au, 7.55010543e-09f}, {0x3FC78D75u, -2.3842496e-08f}, {0x3FC9B9BEu, -5.18225391e-08f}, {0x3FCBEC15u, -4.440113e-10f},
    {0x3FCE248Cu, 8.8113925e-09f}, {0x3FD06334u, -1.52952193e-08f}, {0x3FD2A81Eu, -4.49263098e-08f}, {0x3FD4F35Bu, -3.39957644e-08f},
    {0x3FD744FDu, -2.12359019e-08f}, {0x3FD99D16u, -2.43133815e-08f}, {0x3FDBFBB8u, -4.07101162e-08f}, {0x3FDE60F5u, -4.85806915e-08f},
    {0x3FE0CCDFu, -7.58683782e-09f}, {0x3FE33F89u, 4.34195506e-08f}, {0x3FE5B907u, -9.17609899e-09f}, {0x3FE8396Au, 2.97107601e-08f},
    {0x3FEAC0C7u, -8.84121043e-09f}, {0x3FED4F30u, 1.11787655e-08f}, {0x3FEFE4BAu, -3.58948427e-08f}, {0x3FF28177u, 2.14003624e-08f},
    {0x3FF5257Du, 7.41633155e-09f}, {0x3FF7D0DFu, 3.99192928e-08f}, {0x3FFA83B3u, -1.25475035e-08f}, {0x3FFD3E0Cu, 4.39907888e-09f}};

// What a row's weights are made with.  y = x log2(e) / t, from a factor in two parts, is
// p + low, p rounded to q / 64, q whole, what is left r; w = 2^(y - N), N the ceiling of the largest
// y (so the largest weight lies in (1/2, 1]).  2^(q / 64 - N) comes from a table that the
// row's CTA makes (16 copies side by side, so that a warp's lanes do not meet on banks),
// and what its number is short of goes into r; 2^r - 1 comes from its series to r^3.
// Off by at most 2^-30 of itself: r's rounding (at most 2^-31, times ln 2), the last product's and the inner
// sum's (2^-32 each), what the series leaves out (2^-34.7), and y's (2^-34 at |y| = 8192).
struct Weight {
  float ch, cl;            // ch + cl = log2(e) / t
  float floor;             // logits are taken as this at least: 2^-SMP_LOWEST
  const float2* table;     // this lane's copy
  // a (1 + g): the weight
  __device__ __forceinline__ void of(float x, float& a, float& g) const {
    constexpr float MAGIC = 196608.f;  // 1.5 2^17: sums with it are rounded to 64ths; its low bits are 0
    x = fmaxf(x, floor);               // (also of what is not a number)
    const float p = __fmul_rn(x, ch);
    const float low = fmaf(x, cl, fmaf(x, ch, -p));
    const float shifted = __fadd_rn(p, MAGIC);
    const uint32_t q = __float_as_uint(shifted);
    const float2 e = *reinterpret_cast<const float2*>(reinterpret_cast<const char*>(table) + (q << 7 & 0x1F80u));
    const float r = __fadd_rn(__fsub_rn(p, __fsub_rn(shifted, MAGIC)), __fadd_rn(low, e.y));
    a = __uint_as_float(__float_as_uint(e.x) + (q << 17));  // (the entries make up for what q's low bits add)
    g = __fmul_rn(r, fmaf(r, fmaf(r, 5.55041087e-2f, 2.40226507e-1f), 6.93147181e-1f));
  }
};
static_assert(SMP_EXP2 == 64, "the bits of q");

// A sum of weights, at most SMP_EACH of them: what fits the grid of 2^-18 that numbers from
// 32 to 64 have is added exactly, the rest, below 2^-19 each, beside it.
struct Sum {
  float high = 32.f, low = 0.f;
  __device__ __forceinline__ void add(float a, float g) {
    const float h1 = __fadd_rn(high, a);
    low += __fsub_rn(a, __fsub_rn(h1, high));
    const float h2 = fmaf(a, g, h1);
    low += fmaf(a, g, -__fsub_rn(h2, h1));
    high = h2;
  }
  // in whole steps of 2^-SMP_UNIT: high part of 2^-18, low part from 0 to 2^24 - 1
  __device__ __forceinline__ void parts(int& h, int& l) const {
    h = __float_as_int(high) - __float_as_int(32.f);
    l = __float2int_rn(low * (float)((uint64_t)1 << SMP_UNIT));
    h += l >> 24;
    l &= 0xFFFFFF;
  }
  __device__ __forceinline__ uint64_t steps() const {
    int h, l;
    parts(h, l);
    return (uint64_t)(((int64_t)h << 24) + l);
  }
  __device__ __forceinline__ uint64_t warp_steps() const {
    int h, l;
    parts(h, l);
    h = __reduce_add_sync(0xffffffffu, h);
    l = __reduce_add_sync(0xffffffffu, l);
    return (uint64_t)(((int64_t)h << 24) + l);
  }
};
static_assert(SMP_UNIT == 42, "18 + 24");
static_assert(((uint64_t)SMP_MAX_PER << SMP_PART) >> 32 == 0 && SMP_UNIT <= 3 * SMP_PART,
              "sums of parts, 2^SMP_UNIT itself among them");
static_assert(SMP_MAX_V <= (int64_t)SMP_MAX_PER * ROW_CLUSTER, "parts of a row");
static_assert(SMP_SOLO <= SMP_LIST, "one CTA's list");
static_assert(SMP_BINS == 4 * SMP_FINE, "see keep_share");

// Order of (logit, token) pairs: larger logits first, then lower tokens
__device__ __forceinline__ uint64_t pair_of(float x, int token) {
  const uint32_t b = __float_as_uint(x + 0.f);  // (-0 is 0)
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~token;
}
// The last kept pair: x, then token.
struct Cut {
  float x = -INFINITY;
  int token = INT32_MAX;
  __device__ __forceinline__ bool keeps(float v, int t) const { return v > x || (v == x && t <= token); }
  __device__ __forceinline__ void set(uint64_t pair) {
    const uint32_t k = (uint32_t)(pair >> 32);
    x = __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
    token = (int)~(uint32_t)pair;
  }
};

template <typename T>
struct Words;  // 16 bytes of logits
template <>
struct Words<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void split(uint4 v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
  }
};
template <>
struct Words<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void split(uint4 v, float (&x)[8]) {
    x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
    x[4] = bf16_lo(v.z), x[5] = bf16_hi(v.z), x[6] = bf16_lo(v.w), x[7] = bf16_hi(v.w);
  }
};

// Equal ranges of x, in 64ths: the float MAGIC + 64ths has them in its low bits.
struct Ranges {
  static constexpr float MAGIC = 131072.f;  // 2^17
  float top, per;                           // the first one's upper end; ranges of a unit of x
  __device__ __forceinline__ void set(float top_, float width) {  // SMP_BINS - 4 ranges from top down
    top = top_;
    per = (float)(SMP_BINS - 4) / fmaxf(width, 1e-30f);
  }
  // (1 + 64 (top - x) per, rounded)
  __device__ __forceinline__ int place(float x) const {
    return __float_as_int(fmaf(top - x, per, MAGIC + 1.f / 64)) - __float_as_int(MAGIC);
  }
};

// The first range that brings the sum to the target, and what lies before it.
struct Border {
  bool found;
  uint32_t bin, n;  // n: tokens in it
  uint64_t before;
};

struct SampleShared {
  float2 table[SMP_EXP2][16];
  // tokens of the ranges, then their weights, SMP_PART bits each (of SMP_BINS ranges); or the
  // tokens of SMP_COARSE ranges (16 bits each where a part has no more)
  uint32_t ranges[4][SMP_BINS];
  uint64_t cand[SMP_FEW];
  uint64_t group[SMP_MAX_GROUPS];  // kept weight (on its way in two numbers, 21 bits in the first)
  uint32_t n_list, n_cand;
  int from, to;                  // places of this CTA's part
  float ym, inverse;             // log2 of the largest weight; t / log2(e)
  float thread_max[SMP_THREADS]; // the largest logit that a thread loaded first
  int at[4];
  uint64_t wscan[SMP_WARPS];
  uint32_t wkept[SMP_WARPS];
  float2 fscan[SMP_WARPS];
  Border border;
  float threshold;
  double below;  // of a min_p: t log(p), t the temperature that counts
  uint64_t cut;
  // what the cluster's warps tell one another: two of each, by turns, with a barrier of the
  // cluster between a write and its reads, so that the next write to one comes after them
  struct alignas(16) Told {
    int mx[SMP_WARPS];
    uint64_t sum[SMP_WARPS], lo[SMP_WARPS], hi[SMP_WARPS];
    uint32_t count;
  } told[2];

  // When a range is ranked the histograms are free: this CTA's candidates and their weights,
  // all the cluster's and theirs.
  __device__ __forceinline__ uint64_t* candidates(int which) { return which ? reinterpret_cast<uint64_t*>(ranges[which]) : cand; }
};
static_assert(SMP_BINS * 4 >= SMP_FEW * 8, "room for the candidates");

// floats as whole numbers of the same order
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x);
  return b >= 0 ? b : b ^ 0x7FFFFFFF;
}
__device__ __forceinline__ float from_ordered(int b) { return __int_as_float(b >= 0 ? b : b ^ 0x7FFFFFFF); }

template <typename T>
struct Row {
  static constexpr int W = Words<T>::N, TILES = SMP_EACH / W;  // logits of 16 bytes; 16 bytes of a lane in a group
  const SampleArgs& a;
  SampleShared& s;
  cg::cluster_group cluster;
  const uint4* data;                   // this CTA's part of the row, from an address of 16 bytes on
  float2* left;                        // the list: (logit, token)
  int first, groups;                   // token of place 0
  int ctas, turn;
  float mx;                            // the row's largest logit
  Weight w;
  float origin;                        // see moved()
  bool back;                           // see each_group()
  float alive;                         // smaller logits have weights that no cut asks about
  float whole;                         // N: the largest weight lies in (1/2, 1] 2^N
  Cut cut;
  float low;                           // smaller logits are not kept
  bool listed;                         // the others' places are in the list (each CTA's own matter, as is `low`)
  int solo;                            // > 0: so many tokens are left, and this CTA, which has them, alone
  bool gone;                           // ... another CTA
  bool grouped;                        // the groups' kept weight is known; the list has a part of the tokens only

  static __device__ __forceinline__ int tid() { return threadIdx.x; }
  static __device__ __forceinline__ int lane() { return threadIdx.x & 31; }
  static __device__ __forceinline__ int warp() { return threadIdx.x >> 5; }
  static __device__ __forceinline__ int rank() { return cg::this_cluster().block_rank(); }
  __device__ __forceinline__ typename SampleShared::Told& mine() { return s.told[turn & 1]; }
  __device__ __forceinline__ const typename SampleShared::Told& theirs(int r) {
    return cluster.map_shared_rank(&s, r)->told[turn & 1];
  }
  // A logit as it counts.  Where |m| / t is very large, logits are taken as differences from m:
  // those that count lie so near to it that they are exact.  (A row with +inf is 0 there
  // and -inf elsewhere.)
  __device__ __forceinline__ float moved(float x) const {
    if (origin != 0.f) x = origin == INFINITY ? (x == origin ? 0.f : -INFINITY) : x - origin;
    return x;
  }
  __device__ __forceinline__ float at(int place) const {
    if (place < s.from || place >= s.to) return -INFINITY;
    return moved((float)reinterpret_cast<const T*>(data)[place]);
  }
  // f(e, logit, place) for the SMP_EACH places of a lane in group g (-inf around the part)
  template <typename F>
  __device__ __forceinline__ void each_of(int g, F f) const {
    float x[TILES][W];
    const int v0 = g * TILES * 32 + lane();
    if (g * SMP_GROUP >= s.from && (g + 1) * SMP_GROUP <= s.to) {
      uint4 w[TILES];
#pragma unroll
      for (int t = 0; t < TILES; ++t) w[t] = data[v0 + t * 32];
#pragma unroll
      for (int t = 0; t < TILES; ++t) Words<T>::split(w[t], x[t]);
    } else {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const int place = (v0 + t * 32) * W;
        if (place >= s.from && place + W <= s.to) {
          Words<T>::split(data[v0 + t * 32], x[t]);
        } else {
#pragma unroll
          for (int e = 0; e < W; ++e)
            x[t][e] = place + e >= s.from && place + e < s.to ? (float)reinterpret_cast<const T*>(data)[place + e] : -INFINITY;
        }
      }
    }
    if (origin != 0.f) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < W; ++e) x[t][e] = moved(x[t][e]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < W; ++e) f(t * W + e, x[t][e], (v0 + t * 32) * W + e);
  }
  // f(group) for the warp's groups, every time the other way round: what was read last is
  // what L2 still has
  template <typename F>
  __device__ __forceinline__ void each_group(F f) {
    back = !back;
    for (int i = warp(); i < groups; i += SMP_WARPS) f(back ? groups - 1 - i : i);
  }
  // A barrier of the CTAs that still work on the row.
  __device__ __forceinline__ void meet() {
    if (solo) __syncthreads();
    else cluster.sync();
  }
  // f(logit, token) for the tokens that `low` leaves, a lane each
  template <typename F>
  __device__ __forceinline__ void each_left(F f) {
    if (listed) {
      const int k = solo ? solo : (int)s.n_list;
      for (int i = tid(); i < k; i += SMP_THREADS) f(left[i].x, __float_as_int(left[i].y));
      return;
    }
    float2* const q = left + SMP_LIST + warp() * SMP_QUEUE;
    int held = 0;
    each_group([&](int g) {
      uint32_t take = 0;
      each_of(g, [&](int e, float x, int) { take |= (uint32_t)(x >= low) << e; });
      if (!__any_sync(0xffffffffu, take)) return;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t mine = take >> (8 * half) & 0xFFu;
        const int k = __popc(mine);
        int to = k;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, to, o);
          if (lane() >= o) to += y;
        }
        float2* at = q + held + to - k;
        each_of(g, [&](int e, float x, int place) {
          if (e / 8 == half && (take >> e & 1u)) *at++ = make_float2(x, __int_as_float(first + place));
        });
        held += __shfl_sync(0xffffffffu, to, 31);
        __syncwarp();
        while (held >= 32) {  // (the last ones first)
          held -= 32;
          const float2 y = q[held + lane()];
          f(y.x, __float_as_int(y.y));
        }
        __syncwarp();
      }
    });
    __syncwarp();
    if (lane() < held) f(q[lane()].x, __float_as_int(q[lane()].y));
    __syncwarp();
  }
  // Where few tokens are left, CTA 0 takes them all (logit, token) and goes on alone: a barrier of
  // a cluster takes half a microsecond, and what its CTAs read of one another 10 bytes a clock.
  __device__ __forceinline__ void try_solo() {
    if (ctas == 1) {
      if (listed) solo = s.n_list;
      return;
    }
    if (tid() == 0) mine().count = listed ? s.n_list : SMP_SOLO + 1;
    cluster.sync();
    const int k = lane() < ctas ? (int)theirs(lane()).count : 0;
    ++turn;
    int to = k;
#pragma unroll
    for (int o = 1; o < ROW_CLUSTER; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, to, o);
      if (lane() >= o) to += y;
    }
    const int total = __shfl_sync(0xffffffffu, to, ROW_CLUSTER - 1);
    if (total > SMP_SOLO) return;
    gone = rank() != 0;
    // two warps for each CTA
    const int r = warp() / 2, their_n = __shfl_sync(0xffffffffu, k, r), base = __shfl_sync(0xffffffffu, to, r) - their_n;
    if (rank() == 0 && r > 0 && r < ctas) {
      const float2* theirs_ = cluster.map_shared_rank(left, r);
      for (int i = tid() & 63; i < their_n; i += 64) left[base + i] = theirs_[i];
    }
    cluster.sync();  // (CTA 0 has read the others' memory)
    if (rank() == 0) {
      ctas = 1;
      solo = total;
    }
  }
  // The list of the tokens from `low_` on, where they are few enough.
  __device__ __forceinline__ void list(float low_) {
    low = low_;
    listed = false;
    __syncthreads();
    if (tid() == 0) s.n_list = 0;
    __syncthreads();
    each_group([&](int g) {
      uint32_t take = 0;
      each_of(g, [&](int e, float x, int) { take |= (uint32_t)(x >= low) << e; });
      if (!__any_sync(0xffffffffu, take)) return;
      const int k = __popc(take);
      int to = k;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, to, o);
        if (lane() >= o) to += y;
      }
      int base = 0;
      if (lane() == 31) base = (int)atomicAdd(&s.n_list, (uint32_t)to);
      base = __shfl_sync(0xffffffffu, base, 31) + to - k;
      each_of(g, [&](int e, float x, int place) {
        if ((take >> e & 1u) && base < SMP_LIST) left[base] = make_float2(x, __int_as_float(first + place));
        base += take >> e & 1u;
      });
    });
    __syncthreads();
    listed = s.n_list <= SMP_LIST;
  }

  // m, N and the table for temperature t (inverse: 1 / w.ch, entries: this thread's of the table)
  __device__ __forceinline__ void set_weights(float inverse, const Exp2Entry (&entries)[2]) {
    if (!(fabsf(mx) * w.ch <= 8192.f)) {
      origin = mx;
      s.thread_max[tid()] = moved(s.thread_max[tid()]);
      mx = 0.f;
    }
    const float y = __fmul_rn(mx, w.ch), top = ceilf(y);
    w.floor = (top - SMP_LOWEST) * inverse;
    alive = (top - SMP_ALIVE) * inverse;
    low = alive;
    listed = gone = grouped = false;
    solo = 0;
    w.table = &s.table[0][lane() & 15];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t j = tid() / 16 + i * (SMP_THREADS / 16);
      s.table[j][tid() % 16] =
          make_float2(__uint_as_float(entries[i].bits - (j << 17) - ((uint32_t)(int)top << 23)), entries[i].rest);
    }
    whole = top;
    if (tid() == 0) {
      s.ym = (y - top) + fmaf(mx, w.cl, fmaf(mx, w.ch, -y));
      s.inverse = inverse;
    }
    __syncthreads();
  }

  // The cluster's sum of the warps' sums, of the CTAs before this one, and this one's.
  struct Sums {
    uint64_t all, before, own;
  };
  __device__ __forceinline__ Sums sum_up(uint64_t v) {
    if (lane() == 0) mine().sum[warp()] = v;
    meet();
    // a CTA's sixteen by four lanes
    const int r = lane() >> 2;
    uint64_t of_cta = 0;
    if (r < ctas) {
      const uint64_t* q = theirs(r).sum + (lane() & 3) * (SMP_WARPS / 4);
      const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(q), y = *reinterpret_cast<const ulonglong2*>(q + 2);
      of_cta = x.x + x.y + y.x + y.y;
    }
    of_cta += __shfl_xor_sync(0xffffffffu, of_cta, 1);
    of_cta += __shfl_xor_sync(0xffffffffu, of_cta, 2);
    Sums z;
    z.own = __shfl_sync(0xffffffffu, of_cta, 4 * rank());
    z.all = of_cta, z.before = r < rank() ? of_cta : 0;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      z.all += __shfl_xor_sync(0xffffffffu, z.all, o);
      z.before += __shfl_xor_sync(0xffffffffu, z.before, o);
    }
    ++turn;
    return z;
  }

  // Weight of all tokens; COUNT: those from `from` on in the coarse ranges too
  template <bool COUNT>
  __device__ __forceinline__ Sums weigh_all(float from) {
    uint64_t total = 0;
    each_group([&](int g) {
      Sum sum;
      each_of(g, [&](int, float x, int) {
        float b, c;
        w.of(x, b, c);
        sum.add(b, c);
        if (COUNT) count_coarse(x, from);
      });
      const uint64_t v = sum.warp_steps();
      if (lane() == 0) s.group[g] = v;
      total += v;
    });
    return sum_up(total);
  }
  // ... of the kept ones among those that `low` leaves; COUNT: all of them in the coarse ranges too
  template <bool COUNT>
  __device__ __forceinline__ Sums weigh_kept() {
    __syncthreads();
    uint64_t total = 0;
    each_left([&](float x, int token) {
      if (!cut.keeps(x, token)) return;
      total += steps_of(x);
      if (COUNT) count_coarse(x, alive);
    });
    return sum_up(warp_sum64(total));
  }
  // ... by groups
  __device__ __forceinline__ Sums weigh_groups() {
    uint64_t total = 0;
    __syncthreads();
    if (listed) {
      for (int g = tid(); g < groups; g += SMP_THREADS) s.group[g] = 0;
      __syncthreads();
      uint32_t* const part = reinterpret_cast<uint32_t*>(s.group);
      each_left([&](float x, int token) {
        if (!cut.keeps(x, token)) return;
        const uint64_t v = steps_of(x);
        const int g = (token - first) / SMP_GROUP;
        atomicAdd(part + 2 * g, (uint32_t)v & 0x1FFFFFu);
        atomicAdd(part + 2 * g + 1, (uint32_t)(v >> 21));
      });
      __syncthreads();
      for (int g = tid(); g < groups; g += SMP_THREADS) {
        const uint64_t v = part[2 * g] + ((uint64_t)part[2 * g + 1] << 21);
        s.group[g] = v;
        total += v;
      }
      total = warp_sum64(total);
    } else {
      each_group([&](int g) {
        Sum sum;
        bool some = false;
        each_of(g, [&](int, float x, int place) {
          const bool k = x >= low && cut.keeps(x, first + place);
          if (!__any_sync(0xffffffffu, k)) return;
          some = true;
          float b, c;
          w.of(x, b, c);
          sum.add(k ? b : 0.f, c);
        });
        const uint64_t v = some ? sum.warp_steps() : 0;
        if (lane() == 0) s.group[g] = v;
        total += v;
      });
    }
    return sum_up(total);
  }
  // Where a logit lies below 2^N, in 2048ths of the weights' log2 (by the larger part of y, which
  // rises with x, and is at most N; the fp32 number 4096 + such has them in its low bits), and its
  // range, a 32nd.
  __device__ __forceinline__ float place_float(float x) const {
    return __fsub_rn(whole + 4096.f, __fmul_rn(fmaxf(x, w.floor), w.ch));
  }
  __device__ __forceinline__ int place_of(float x) const { return __float_as_int(place_float(x)) - __float_as_int(4096.f); }
  __device__ __forceinline__ int range_of(float x) const { return min(place_of(x) >> 6, SMP_BINS - 1); }
  // a logit that those of the ranges up to `bin` are not below (which are `per` of log2)
  __device__ __forceinline__ float below(int bin, int bins = SMP_BINS, float per = 1.f / 32) const {
    return bin >= bins - 1 ? -INFINITY : (whole - ((float)bin + 1.25f) * per) * s.inverse;
  }
  // Counts x in its coarse range if it is `from` or more (alive at least); a predicate, no branch:
  // with one, and a second atomic for a mean in ranges twice as wide, 272 rows of 151936 at
  // p = 0.9 take 203 us for 190.
  __device__ __forceinline__ void count_coarse(float x, float from) {
    const int narrow = !wide(), bin = min((int)(__float_as_uint(place_float(x)) >> 5 & 0x3FFFFu), SMP_COARSE - 1);
    const uint32_t at = smem_u32(&s.ranges[0][0]) + ((bin >> narrow) << 2), n = 1u << ((bin & narrow) << 4);
    asm volatile("{\n.reg .pred p;\nsetp.ge.f32 p, %2, %3;\n@p red.shared.add.u32 [%0], %1;\n}" ::"r"(at), "r"(n), "f"(x), "f"(from)
                 : "memory");
  }
  __device__ __forceinline__ bool wide() const { return a.per > 0xFFFF; }
  __device__ __forceinline__ void count_in(int bin) {
    uint32_t* const n = &s.ranges[0][0];
    if (wide()) atomicAdd(n + bin, 1u);
    else atomicAdd(n + (bin >> 1), 1u << (16 * (bin & 1)));
  }
  static __device__ __forceinline__ uint64_t warp_sum64(uint64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }

  // Two ranges' tokens of the cluster, each thread its own; MASS: and their weights.
  template <bool MASS>
  __device__ __forceinline__ void gather_ranges(uint32_t (&n)[2], uint64_t (&m)[2]) {
    static_assert(SMP_BINS == 2 * SMP_THREADS && ROW_CLUSTER == 8, "two ranges a thread");
    n[0] = n[1] = 0;
    m[0] = m[1] = 0;
    if (MASS && !solo && 2 * tid() >= SMP_FINE) return;
    constexpr int PARTS = MASS ? 3 : 0, BATCH = MASS ? 2 : 4;  // CTAs whose loads are in flight
#pragma unroll
    for (int r0 = 0; r0 < ROW_CLUSTER; r0 += BATCH) {
      if (r0 >= ctas) break;
      uint2 c[BATCH], b[BATCH][PARTS + 1];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        c[k] = make_uint2(0, 0);
        if (r0 + k >= ctas) continue;
        const SampleShared& o = *cluster.map_shared_rank(&s, r0 + k);
        if (wide()) c[k] = *reinterpret_cast<const uint2*>(&o.ranges[0][2 * tid()]);
        else c[k].x = o.ranges[0][tid()], c[k].y = c[k].x >> 16, c[k].x &= 0xFFFFu;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) b[k][i] = *reinterpret_cast<const uint2*>(&o.ranges[1 + i][2 * tid()]);
      }
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        n[0] += c[k].x, n[1] += c[k].y;
        if (r0 + k >= ctas) continue;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) m[0] += (uint64_t)b[k][i].x << (SMP_PART * i), m[1] += (uint64_t)b[k][i].y << (SMP_PART * i);
      }
    }
  }
  // The first range that brings the sum of the tokens' number (MASS: weight) to the target,
  // after a barrier: all histograms are complete.  One follows here: all have read them.
  template <bool MASS>
  __device__ __forceinline__ Border find_border(uint64_t target) {
    uint32_t n[2];
    uint64_t m[2];
    gather_ranges<MASS>(n, m);
    if (!MASS) m[0] = n[0], m[1] = n[1];
    uint64_t to = prefix(m[0] + m[1]);
    __syncthreads();
    if (lane() == 31) s.wscan[warp()] = to;
    if (tid() == 0) s.border.found = false;
    __syncthreads();
    const uint64_t ahead = lane() < warp() ? s.wscan[lane()] : 0;  // (warp < 16)
    to += warp_sum64(ahead);
    uint64_t from = to - m[0] - m[1];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (from < target && from + m[j] >= target) {
        s.border.found = true, s.border.bin = 2 * tid() + j, s.border.n = n[j], s.border.before = from;
      }
      from += m[j];
    }
    meet();
    return s.border;
  }

  __device__ __forceinline__ void clear_ranges(bool mass) {
    __syncthreads();
    for (int i = tid(); i < SMP_BINS; i += SMP_THREADS) {
      s.ranges[0][i] = 0;
      if (mass) s.ranges[1][i] = s.ranges[2][i] = s.ranges[3][i] = 0;
    }
    __syncthreads();
  }
  __device__ __forceinline__ uint64_t steps_of(float x) const {
    Sum one;
    float b, c;
    w.of(x, b, c);
    one.add(b, c);
    return one.steps();
  }
  __device__ __forceinline__ void add_to_range(int bin, uint64_t v) {
    count_in(bin);
    constexpr uint32_t MASK = (1u << SMP_PART) - 1;
    atomicAdd(&s.ranges[1][bin], (uint32_t)v & MASK);
    atomicAdd(&s.ranges[2][bin], (uint32_t)(v >> SMP_PART) & MASK);
    atomicAdd(&s.ranges[3][bin], (uint32_t)(v >> (2 * SMP_PART)));
  }

  // The cut among the tokens in(x, token), `n` of the cluster: the one that brings the sum
  // of their number (MASS: weight) to the target.
  template <bool MASS, typename F>
  __device__ __forceinline__ void cut_among(uint32_t n, uint64_t target, F in) {
    if (n <= SMP_FEW) {
      rank_few<MASS>(target, in);
      return;
    }
    uint64_t lo = ~(uint64_t)0, hi = 0;
    each_left([&](float x, int token) {
      if (in(x, token)) {
        const uint64_t p = pair_of(x, token);
        lo = min(lo, p), hi = max(hi, p);
      }
    });
    warp_bounds(lo, hi);
    if (lane() == 0) mine().lo[warp()] = lo, mine().hi[warp()] = hi;
    meet();
    lo = ~(uint64_t)0, hi = 0;
    for (int i = lane(); i < ctas * SMP_WARPS; i += 32) {
      const auto& o = theirs(i / SMP_WARPS);
      lo = min(lo, o.lo[i % SMP_WARPS]), hi = max(hi, o.hi[i % SMP_WARPS]);
    }
    warp_bounds(lo, hi);
    ++turn;
    for (int level = 0; level < 9; ++level) {  // (each takes eight bits or more off 64)
      const int shift = max(0, (MASS && !solo ? 56 : 54) - __clzll((long long)(hi - lo)));
      const auto inside = [&](float x, int token) {
        const uint64_t p = pair_of(x, token);
        return p >= lo && p <= hi;
      };
      clear_ranges(true);
      each_left([&](float x, int token) {
        if (!inside(x, token)) return;
        add_to_range((int)((hi - pair_of(x, token)) >> shift), MASS ? steps_of(x) : 0);
      });
      meet();
      const Border b = find_border<MASS>(target);
      if (!b.found) {  // (weights that rounding makes a step too small: to the end of these)
        cut.set(lo);
        return;
      }
      target -= b.before;
      hi -= (uint64_t)b.bin << shift;
      const uint64_t bottom = hi - (((uint64_t)1 << shift) - 1);
      lo = bottom > lo ? bottom : lo;
      if (b.n <= SMP_FEW) {
        rank_few<MASS>(target, inside);
        return;
      }
    }
  }
  static __device__ __forceinline__ void warp_bounds(uint64_t& lo, uint64_t& hi) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
  }

  // ... which every CTA ranks for itself
  template <bool MASS, typename F>
  __device__ __forceinline__ void rank_few(uint64_t target, F in) {
    __syncthreads();
    if (tid() == 0) s.n_cand = 0, s.cut = 0;
    __syncthreads();
    each_left([&](float x, int token) {
      if (!in(x, token)) return;
      const uint32_t i = atomicAdd(&s.n_cand, 1u);
      if (PCED_IN_BOUNDS(i < SMP_FEW, a.status))
        s.candidates(0)[i] = pair_of(x, token), s.candidates(1)[i] = MASS ? steps_of(x) : 1;
    });
    cut.set(rank_candidates(target));
  }
  // Of the cluster's candidates the one that brings the sum of their weights to the target.
  __device__ __forceinline__ uint64_t rank_candidates(uint64_t target) {
    __syncthreads();
    if (tid() == 0) mine().count = s.n_cand;
    meet();
    // the candidates of all CTAs, two warps for each
    uint64_t *pairs = s.candidates(2), *weights = s.candidates(3);
    const int their_n = lane() < ctas ? (int)theirs(lane()).count : 0;
    int to = their_n;
#pragma unroll
    for (int o = 1; o < ROW_CLUSTER; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, to, o);
      if (lane() >= o) to += y;
    }
    const int total = __shfl_sync(0xffffffffu, to, ROW_CLUSTER - 1);
    const int r = warp() / 2, n = __shfl_sync(0xffffffffu, their_n, r), base = __shfl_sync(0xffffffffu, to, r) - n;
    if (r < ctas) {
      SampleShared& o = *cluster.map_shared_rank(&s, r);
      for (int i = tid() & 63; i < n; i += 64)
        if (PCED_IN_BOUNDS(base + i < SMP_FEW, a.status))
          pairs[base + i] = o.candidates(0)[i], weights[base + i] = o.candidates(1)[i];
    }
    ++turn;
    __syncthreads();
    if (tid() < total) {
      const uint64_t own = pairs[tid()], ow = weights[tid()];
      uint64_t before = 0, last = ~(uint64_t)0;
#pragma unroll 4
      for (int i = 0; i < total; ++i) {
        if (pairs[i] > own) before += weights[i];
        last = min(last, pairs[i]);
      }
      // (the last one also where rounding left the sum a step short)
      if (before < target && (before + ow >= target || own == last)) s.cut = own;
    }
    __syncthreads();
    return s.cut;
  }

  // The first k tokens.
  __device__ __forceinline__ void keep_top(int k) {
    // At least k tokens lie from the k-th of the threads' largest logits on, or of those of the
    // lanes in each group, so where k is below their number, their ranges tell where to look.
    const bool few = k <= SMP_THREADS * ctas / 2;
    if (few || k <= a.V / SMP_EACH / 2) {
      clear_ranges(false);
      if (few) {
        if (s.thread_max[tid()] >= alive) count_in(range_of(s.thread_max[tid()]));
      } else {
        each_group([&](int g) {
          float top = -INFINITY;
          each_of(g, [&](int, float x, int) { top = fmaxf(top, x); });
          if (top >= alive) count_in(range_of(top));
        });
      }
      meet();
      const Border b = find_border<false>((uint64_t)k);
      if (b.found) {
        list(fmaxf(alive, below((int)b.bin)));
        try_solo();
        if (gone) return;
      }
    }
    if (solo && solo <= SMP_RANK) {
      if (solo > k) rank_few<false>((uint64_t)k, [](float, int) { return true; });
      return;
    }
    clear_ranges(false);
    each_left([&](float x, int) { count_in(range_of(x)); });
    meet();
    const Border b = find_border<false>((uint64_t)k);
    if (!b.found) {  // there are no more than k; smaller ones may be among the first k, but are nothing
      if (!solo) cut.x = low, cut.token = INT32_MAX;
      return;
    }
    if (!listed) list(fmaxf(alive, below((int)b.bin)));
    cut_among<false>(b.n, k - b.before, [&](float x, int) { return range_of(x) == (int)b.bin; });
  }

  // The shortest first part of the kept tokens that holds `share` of their weight.
  __device__ __forceinline__ void keep_share(double share) {
    if (cut.x != -INFINITY) meet();  // (all have read the candidates of the top k, which lie in the ranges)
    clear_ranges(true);
    constexpr float UNIT = 1.f / (float)((uint64_t)1 << SMP_UNIT);
    uint64_t all;
    float counted = alive, missed = 0.f;  // smaller ones are not counted; bound of their weight
    if (cut.x == -INFINITY && !solo) {
      // Tokens of weight c weigh V c at most, so those of c = (1 - p) / 4 of all / V have no part in
      // the border; all is more than the threads' largest together.
      float b, c;
      w.of(s.thread_max[tid()], b, c);
      const float some = (float)sum_up(warp_sum64((uint64_t)(b * (float)((uint64_t)1 << SMP_UNIT)))).all * UNIT;
      missed = 0.25f * (1.f - (float)share) * some;
      counted = fmaxf(alive, (whole + log2f(missed / (float)a.V)) / w.ch);
      all = weigh_all<true>(counted).all;
    } else {
      all = weigh_kept<true>().all;
    }
    const double want = ceil(share * (double)all);
    const uint64_t target = want < 1.0 ? 1 : (uint64_t)want;
    const Window win = window((float)all * UNIT, (float)want * UNIT, 1.01f * missed);  // (`counted` is rounded)
    if (win.lo == SMP_COARSE) return;  // all are kept
    // the border lies among the logits from `least` on and below `above` (of which all are kept so far)
    const float least = fmaxf(counted, below(win.hi, SMP_COARSE, 1.f / 64));
    const float above = win.lo == 0 ? INFINITY : (whole - ((float)win.lo - 0.25f) * (1.f / 64)) * s.inverse;
    if (!solo && win.through <= SMP_SOLO) {
      listed = false;
      list(least);
      try_solo();
      if (gone) return;
    }
    const Cut old = cut;
    const auto inside = [&](float x, int token) { return x >= least && x < above && old.keeps(x, token); };
    uint64_t before = 0;
    if (solo) {
      each_left([&](float x, int) {
        if (x >= above) before += steps_of(x);
      });
      before = sum_up(warp_sum64(before)).all;
    } else {
      before = group_and_list(least, above, 32 * (int64_t)win.before > a.V);
    }
    const uint64_t rest = target > before ? target - before : 1;
    if (win.inside <= SMP_RANK) {
      rank_few<true>(rest, inside);
    } else {
      // the window's weight in finer ranges (a quarter of them where the cluster weighs)
      Ranges fine;
      const float top = fminf(mx, above);
      fine.set(top, top - least);
      const int shift = solo ? 6 : 8, bins = solo ? SMP_BINS : SMP_FINE;
      const auto bin_of = [&](float x) { return min(max(fine.place(x), 0) >> shift, bins - 1); };
      clear_ranges(true);
      each_left([&](float x, int token) {
        if (inside(x, token)) add_to_range(bin_of(x), steps_of(x));
      });
      meet();
      const Border b = find_border<true>(rest);
      if (!b.found) {  // (weights that rounding makes a step too small: to the end of these)
        if (cut.x < least) cut.x = least, cut.token = INT32_MAX;
      } else {
        cut_among<true>(b.n, rest - b.before, [&](float x, int token) { return inside(x, token) && bin_of(x) == (int)b.bin; });
      }
    }
    if (!solo) {  // the groups' weight with what is kept of the window
      __syncthreads();
      each_left([&](float x, int token) {
        if (inside(x, token) && cut.keeps(x, token))
          atomicAdd((unsigned long long*)&s.group[(token - first) / SMP_GROUP], (unsigned long long)steps_of(x));
      });
      grouped = true;
    }
  }
  // Ranges that can hold the border.  A range's tokens weigh between as many times the weights at
  // its ends (a little apart, as places are rounded); the last one takes what lies lower too, and
  // may weigh nothing.  Summed from the first range on, and from the last one back, where `missed`
  // comes on top, from the weight of all: half a percent of the smaller of both sides.
  struct Window {
    int lo, hi;                        // lo = SMP_COARSE: no range
    uint32_t before, inside, through;  // tokens up to two before them, from there on up to one behind them, in all
  };
  __device__ __forceinline__ Window window(float all, float goal, float missed) {
    static_assert(SMP_COARSE == 4 * SMP_THREADS, "four ranges a thread");
    uint32_t n[4] = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < ROW_CLUSTER; ++r) {
      if (r >= ctas) break;
      const uint32_t* o = &cluster.map_shared_rank(&s, r)->ranges[0][0];
      uint4 c;
      if (wide()) {
        c = *reinterpret_cast<const uint4*>(o + 4 * tid());
      } else {
        const uint2 h = *reinterpret_cast<const uint2*>(o + 2 * tid());
        c = make_uint4(h.x & 0xFFFFu, h.x >> 16, h.y & 0xFFFFu, h.y >> 16);
      }
      n[0] += c.x, n[1] += c.y, n[2] += c.z, n[3] += c.w;
    }
    const float off = 1.f / 4096 + (fabsf(whole) + 64.f) * (1.f / (1 << 23));  // (the roundings of a place and of y)
    const float upper = exp2f((float)tid() * (-4.f / 64) + off) * (1.f + 1.f / (1 << 20)), ratio = exp2f(-1.f / 64 - 2.f * off);
    float up[4], down[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      constexpr float STEP[4] = {1.f, 0.989228f, 0.978572f, 0.968031f};  // 2^(-j / 64), and up
      up[j] = (float)n[j] * (upper * STEP[j]);
      down[j] = 4 * tid() + j == SMP_COARSE - 1 ? 0.f : up[j] * ratio * (1.f - 1.f / (1 << 17));
    }
    float tu = (up[0] + up[1]) + (up[2] + up[3]), td = (down[0] + down[1]) + (down[2] + down[3]);
    uint32_t tn = n[0] + n[1] + n[2] + n[3];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float y = __shfl_up_sync(0xffffffffu, tu, o), z = __shfl_up_sync(0xffffffffu, td, o);
      const uint32_t c = __shfl_up_sync(0xffffffffu, tn, o);
      if (lane() >= o) tu += y, td += z, tn += c;
    }
    __syncthreads();
    if (lane() == 31) s.fscan[warp()] = make_float2(tu, td), s.wkept[warp()] = tn;
    if (tid() == 0) s.at[0] = s.at[1] = SMP_COARSE, s.at[2] = s.at[3] = 0;
    __syncthreads();
    float all_up = 0.f, all_down = 0.f;
    for (int i = 0; i < SMP_WARPS; ++i) {
      const float2 o = s.fscan[i];
      if (i < warp()) tu += o.x, td += o.y, tn += s.wkept[i];
      all_up += o.x, all_down += o.y;
    }
    const float slack = all * (1.f / (1 << 18));  // (sums in fp32)
    {
      float u = tu, d = td;  // up to range 4 tid + j
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        if (fminf(u, all - (all_down - d)) + slack >= goal) atomicMin(&s.at[0], 4 * tid() + j);
        if (fmaxf(d, all - (all_up - u) - missed) - slack >= goal) atomicMin(&s.at[1], 4 * tid() + j);
        u -= up[j], d -= down[j];
      }
    }
    __syncthreads();
    Window z;
    z.lo = s.at[0], z.hi = min(s.at[1], SMP_COARSE - 1);
    {
      uint32_t c = tn;  // tokens up to range b
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        const int b = 4 * tid() + j;
        if (b == z.lo - 2) s.at[2] = c;
        if (b == min(z.hi + 1, SMP_COARSE - 1)) s.at[3] = c;
        c -= n[j];
      }
    }
    meet();  // (all have read the ranges)
    z.before = s.at[2], z.through = s.at[3], z.inside = z.through - z.before;
    return z;
  }
  // Weight by groups of the tokens from `above` on; the list of the kept ones below it from `least` on.
  __device__ __forceinline__ uint64_t group_and_list(float least, float above, bool dense) {
    low = least;
    listed = false;
    __syncthreads();
    if (tid() == 0) s.n_list = 0;
    for (int g = tid(); g < groups; g += SMP_THREADS) s.group[g] = 0;
    __syncthreads();
    uint32_t* const part = reinterpret_cast<uint32_t*>(s.group);
    uint64_t total = 0;
    const auto put = [&](float x, int token) {
      if (!cut.keeps(x, token)) return;
      const uint32_t i = atomicAdd(&s.n_list, 1u);
      if (i < SMP_LIST) left[i] = make_float2(x, __int_as_float(token));
    };
    if (dense) {
      each_group([&](int g) {
        Sum sum;
        uint32_t take = 0;
        each_of(g, [&](int e, float x, int) {
          float b, c;
          w.of(x, b, c);
          sum.add(x >= above ? b : 0.f, c);
          take |= (uint32_t)(x >= least && x < above) << e;
        });
        const uint64_t v = sum.warp_steps();
        if (lane() == 0) s.group[g] = v;
        total += v;
        for (; take; take &= take - 1) {  // (few)
          const int e = __ffs(take) - 1, place = ((g * TILES + e / W) * 32 + lane()) * W + e % W;
          put(at(place), first + place);
        }
        __syncwarp();
      });
    } else {
      each_left([&](float x, int token) {
        if (x < above) {
          put(x, token);
          return;
        }
        const uint64_t m = steps_of(x);
        const int g = (token - first) / SMP_GROUP;
        atomicAdd(part + 2 * g, (uint32_t)m & 0x1FFFFFu);
        atomicAdd(part + 2 * g + 1, (uint32_t)(m >> 21));
      });
      __syncthreads();
      for (int g = tid(); g < groups; g += SMP_THREADS) {
        const uint64_t v = part[2 * g] + ((uint64_t)part[2 * g + 1] << 21);
        s.group[g] = v;
        total += v;
      }
      total = warp_sum64(total);
    }
    __syncthreads();
    listed = s.n_list <= SMP_LIST;
    return sum_up(total).all;
  }
  __device__ __forceinline__ Sums sum_groups() {
    __syncthreads();
    uint64_t total = 0;
    for (int g = tid(); g < groups; g += SMP_THREADS) total += s.group[g];
    return sum_up(warp_sum64(total));
  }

  // Tokens from m + `below` on.
  __device__ __forceinline__ void keep_from(const double& below) {
    __syncthreads();
    if (tid() == 0) s.threshold = __double2float_ru((double)mx + below);
    __syncthreads();
    const float x = s.threshold;
    if (x > cut.x) {
      cut.x = x, cut.token = INT32_MAX;
      if (!solo) {
        if (grouped || (!listed && x > low)) list(x);
        grouped = false;
        try_solo();
      }
    }
  }

  // The token of this CTA's part up to which the kept weights sum to more than `left`, by groups.
  __device__ __forceinline__ void draw(uint64_t left, int64_t row, float t, uint64_t total) {
    // its group: each lane some of them in a row
    const int each = (groups + 31) / 32;
    uint64_t sum = 0;
    for (int i = lane() * each; i < min(groups, (lane() + 1) * each); ++i) sum += s.group[i];
    uint64_t to = prefix(sum);
    const int who = __ffs(__ballot_sync(0xffffffffu, to > left)) - 1;
    left -= __shfl_sync(0xffffffffu, to - sum, who);
    int g = who * each;
    while (left >= s.group[g]) left -= s.group[g++];
    // a thread for each of its tokens
    static_assert(SMP_GROUP == SMP_THREADS, "a thread for each token of a group");
    const int token = first + g * SMP_GROUP + tid();
    const float x = at(g * SMP_GROUP + tid());
    // (without a cut the groups have the smallest weights too)
    const bool keep = cut.x == -INFINITY ? x > -INFINITY : x >= low && cut.keeps(x, token);
    const uint64_t m = keep ? steps_of(x) : 0;
    to = prefix(m);
    if (lane() == 31) s.wscan[warp()] = to;
    const uint32_t kept = __ballot_sync(0xffffffffu, keep);
    if (lane() == 0) s.wkept[warp()] = kept;
    __syncthreads();
    to += warp_sum64(lane() < warp() ? s.wscan[lane()] : 0);
    const bool mine_ = keep && to > left && to - m <= left;
    // (where rounding left the tokens' sum short of the group's: the last kept one)
    const bool in_later_warps = __any_sync(0xffffffffu, lane() > warp() && lane() < SMP_WARPS && s.wkept[lane() & (SMP_WARPS - 1)]);
    const bool last = !__syncthreads_or(mine_) && keep && !in_later_warps && !(kept >> lane() >> 1);
    if (mine_ || last) write(x, token, row, t, total);
  }
  // ... of the tokens that are left to this CTA: by ranges of tokens, then one by one
  __device__ __forceinline__ void draw_solo(uint64_t left, int64_t row, float t, uint64_t total) {
    const int shift = max(0, 22 - __clz(a.V));  // at most SMP_BINS ranges of at most SMP_FEW tokens
    static_assert(SMP_BINS == 1 << 10 && SMP_MAX_V <= SMP_BINS * SMP_FEW, "see there");
    int bin = -1;
    uint64_t before = 0;
    if (solo > SMP_RANK) {
      clear_ranges(true);
      each_left([&](float x, int token) {
        if (cut.keeps(x, token)) add_to_range(token >> shift, steps_of(x));
      });
      __syncthreads();
      const Border b = find_border<true>(left + 1);
      bin = b.bin, before = b.before;
    }
    __syncthreads();
    if (tid() == 0) s.n_cand = 0, s.cut = 0;
    __syncthreads();
    each_left([&](float x, int token) {
      if ((bin >= 0 && token >> shift != bin) || !cut.keeps(x, token)) return;
      const uint32_t i = atomicAdd(&s.n_cand, 1u);
      if (PCED_IN_BOUNDS(i < SMP_FEW, a.status))
        s.candidates(0)[i] = (uint32_t)~token, s.candidates(1)[i] = steps_of(x);
    });
    const int token_drawn = (int)~(uint32_t)rank_candidates(left + 1 - before);
    each_left([&](float x, int token) {
      if (token == token_drawn) write(x, token, row, t, total);
    });
  }
  __device__ __forceinline__ void write(float x, int token, int64_t row, float t, uint64_t total) const {
    a.token[row] = token;
    if (a.logprob) {
      // the largest weight is 2^ym of 2^SMP_UNIT steps; 32 bits serve a logarithm's own rounding
      const float all = (float)total;
      const float rest = (float)((int64_t)(total - (uint64_t)all)) / all;
      const float log_all = logf(all * (1.f / (float)((uint64_t)1 << SMP_UNIT))) + rest;
      a.logprob[row] = (mx == x ? 0.f : (x - mx) / t) - (log_all - s.ym * 0.693147181f);
    }
  }
  __device__ __forceinline__ uint64_t prefix(uint64_t v) const {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane() >= o) v += y;
    }
    return v;
  }
};

// ROOM: CTAs that an SM holds
template <typename T, int ROOM>
__global__ void __launch_bounds__(SMP_THREADS, ROOM) sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  __shared__ __align__(16) SampleShared s;
  cg::cluster_group cluster = cg::this_cluster();
  constexpr int W = Words<T>::N;
  const int ctas = cluster.num_blocks(), rank = cluster.block_rank(), tid = threadIdx.x;
  const int64_t row = blockIdx.x / ctas;
  const int start = rank * a.per, n = max(0, min(a.per, a.V - start));  // this CTA's tokens
  const T* src = (const T*)a.x + row * a.stride + start;
  const int phase = (int)((uintptr_t)src / sizeof(T) % W);
  const int groups = (phase + n + SMP_GROUP - 1) / SMP_GROUP;
  Row<T> R = {a, s, cluster, reinterpret_cast<const uint4*>(src - phase), reinterpret_cast<float2*>(smem_raw), start - phase,
              groups, ctas, 0};
  R.origin = 0.f, R.back = true;
  if (tid == 0) s.from = phase, s.to = phase + n;
  __syncthreads();
  static_assert(SMP_EXP2 == 2 * (SMP_THREADS / 16), "two entries a thread");
  const Exp2Entry entries[2] = {kExp2Table[tid / 16], kExp2Table[tid / 16 + SMP_THREADS / 16]};
  pdl_wait();
  // ---- what the row asks for
  const float t = a.temperature ? a.temperature[row] : 1.f, u = a.u[row];
  const float p = a.top_p ? a.top_p[row] : 1.f, least = a.min_p ? a.min_p[row] : 0.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  // ---- its largest logit
  float mx = -INFINITY;
  R.each_group([&](int g) { R.each_of(g, [&](int, float x, int) { mx = fmaxf(mx, x); }); });
  // (the reciprocals come while the last loads are on their way; held: the temperature that counts)
  const float held = fminf(fmaxf(t, 1e-37f), 1e30f), lh = 1.44269502f, ll = 1.92596303e-08f;
  R.w.ch = __fdiv_rn(lh, held);
  R.w.cl = __fdiv_rn(fmaf(-R.w.ch, held, lh) + ll, held);
  const float inverse = held * 0.693147181f;
  s.thread_max[tid] = mx + 0.f;
  {
    const int hi = __reduce_max_sync(0xffffffffu, ordered(mx + 0.f));
    if (R.lane() == 0) R.mine().mx[R.warp()] = hi;
    cluster.barrier_arrive();
    if (tid == SMP_THREADS - 1 && least > 0.f) s.below = (double)held * log((double)least);  // (takes a microsecond)
    __syncwarp();
    cluster.barrier_wait();
    const int r = R.lane() >> 2;  // a CTA's sixteen by four lanes
    int4 x = make_int4(INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN);
    if (r < ctas) x = *reinterpret_cast<const int4*>(R.theirs(r).mx + 4 * (R.lane() & 3));
    R.mx = mx = from_ordered(__reduce_max_sync(0xffffffffu, max(max(x.x, x.y), max(x.z, x.w))));
    ++R.turn;
  }
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
    R.each_group([&](int g) {
      R.each_of(g, [&](int, float x, int place) { at = x == mx ? min(at, (uint32_t)(R.first + place)) : at; });
    });
    at = __reduce_min_sync(0xffffffffu, at);
    if (R.lane() == 0) R.mine().sum[R.warp()] = at;
    cluster.sync();
    if (rank == 0 && R.warp() == 0) {
      for (int i = R.lane(); i < ctas * SMP_WARPS; i += 32) at = min(at, (uint32_t)R.theirs(i / SMP_WARPS).sum[i % SMP_WARPS]);
      at = __reduce_min_sync(0xffffffffu, at);
      if (R.lane() == 0) {
        a.token[row] = (int32_t)at;
        if (a.logprob) a.logprob[row] = 0.f;
      }
    }
    cluster.sync();
    return;
  }
  R.set_weights(inverse, entries);
  // ---- cuts
  if (k > 1 && k < a.V) R.keep_top(k);
  if (!R.gone && p < 1.f) R.keep_share((double)p);
  if (!R.gone && least > 0.f) R.keep_from(s.below);
  if (R.gone) return;
  // ---- the kept weights, and where u falls (off by 2^-52)
  const auto seek = [&](uint64_t total) { return min((uint64_t)((double)u * (double)total), total - 1); };
  if (R.solo) {
    const uint64_t total = R.template weigh_kept<false>().all;
    R.draw_solo(seek(total), row, held, total);
    return;
  }
  const typename Row<T>::Sums sums =
      R.grouped ? R.sum_groups() : R.cut.x == -INFINITY ? R.template weigh_all<false>(0.f) : R.weigh_groups();
  const uint64_t left = seek(sums.all);
  if (left >= sums.before && left < sums.before + sums.own) R.draw(left - sums.before, row, held, sums.all);
  cluster.sync();  // (a CTA's memory stays until the others have read it)
}

constexpr size_t SMP_SMEM = (SMP_LIST + SMP_WARPS * SMP_QUEUE) * sizeof(float2);

template <typename T, int ROOM>
static cudaError_t launch_sample(const SampleArgs& a, int32_t rows, int ctas, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  const auto kernel = sample_kernel<T, ROOM>;
  const cudaError_t e = pced_host::allow_smem(kernel, SMP_SMEM, done);
  if (e != cudaSuccess) return e;
  return pced_host::launch_cluster(kernel, dim3((unsigned)(rows * ctas)), ctas, SMP_THREADS, SMP_SMEM, stream, true, a);
}
// Whether the SMs hold so many clusters of `ctas` at once, ROOM CTAs on each (not whenever the SMs'
// number allows it: a cluster lies within a part of the device).
template <typename T, int ROOM>
static cudaError_t all_at_once(int32_t rows, int ctas, bool& yes) {
  static std::atomic<int> cache[64][ROW_CLUSTER + 1];  // (0: not asked yet)
  static std::atomic<bool> done[64];
  const auto kernel = sample_kernel<T, ROOM>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = pced_host::allow_smem(kernel, SMP_SMEM, done);
  if (e != cudaSuccess) return e;
  int held = cache[dev][ctas];
  if (!held) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas), cfg.blockDim = dim3(SMP_THREADS), cfg.dynamicSmemBytes = SMP_SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    cfg.attrs = attr, cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&held, kernel, &cfg);
    if (e != cudaSuccess) return e;
    cache[dev][ctas] = held;
  }
  yes = rows <= held;
  return cudaSuccess;
}
template <typename T>
cudaError_t launch_sample_t(SampleArgs a, int32_t rows, cudaStream_t stream) {
  // CTAs of a row: eight or four with an SM each (and twice the registers), else four or two with
  // half an SM, as long as all rows run at once and a part is more than a few tokens a thread.  fp32, us
  // at p = 0.9 with 1, 2, 4, 8 on an SM each | on half of one: a row of 128256 78, 49, 34, 30 | 79, 50, 37,
  // 33; 19 of 151936 88, 55, 38, 64 (not all at once) | 90, 57, 40, 48; 38 of them 88, 55, 73, 96 | 90, 57,
  // 56, 82; 152 of them 112, 131, 200, 358 | 113, 104, 154, 236.  Where the requests differ
  // the longest rules, and more CTAs gain: mixed cuts, 38 rows 117, 69, 73, - | 125, 74, 52, 52.  More rows
  // than that run two a row if that is long, so that those waiting fill the gaps: 272 of 151936 at
  // p = 0.9 178 with one, 191 with two, mixed cuts 196 and 152; of 65536 mixed 90 and 83, of 32768 60 and 69.
  const auto long_enough = [&](int ctas) { return a.V > 4 * SMP_THREADS * ctas; };
  bool yes = false;
  cudaError_t e = cudaSuccess;
  int ctas = 0;
  const int alone[] = {8, 4}, shared[] = {4, 2};
  static_assert(ROW_CLUSTER == 8, "the largest of these");
  bool room = false;
  for (int n : alone)
    if (!ctas && e == cudaSuccess && long_enough(n) && (e = all_at_once<T, 1>(rows, n, yes)) == cudaSuccess && yes)
      ctas = n, room = true;
  for (int n : shared)
    if (!ctas && e == cudaSuccess && long_enough(n) && (e = all_at_once<T, 2>(rows, n, yes)) == cudaSuccess && yes) ctas = n;
  if (e != cudaSuccess) return e;
  if (!ctas) ctas = a.V >= SMP_LONG ? 2 : 1;
  if (ctas == 1 && rows <= pced_host::num_sms()) room = true;
  while (a.V > SMP_MAX_PER * ctas) ctas *= 2;
  a.per = (a.V + ctas - 1) / ctas;
  return room ? launch_sample<T, 1>(a, rows, ctas, stream) : launch_sample<T, 2>(a, rows, ctas, stream);
}
// (a translation unit each: they compile for a minute)
extern template cudaError_t launch_sample_t<float>(SampleArgs, int32_t, cudaStream_t);
extern template cudaError_t launch_sample_t<__nv_bfloat16>(SampleArgs, int32_t, cudaStream_t);

}  // namespace pced
