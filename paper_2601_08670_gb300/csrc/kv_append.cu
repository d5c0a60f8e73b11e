// kv_append.cu -- new keys and values into a paged cache, rotated on the way,
// and the key summaries of its blocks (pced_kv_append, pced_block_summaries).
//
// Rotation (rotate-half): y_f = x_f c_f - x_{f+D/2} s_f and
// y_{f+D/2} = x_{f+D/2} c_f + x_f s_f, every product and sum rounded to fp32 and
// not contracted, so that the keys, and the whole numbers counted from them, are
// the same whatever else a kernel does.
//
// What bounds them (one GB300, GPU time in a graph): HBM where there are many
// tokens (sixteen documents, 18,366 tokens of 32 + 16 heads of 128: 466 MB in 76 us,
// 6.1 TB/s, 90 % of the copy rate), latency where there are few (nine tokens:
// 2.6 us, a launch and three round trips).
#include <cooperative_groups.h>

#include "paged.cuh"

namespace pced {

namespace cg = cooperative_groups;

struct AppendArgs {
  pced_paged_cache c;
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  __nv_bfloat16* q_out;
  int32_t Hq, G;             // G: query heads of a group (0: no queries)
  const int32_t* tok_start;  // null: one token per sequence
  int32_t T;
  const float* rope;
  int32_t rope_rows;
  const int32_t* positions;
  int32_t heads;  // kv-heads of a CTA (any number of tokens): a power of two that divides Hkv, at most its units
  int* status;
};

constexpr int APP_THREADS = 128;

// tokens [t0, t0 + m) of one sequence, which go to rows r0 ... of one block
struct AppendItem {
  int s, t0, r0, m;
};

// New rows of sequence s: {first token, count, live rows}; count 0 where the
// counts do not fit (flagged).  falls: its starts fall.
__device__ __forceinline__ int3 new_rows(const AppendArgs& a, int s, bool& falls) {
  const int n = a.c.seq_len[s], t0 = a.tok_start[s], t1 = a.tok_start[s + 1];
  falls = t1 < t0;
  if (n < 0 || n > a.c.max_blocks * a.c.block_rows || t0 < 0 || t1 < t0 || t1 > a.T || t1 - t0 > n) {
    dev_flag(a.status, PCED_DEV_BAD_LENGTH);
    return make_int3(0, 0, 0);
  }
  return make_int3(t0, t1 - t0, n);
}
__device__ __forceinline__ int blocks_touched(int3 r, int P) {
  return r.y > 0 ? (r.z - 1) / P - (r.z - r.y) / P + 1 : 0;
}

// Item `want` of the call: its sequence by the prefix of blocks touched.  All
// threads; s = -1 past the last.  Up to where the starts first fall they share
// the tokens out, so that the launch has an item for every block touched; from
// there on tokens could be named twice, and no sequence gets any.
__device__ __forceinline__ AppendItem find_item(const AppendArgs& a, int want) {
  constexpr int PER = PAGED_MAX_S / APP_THREADS;  // sequences of a thread
  __shared__ int wsum[APP_THREADS / 32], wfall[APP_THREADS / 32];
  __shared__ AppendItem it;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, P = a.c.block_rows;
  const int per = (a.c.S + APP_THREADS - 1) / APP_THREADS, s0 = tid * per;
  int3 r[PER];
  int nb[PER], own = 0, fall = INT32_MAX;  // the first sequence at which the starts fall
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool in = i < per && s0 + i < a.c.S;
    bool falls = false;
    r[i] = in ? new_rows(a, s0 + i, falls) : make_int3(0, 0, 0);
    if (falls) fall = min(fall, s0 + i);
    nb[i] = blocks_touched(r[i], P);
    own += nb[i];
  }
  int incl = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) wsum[warp] = incl;
  if (tid == 0) it.s = -1;
  if (__syncthreads_or(fall != INT32_MAX)) {
    fall = __reduce_min_sync(0xffffffffu, fall);
    if (lane == 0) wfall[warp] = fall;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < APP_THREADS / 32; ++w) fall = min(fall, wfall[w]);
  }
  int at = incl - own;
#pragma unroll
  for (int w = 0; w < APP_THREADS / 32; ++w) at += w < warp ? wsum[w] : 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (want >= at && want < at + nb[i] && s0 + i < fall) {
      const int first = r[i].z - r[i].y, j = first / P + (want - at);
      it.s = s0 + i;
      it.r0 = max(first, j * P);
      it.m = min(r[i].z, (j + 1) * P) - it.r0;
      it.t0 = r[i].x + (it.r0 - first);
    }
    at += nb[i];
  }
  __syncthreads();
  return it;
}

__device__ __forceinline__ void unpack8(uint4 w, float (&x)[8]) {
  x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
  x[4] = bf16_lo(w.z), x[5] = bf16_hi(w.z), x[6] = bf16_lo(w.w), x[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// One head's row of a token: eight channels and their eight rotation partners.
struct HeadRow {
  uint4 a, b;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int half) {
    a = *reinterpret_cast<const uint4*>(p);
    b = *reinterpret_cast<const uint4*>(p + half);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p, int half) const {
    *reinterpret_cast<uint4*>(p) = a;
    *reinterpret_cast<uint4*>(p + half) = b;
  }
  __device__ __forceinline__ void rotate(const float (&co)[8], const float (&si)[8]) {
    float x[8], y[8];
    unpack8(a, x);
    unpack8(b, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = __fsub_rn(__fmul_rn(x[e], co[e]), __fmul_rn(y[e], si[e]));
      y[e] = __fadd_rn(__fmul_rn(y[e], co[e]), __fmul_rn(x[e], si[e]));
      x[e] = u;
    }
    a = pack8(x);
    b = pack8(y);
  }
};
// cosines and sines of eight angles of position p; false (flagged) outside the table
__device__ __forceinline__ bool load_angles(const AppendArgs& a, int D, int p, int f, float (&co)[8], float (&si)[8]) {
  if (p < 0 || p >= a.rope_rows) {
    dev_flag(a.status, PCED_DEV_BAD_INDEX);
    return false;
  }
  const float4* tc = reinterpret_cast<const float4*>(a.rope + (int64_t)p * D + f);
  const float4* ts = reinterpret_cast<const float4*>(a.rope + (int64_t)p * D + D / 2 + f);
  *reinterpret_cast<float4*>(co) = tc[0], *reinterpret_cast<float4*>(co + 4) = tc[1];
  *reinterpret_cast<float4*>(si) = ts[0], *reinterpret_cast<float4*>(si + 4) = ts[1];
  return true;
}
// a block's summary taken up to date with the bounds of eight channels from f on
// (half: 0) or their partners (half: D / 2)
__device__ __forceinline__ void update_summary(int8_t* summary, int D, int f, const uint32_t (&mx)[4],
                                               const uint32_t (&mn)[4], float inv, bool fresh) {
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    uint2* at = reinterpret_cast<uint2*>(summary + which * D + f);
    const uint32_t(&k)[4] = which ? mn : mx;
    uint2 w = make_uint2(steps4(k[0], k[1], !which, inv), steps4(k[2], k[3], !which, inv));
    if (!fresh) {
      const uint2 old = *at;
      w = which ? make_uint2(__vmins4(w.x, old.x), __vmins4(w.y, old.y))
                : make_uint2(__vmaxs4(w.x, old.x), __vmaxs4(w.y, old.y));
    }
    *at = w;
  }
}

// One token per sequence: a CTA per (sequence, kv-head), D/16 lanes for each row
// of a head (key, value, the group's queries), so every row's load is asked for at
// once, beside the length.  Nine tokens 2.6 us; with the kernel for any number of
// tokens, which looks for its tokens first, 3.1 us.
constexpr int APP_ONE_THREADS = 8 * (PAGED_MAX_G + 2);  // (D = 128)

template <int D>
__global__ void __launch_bounds__(APP_ONE_THREADS) kv_append_one_kernel(AppendArgs a) {
  constexpr int LANES = D / 16;
  const int tid = threadIdx.x, s = blockIdx.y, h = blockIdx.x, G = a.G, P = a.c.block_rows;
  const int role = tid / LANES, f = 8 * (tid % LANES);  // role 0: key, 1: value, then queries
  if (role >= G + 2) return;
  pdl_wait();
  HeadRow r;
  __nv_bfloat16* dst = nullptr;
  if (role >= 2) {
    const int head = h * G + role - 2;
    r.load(a.q + s * a.q_stride + (int64_t)head * D + f, D / 2);
    dst = a.q_out + ((int64_t)s * a.Hq + head) * D + f;
  } else {
    r.load((role ? a.v + s * a.v_stride : a.k + s * a.k_stride) + h * D + f, D / 2);
  }
  bool fits;
  const int n = paged_len(a.c, s, a.status, fits);
  if (n == 0) {  // an idle sequence: no query either
    r.a = r.b = make_uint4(0, 0, 0, 0);
    if (role >= 2) r.store(dst, D / 2);
    return;
  }
  if (a.rope && role != 1) {
    float co[8], si[8];
    if (load_angles(a, D, a.positions ? a.positions[s] : n - 1, f, co, si)) r.rotate(co, si);
  }
  if (role >= 2) {
    r.store(dst, D / 2);
    return;
  }
  if (!fits) return;  // (the table's last row is another token's)
  const int blk = paged_block(a.c, s, (n - 1) / P, a.status), at = (n - 1) % P;
  if (blk < 0) return;
  const int64_t page = (int64_t)blk * a.c.Hkv + h;
  if (!PCED_IN_BOUNDS(in_pool(a.c, page, at), a.status)) return;
  r.store((__nv_bfloat16*)(role ? a.c.v : a.c.k) + (page * P + at) * D + f, D / 2);
  if (role == 0 && a.c.summary) {
    const float inv = __fdiv_rn(1.f, a.c.key_step[h]);
    const uint32_t lo[4] = {r.a.x, r.a.y, r.a.z, r.a.w}, hi[4] = {r.b.x, r.b.y, r.b.z, r.b.w};
    update_summary(a.c.summary + page * 2 * D, D, f, lo, lo, inv, at == 0);
    update_summary(a.c.summary + page * 2 * D, D, f + D / 2, hi, hi, inv, at == 0);
  }
}

// Any number of tokens: a CTA takes one item and a kv-head, or `heads` of them.  D/16
// lanes (a unit) share a row of one kv-head and its group, each with the same channels
// of all these heads, so a position's angles are read once for them, and a thread
// holds the bounds of its channels' keys in registers.  (A page and kv-head has one
// CTA, or one cluster, so its summary has one writer.)  APP_SEVERAL: more than one
// kv-head, where items have so few rows that a CTA's units would idle (272 sequences
// of two tokens: 17.5 us with one, 6.7 with eight; but 33 of 32 tokens, with two, 14.3
// against 9.0).  APP_SHARED: where CTAs are few and their rows many, a cluster shares
// the item's rows, and its first CTA brings the bounds together (eight sequences of 278
// tokens in 256-row pages: 44.3 us, 21.0 with clusters of four; but where the CTAs of
// clusters no longer fit the SMs at once, four documents of 64-row pages, 24.1 us
// became 29.7).
// Sixteen documents: 134 us with a unit per head's row (angles read again for every
// head), 89 us this way at 2 CTAs of 256 threads an SM, 81 us at 3, 78 us with an
// item's heads side by side in the grid, 76 us with 6 CTAs of 128 threads.
constexpr int APP_CTAS = 6;     // CTAs that an SM holds
constexpr int APP_CLUSTER = 8;  // most CTAs of an item and kv-head
constexpr int APP_HEADS = 3;  // heads whose loads a thread has in flight (six, at 2/3 of the CTAs: 1 % less time)

enum AppendMode { APP_ONE_HEAD, APP_SEVERAL, APP_SHARED };

template <int D, AppendMode MODE>
__global__ void __launch_bounds__(APP_THREADS, APP_CTAS) kv_append_kernel(AppendArgs a) {
  constexpr int LANES = D / 16, UNITS = APP_THREADS / LANES;
  constexpr int SIDE = 32 / LANES;  // units of a warp
  // (the heads of an item side by side: their parts of a token's row are neighbours in memory)
  const int tid = threadIdx.x, unit = tid / LANES, G = a.G, P = a.c.block_rows;
  const int heads = MODE == APP_SEVERAL ? a.heads : 1;
  uint32_t group = blockIdx.x;
  int ctas = 1, rank = 0;
  if constexpr (MODE == APP_SHARED) {
    ctas = cg::this_cluster().num_blocks(), rank = cg::this_cluster().block_rank();
    group /= ctas;
  }
  const int per_item = a.c.Hkv / heads;
  const int h0 = group % per_item * heads, h = h0 + (unit & (heads - 1));
  __shared__ uint32_t bounds[UNITS][2][D / 2];  // largest, smallest keys
  pdl_wait();
  const AppendItem it = find_item(a, group / per_item);
  if (it.s < 0) return;
  const int blk = paged_block(a.c, it.s, it.r0 / P, a.status);
  const int64_t page = (int64_t)blk * a.c.Hkv + h;
  const int f = 8 * (tid % LANES);
  KeyBounds2 kb[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) kb[e].reset();
  int i0 = 0, i_end = it.m;  // this CTA's rows
  if constexpr (MODE == APP_SHARED) {
    const int part = (it.m + ctas - 1) / ctas;
    i0 = rank * part, i_end = min(it.m, i0 + part);
  }
  for (int i = i0 + unit / heads; i < i_end; i += UNITS / heads) {
    const int64_t t = it.t0 + i;
    const int64_t row = (page * P + it.r0 % P + i) * D + f;
    float co[8], si[8];
    const bool rotated = a.rope && load_angles(a, D, a.positions ? a.positions[t] : it.r0 + i, f, co, si);
    for (int r0 = 0; r0 < G + 2; r0 += APP_HEADS) {  // role 0: key, 1: value, then queries
      HeadRow x[APP_HEADS];
#pragma unroll
      for (int u = 0; u < APP_HEADS; ++u) {
        const int role = r0 + u;
        if (role >= G + 2) break;
        const __nv_bfloat16* src = role == 0   ? a.k + t * a.k_stride + h * D
                                   : role == 1 ? a.v + t * a.v_stride + h * D
                                               : a.q + t * a.q_stride + (int64_t)(h * G + role - 2) * D;
        x[u].load(src + f, D / 2);
      }
#pragma unroll
      for (int u = 0; u < APP_HEADS; ++u) {
        const int role = r0 + u;
        if (role >= G + 2) break;
        if (rotated && role != 1) x[u].rotate(co, si);
        if (!PCED_IN_BOUNDS(t < a.T && (blk < 0 || in_pool(a.c, page, it.r0 % P + i)), a.status)) continue;
        if (role >= 2) {
          x[u].store(a.q_out + (t * a.Hq + h * G + role - 2) * D + f, D / 2);
        } else if (blk >= 0) {
          x[u].store((__nv_bfloat16*)(role ? a.c.v : a.c.k) + row, D / 2);
        }
        if (role == 0) {
          const uint32_t w[8] = {x[u].a.x, x[u].a.y, x[u].a.z, x[u].a.w, x[u].b.x, x[u].b.y, x[u].b.z, x[u].b.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) kb[e].take(w[e]);
        }
      }
    }
  }
  if (!a.c.summary || blk < 0) return;
  // units of the same head meet: in the warp, then in shared memory
#pragma unroll
  for (int o = LANES; o < 32; o <<= 1)
    if (o >= LANES * heads)
#pragma unroll
    for (int e = 0; e < 8; ++e) kb[e].merge_xor(o);
  if (unit % SIDE < heads) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = f / 2 + (e < 4 ? e : D / 4 + e - 4);
      bounds[unit][0][at] = kb[e].top();
      bounds[unit][1][at] = kb[e].bottom();
    }
  }
  if constexpr (MODE == APP_SHARED) cg::this_cluster().sync();
  else __syncthreads();
  for (int i = tid; rank == 0 && i < heads * (D / 8); i += APP_THREADS) {  // eight channels of a head
    const int hh = i / (D / 8), d = 8 * (i % (D / 8));
    uint32_t mx[4], mn[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      KeyBounds2 b;
      b.reset();
      for (int u = hh; u < UNITS; u += max(heads, SIDE)) b.merge(bounds[u][0][d / 2 + e], bounds[u][1][d / 2 + e]);
      if constexpr (MODE == APP_SHARED) {
        for (int r = 1; r < ctas; ++r) {
          const auto& of = *cg::this_cluster().map_shared_rank(&bounds, r);
          for (int u = 0; u < UNITS; u += SIDE) b.merge(of[u][0][d / 2 + e], of[u][1][d / 2 + e]);
        }
      }
      mx[e] = b.top(), mn[e] = b.bottom();
    }
    update_summary(a.c.summary + ((int64_t)blk * a.c.Hkv + h0 + hh) * 2 * D, D, d, mx, mn,
                   __fdiv_rn(1.f, a.c.key_step[h0 + hh]), it.r0 % P == 0);
  }
  if constexpr (MODE == APP_SHARED) cg::this_cluster().sync();  // (the others' bounds stay until they are read)
}

// ------------------------------------------------------------------ summaries
// A warp takes up to SUM_ROWS rows of one block and kv-head at a time, D/8 lanes a
// row; the warps of a block (a power of two of them) meet in shared memory.  HBM
// bounds it: 272 ragged caches, 664 MB in 97 us (6.8 TB/s); nine of 2080 rows 8.3 us
// for 39 MB, of which a launch and the chain length, table, rows, sums take 3.
constexpr int SUM_WARPS = 8;
constexpr int SUM_ROWS = 32;
constexpr int SUM_BATCH = 8;  // loads of a lane in flight

template <int D>
__global__ void __launch_bounds__(32 * SUM_WARPS) block_summaries_kernel(pced_paged_cache c, int split, int* status) {
  constexpr int LANES = D / 8, ROWS = 32 / LANES;  // lanes of a row, rows of a load
  __shared__ uint32_t bounds[SUM_WARPS][2][D / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.y, P = c.block_rows;
  const int unit = blockIdx.x * (SUM_WARPS / split) + warp / split;  // block and kv-head
  const int j = unit / c.Hkv, h = unit % c.Hkv, part = warp % split;
  pdl_wait();
  const int live = j < c.max_blocks ? min(P, paged_len(c, s, status) - j * P) : 0;
  const int blk = live > 0 ? paged_block(c, s, j, status) : -1;
  const int64_t page = (int64_t)blk * c.Hkv + h;
  KeyBounds2 kb[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) kb[e].reset();
  const int f = 8 * (lane % LANES);
  if (blk >= 0) {
    const __nv_bfloat16* k = (const __nv_bfloat16*)c.k + page * P * D + f;
    const int step = split * ROWS;
    for (int r = part * ROWS + lane / LANES; r < live; r += SUM_BATCH * step) {
      uint4 w[SUM_BATCH];
#pragma unroll
      for (int u = 0; u < SUM_BATCH; ++u)
        w[u] = *reinterpret_cast<const uint4*>(k + (int64_t)min(r + u * step, live - 1) * D);  // (a row twice: no harm)
#pragma unroll
      for (int u = 0; u < SUM_BATCH; ++u) kb[0].take(w[u].x), kb[1].take(w[u].y), kb[2].take(w[u].z), kb[3].take(w[u].w);
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1) kb[e].merge_xor(o);
    if (split > 1 && lane < LANES) {
      bounds[warp][0][f / 2 + e] = kb[e].top();
      bounds[warp][1][f / 2 + e] = kb[e].bottom();
    }
  }
  if (split > 1) __syncthreads();
  if (part > 0 || lane >= LANES || blk < 0) return;
  uint32_t mx[4], mn[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    for (int w = 1; w < split; ++w) kb[e].merge(bounds[warp + w][0][f / 2 + e], bounds[warp + w][1][f / 2 + e]);
    mx[e] = kb[e].top(), mn[e] = kb[e].bottom();
  }
  if (PCED_IN_BOUNDS(in_pool(c, page, live - 1), status))
    update_summary(c.summary + page * 2 * D, D, f, mx, mn, __fdiv_rn(1.f, c.key_step[h]), true);
}

}  // namespace pced

using namespace pced;
using namespace pced_host;

namespace pced_host {

pced_status check_paged_cache(const pced_paged_cache* c, const char* fn) {
  if (!c || !c->block_table || !c->seq_len) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (c->S < 1 || c->Hkv < 1 || c->num_blocks < 1 || c->max_blocks < 1 || c->block_rows < 1 || c->D < 1)
    return fail(PCED_ERR_INVALID_ARG, "%s: sizes below 1", fn);
  if (c->block_rows % 16) return fail(PCED_ERR_INVALID_ARG, "%s: block_rows %d is no multiple of 16", fn, c->block_rows);
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->summary, 16) || !aligned(c->key_step, 4) ||
      !aligned(c->block_table, 4) || !aligned(c->seq_len, 4))
    return fail(PCED_ERR_INVALID_ARG, "%s: misaligned cache pointer", fn);
  if (c->D != 64 && c->D != 128) return fail(PCED_ERR_UNSUPPORTED, "%s: head dim %d", fn, c->D);
  if (c->S > PAGED_MAX_S) return fail(PCED_ERR_UNSUPPORTED, "%s: %d sequences, at most %d", fn, c->S, PAGED_MAX_S);
  if ((int64_t)c->max_blocks * c->block_rows + c->block_rows > INT32_MAX)
    return fail(PCED_ERR_UNSUPPORTED, "%s: a sequence's table holds 2^31 rows or more", fn);
  if ((int64_t)c->num_blocks * c->Hkv >= (INT64_C(1) << 31) ||
      (int64_t)c->num_blocks * c->Hkv * c->block_rows >= (INT64_C(1) << 31))
    return fail(PCED_ERR_UNSUPPORTED, "%s: more than 2^31 rows in the pool", fn);
  return PCED_OK;
}

pced_status check_paged_heads(const pced_paged_cache* c, int32_t Hq, const char* fn) {
  if (Hq < 1 || Hq % c->Hkv) return fail(PCED_ERR_INVALID_ARG, "%s: Hq is no multiple of Hkv", fn);
  if (Hq / c->Hkv > PAGED_MAX_G)
    return fail(PCED_ERR_UNSUPPORTED, "%s: more than %d query heads per kv-head", fn, PAGED_MAX_G);
  return PCED_OK;
}

}  // namespace pced_host

extern "C" pced_status pced_kv_append(const pced_paged_cache* cache, const void* q, int64_t q_stride, const void* k,
                                      int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int32_t Hq,
                                      const int32_t* tok_start, int32_t T, const float* rope, int32_t rope_rows,
                                      const int32_t* positions, int32_t* status, void* stream) {
  const char* fn = "pced_kv_append";
  pced_status st = check_paged_cache(cache, fn);
  if (st == PCED_OK) st = check_paged_heads(cache, Hq, fn);
  if (st != PCED_OK) return st;
  const pced_paged_cache& c = *cache;
  if (T < 0) return fail(PCED_ERR_INVALID_ARG, "%s: T < 0", fn);
  if (!tok_start && T != c.S) return fail(PCED_ERR_INVALID_ARG, "%s: without tok_start T must be S", fn);
  if (T == 0) return PCED_OK;
  if (!c.k || !c.v || !k || !v || !q != !q_out || (c.summary && !c.key_step))
    return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (!q && Hq != c.Hkv) return fail(PCED_ERR_INVALID_ARG, "%s: Hq without queries", fn);
  if (rope && rope_rows < 1) return fail(PCED_ERR_INVALID_ARG, "%s: empty rotation table", fn);
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(rope, 16) ||
      !aligned(tok_start, 4) || !aligned(positions, 4) || !aligned(status, 4))
    return fail(PCED_ERR_INVALID_ARG, "%s: misaligned pointer", fn);
  const int64_t need_q = (int64_t)Hq * c.D, need_kv = (int64_t)c.Hkv * c.D;
  if ((q && (q_stride % 8 || q_stride < need_q)) || k_stride % 8 || k_stride < need_kv || v_stride % 8 ||
      v_stride < need_kv)
    return fail(PCED_ERR_INVALID_ARG, "%s: token stride no multiple of 8 or below a token's heads", fn);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  AppendArgs a;
  a.c = c;
  a.q = (const __nv_bfloat16*)q, a.k = (const __nv_bfloat16*)k, a.v = (const __nv_bfloat16*)v;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.q_out = (__nv_bfloat16*)q_out;
  a.Hq = Hq, a.G = q ? Hq / c.Hkv : 0;
  a.tok_start = tok_start, a.T = T;
  a.rope = rope, a.rope_rows = rope_rows, a.positions = positions;
  a.status = status;
  cudaError_t e;
  if (!tok_start) {
    const int threads = (a.G + 2) * (c.D / 16);
    e = launch_pdl(c.D == 128 ? kv_append_one_kernel<128> : kv_append_one_kernel<64>, dim3(c.Hkv, c.S), threads, 0,
                   (cudaStream_t)stream, a);
  } else {
    // blocks touched: at most two more than whole ones for every sequence with tokens
    const int64_t items = (int64_t)T / c.block_rows + 2 * (int64_t)(T < c.S ? T : c.S);
    if (items * c.Hkv * APP_CLUSTER >= (INT64_C(1) << 31)) return fail(PCED_ERR_UNSUPPORTED, "%s: too many tokens", fn);
    const int units = APP_THREADS / (c.D / 16);
    const int64_t rows = T / items > 0 ? T / items : 1;  // of an item, about
    a.heads = 1;
    while (2 * a.heads * rows <= units && c.Hkv % (2 * a.heads) == 0) a.heads *= 2;
    const int64_t groups = items * (c.Hkv / a.heads);
    // rows of a full item, about; CTAs of a cluster for them, while that leaves each its units' worth and all
    // fit the SMs at once
    const int64_t full = min((int64_t)c.block_rows, (int64_t)T / (T < c.S ? T : c.S));
    int ctas = 1;
    while (a.heads == 1 && ctas < APP_CLUSTER && 2 * ctas * groups <= APP_CTAS * (int64_t)num_sms() &&
           full >= 2 * ctas * units)
      ctas *= 2;
    const dim3 grid((unsigned)(groups * ctas));
    if (ctas > 1)
      e = launch_cluster(c.D == 128 ? kv_append_kernel<128, APP_SHARED> : kv_append_kernel<64, APP_SHARED>, grid, ctas,
                         APP_THREADS, 0, (cudaStream_t)stream, true, a);
    else if (a.heads > 1)
      e = launch_pdl(c.D == 128 ? kv_append_kernel<128, APP_SEVERAL> : kv_append_kernel<64, APP_SEVERAL>, grid,
                     APP_THREADS, 0, (cudaStream_t)stream, a);
    else
      e = launch_pdl(c.D == 128 ? kv_append_kernel<128, APP_ONE_HEAD> : kv_append_kernel<64, APP_ONE_HEAD>, grid,
                     APP_THREADS, 0, (cudaStream_t)stream, a);
  }
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "kv_append launch");
}

extern "C" pced_status pced_block_summaries(const pced_paged_cache* cache, int32_t* status, void* stream) {
  const char* fn = "pced_block_summaries";
  const pced_status st = check_paged_cache(cache, fn);
  if (st != PCED_OK) return st;
  const pced_paged_cache& c = *cache;
  if (!c.k || !c.summary || !c.key_step) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (!aligned(status, 4)) return fail(PCED_ERR_INVALID_ARG, "%s: misaligned pointer", fn);
  int split = 1;  // warps of a block's rows
  while (split < SUM_WARPS && split * SUM_ROWS < c.block_rows) split *= 2;
  const int64_t gx = ((int64_t)c.max_blocks * c.Hkv + SUM_WARPS / split - 1) / (SUM_WARPS / split);
  if ((int64_t)c.max_blocks * c.Hkv >= (INT64_C(1) << 31) - SUM_WARPS)
    return fail(PCED_ERR_UNSUPPORTED, "%s: max_blocks * Hkv >= 2^31", fn);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  const cudaError_t e = launch_pdl(c.D == 128 ? block_summaries_kernel<128> : block_summaries_kernel<64>,
                                   dim3((unsigned)gx, c.S), 32 * SUM_WARPS, 0, (cudaStream_t)stream, c, split, status);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "block_summaries launch");
}
