// kv_append.cuh -- what the appends to paged caches of bf16 (kv_append.cu) and of
// 8-bit numbers (kv_append8.cu) share: their arguments and checks, the tokens of a
// block, a head's row of a token and its rotation.
//
// Rotation (rotate-half): y_f = x_f c_f - x_{f+D/2} s_f and
// y_{f+D/2} = x_{f+D/2} c_f + x_f s_f, every product and sum rounded to fp32 and
// not contracted, so that the keys, and the whole numbers counted from them, are
// the same whatever else a kernel does.
#pragma once
#include "paged.cuh"

namespace pced {

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

// eight channels x and their rotation partners y
__device__ __forceinline__ void rotate8(float (&x)[8], float (&y)[8], const float (&co)[8], const float (&si)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float u = __fsub_rn(__fmul_rn(x[e], co[e]), __fmul_rn(y[e], si[e]));
    y[e] = __fadd_rn(__fmul_rn(y[e], co[e]), __fmul_rn(x[e], si[e]));
    x[e] = u;
  }
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
    rotate8(x, y, co, si);
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
// Checks of a call and its arguments (a.T = 0: nothing to append)
inline pced_status append_args(const pced_paged_cache* cache, const void* q, int64_t q_stride, const void* k,
                               int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int32_t Hq,
                               const int32_t* tok_start, int32_t T, const float* rope, int32_t rope_rows,
                               const int32_t* positions, int32_t* status, const char* fn, AppendArgs& a) {
  using namespace pced_host;
  pced_status st = check_paged_cache(cache, fn);
  if (st == PCED_OK) st = check_paged_heads(cache, Hq, fn);
  if (st != PCED_OK) return st;
  const pced_paged_cache& c = *cache;
  if (T < 0) return fail(PCED_ERR_INVALID_ARG, "%s: T < 0", fn);
  if (!tok_start && T != c.S) return fail(PCED_ERR_INVALID_ARG, "%s: without tok_start T must be S", fn);
  a.T = T;
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
  a.c = c;
  a.q = (const __nv_bfloat16*)q, a.k = (const __nv_bfloat16*)k, a.v = (const __nv_bfloat16*)v;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.q_out = (__nv_bfloat16*)q_out;
  a.Hq = Hq, a.G = q ? Hq / c.Hkv : 0;
  a.tok_start = tok_start;
  a.rope = rope, a.rope_rows = rope_rows, a.positions = positions;
  a.status = status;
  return PCED_OK;
}

// Items of a call with tok_start (blocks touched: at most two more than whole ones for
// every sequence with tokens) and the kv-heads that a CTA takes of one, so that its
// `units` have a row each where items have few; 0 items: too many for a grid of up to `cluster`
// CTAs each
inline int64_t append_items(AppendArgs& a, int units, int cluster) {
  const pced_paged_cache& c = a.c;
  const int64_t items = (int64_t)a.T / c.block_rows + 2 * (int64_t)(a.T < c.S ? a.T : c.S);
  if (items * c.Hkv * cluster >= (INT64_C(1) << 31)) return 0;
  const int64_t rows = a.T / items > 0 ? a.T / items : 1;  // of an item, about
  a.heads = 1;
  while (2 * a.heads * rows <= units && c.Hkv % (2 * a.heads) == 0) a.heads *= 2;
  return items;
}

}  // namespace pced
