// kv_append.cu -- new keys and values into a paged cache, rotated on the way,
// and the key summaries of its blocks (pced_kv_append, pced_block_summaries).
//
// Rotation (rotate-half): y_f = x_f c_f - x_{f+D/2} s_f and
// y_{f+D/2} = x_{f+D/2} c_f + x_f s_f, every product and sum rounded to fp32 and
// not contracted, so that the keys, and the whole numbers counted from them, are
// the same whatever else a kernel does.
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
  int* status;
};

constexpr int APP_THREADS = 256;

// tokens [t0, t0 + m) of one sequence, which go to rows r0 ... of one block
struct AppendItem {
  int s, t0, r0, m;
};

// New rows of sequence s: {first token, count, live rows}; count 0 where the
// counts do not fit (flagged).
__device__ __forceinline__ int3 new_rows(const AppendArgs& a, int s) {
  const int n = paged_len(a.c, s, a.status);
  const int t0 = a.tok_start[s], t1 = a.tok_start[s + 1];
  if (t0 < 0 || t1 < t0 || t1 > a.T || t1 - t0 > n) {
    dev_flag(a.status, PCED_DEV_BAD_LENGTH);
    return make_int3(0, 0, n);
  }
  return make_int3(t0, t1 - t0, n);
}
__device__ __forceinline__ int blocks_touched(int3 r, int P) {
  return r.y > 0 ? (r.z - 1) / P - (r.z - r.y) / P + 1 : 0;
}

// Item `want` of the call: its sequence by the prefix of blocks touched.  All
// threads; s = -1 past the last.
__device__ __forceinline__ AppendItem find_item(const AppendArgs& a, int want) {
  __shared__ int wsum[APP_THREADS / 32];
  __shared__ AppendItem it;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, P = a.c.block_rows;
  const int per = (a.c.S + APP_THREADS - 1) / APP_THREADS;
  const int s0 = min(a.c.S, tid * per), s1 = min(a.c.S, s0 + per);
  int own = 0;
  for (int s = s0; s < s1; ++s) own += blocks_touched(new_rows(a, s), P);
  int incl = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) wsum[warp] = incl;
  if (tid == 0) it.s = -1;
  __syncthreads();
  int at = incl - own;
  for (int w = 0; w < warp; ++w) at += wsum[w];
  if (want >= at && want < at + own) {
    for (int s = s0; s < s1; ++s) {
      const int3 r = new_rows(a, s);
      const int nb = blocks_touched(r, P);
      if (want < at + nb) {
        const int first = r.z - r.y, j = first / P + (want - at);
        it.s = s;
        it.r0 = max(first, j * P);
        it.m = min(r.z, (j + 1) * P) - it.r0;
        it.t0 = r.x + (it.r0 - first);
        break;
      }
      at += nb;
    }
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

// A CTA takes one item and one kv-head: the rows of K and V and the group's
// queries.  D/16 lanes share a row of one head (a unit), each with eight channels
// and their eight rotation partners, so a thread sees the same channels of every
// key row it takes and holds their bounds in registers.
template <int D, bool ONE>
__global__ void __launch_bounds__(APP_THREADS) kv_append_kernel(AppendArgs a) {
  constexpr int LANES = D / 16;
  const int tid = threadIdx.x, h = blockIdx.y, G = a.G, P = a.c.block_rows;
  pdl_wait();
  AppendItem it;
  if (ONE) {
    it.s = it.t0 = blockIdx.x;
    const int n = paged_len(a.c, it.s, a.status);
    it.r0 = n - 1;
    it.m = n > 0;
    if (n == 0) {  // an idle sequence: no query either
      for (int i = tid; i < G * D / 8; i += blockDim.x)
        reinterpret_cast<uint4*>(a.q_out + ((int64_t)it.t0 * a.Hq + h * G) * D)[i] = make_uint4(0, 0, 0, 0);
      return;
    }
  } else {
    it = find_item(a, blockIdx.x);
    if (it.s < 0) return;
  }
  const int blk = paged_block(a.c, it.s, it.r0 / P, a.status);
  const int64_t row0 = ((int64_t)blk * a.c.Hkv + h) * P + it.r0 % P;
  const bool summarise = a.c.summary != nullptr;
  const float inv = summarise ? __fdiv_rn(1.f, a.c.key_step[h]) : 0.f;
  const int l = tid % LANES, f = 8 * l;
  KeyBounds lo[8], hi[8];
  const int units = it.m * (G + 2);
  for (int u = tid / LANES; u < units; u += blockDim.x / LANES) {
    const int i = u / (G + 2), role = u - i * (G + 2);  // role 0: key, 1: value, then queries
    const int64_t t = it.t0 + i;
    const __nv_bfloat16* src;
    __nv_bfloat16* dst;
    if (role < 2) {
      src = (role ? a.v + t * a.v_stride : a.k + t * a.k_stride) + h * D;
      dst = (__nv_bfloat16*)(role ? a.c.v : a.c.k) + (row0 + i) * D;
    } else {
      const int head = h * G + role - 2;
      src = a.q + t * a.q_stride + (int64_t)head * D;
      dst = a.q_out + (t * a.Hq + head) * D;
    }
    uint4 w0 = *reinterpret_cast<const uint4*>(src + f), w1 = *reinterpret_cast<const uint4*>(src + f + D / 2);
    if (a.rope && role != 1) {
      const int p = a.positions ? a.positions[t] : it.r0 + i;
      if (p >= 0 && p < a.rope_rows) {
        float x[8], y[8], co[8], si[8];
        unpack8(w0, x);
        unpack8(w1, y);
        const float4* tc = reinterpret_cast<const float4*>(a.rope + (int64_t)p * D + f);
        const float4* ts = reinterpret_cast<const float4*>(a.rope + (int64_t)p * D + D / 2 + f);
        *reinterpret_cast<float4*>(co) = tc[0], *reinterpret_cast<float4*>(co + 4) = tc[1];
        *reinterpret_cast<float4*>(si) = ts[0], *reinterpret_cast<float4*>(si + 4) = ts[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u0 = __fsub_rn(__fmul_rn(x[e], co[e]), __fmul_rn(y[e], si[e]));
          y[e] = __fadd_rn(__fmul_rn(y[e], co[e]), __fmul_rn(x[e], si[e]));
          x[e] = u0;
        }
        w0 = pack8(x);
        w1 = pack8(y);
      } else if (l == 0) {
        dev_flag(a.status, PCED_DEV_BAD_INDEX);
      }
    }
    if (role >= 2 || blk >= 0) {
      *reinterpret_cast<uint4*>(dst + f) = w0;
      *reinterpret_cast<uint4*>(dst + f + D / 2) = w1;
    }
    if (role == 0 && summarise) {
      float x[8], y[8];
      unpack8(w0, x);
      unpack8(w1, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) lo[e].take(x[e], inv), hi[e].take(y[e], inv);
    }
  }
  if (!summarise) return;
  // the bounds of all units, channel by channel
  __shared__ float bounds[2][APP_THREADS / 32][D];
  const int lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1) {
      lo[e].merge(__shfl_xor_sync(0xffffffffu, lo[e].mx, o), __shfl_xor_sync(0xffffffffu, lo[e].mn, o));
      hi[e].merge(__shfl_xor_sync(0xffffffffu, hi[e].mx, o), __shfl_xor_sync(0xffffffffu, hi[e].mn, o));
    }
    if (lane < LANES) {
      bounds[0][warp][f + e] = lo[e].mx, bounds[1][warp][f + e] = lo[e].mn;
      bounds[0][warp][f + D / 2 + e] = hi[e].mx, bounds[1][warp][f + D / 2 + e] = hi[e].mn;
    }
  }
  __syncthreads();
  if (blk < 0) return;
  uint32_t* sum = reinterpret_cast<uint32_t*>(a.c.summary + ((int64_t)blk * a.c.Hkv + h) * 2 * D);
  const bool fresh = it.r0 % P == 0;
  for (int i = tid; i < 2 * D / 4; i += blockDim.x) {  // four channels of one bound
    const int which = i / (D / 4), d = 4 * (i % (D / 4));
    const uint32_t old = fresh ? 0u : sum[i];
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = bounds[which][0][d + e];
      for (int w = 1; w < warps; ++w)
        x[e] = which ? fminf(x[e], bounds[1][w][d + e]) : fmaxf(x[e], bounds[0][w][d + e]);
      if (!fresh) x[e] = which ? fminf(x[e], unpack_s8(old, e)) : fmaxf(x[e], unpack_s8(old, e));
    }
    sum[i] = pack_s8(x[0], x[1], x[2], x[3]);
  }
}

// ------------------------------------------------------------------ summaries
constexpr int SUM_THREADS = 128;

template <int D>
__global__ void __launch_bounds__(SUM_THREADS) block_summaries_kernel(pced_paged_cache c, int* status) {
  constexpr int LANES = D / 8, ROWS = SUM_THREADS / LANES;  // a lane holds eight channels
  const int tid = threadIdx.x, s = blockIdx.y, j = blockIdx.x / c.Hkv, h = blockIdx.x % c.Hkv, P = c.block_rows;
  __shared__ float bounds[2][SUM_THREADS / 32][D];
  pdl_wait();
  const int live = min(P, paged_len(c, s, status) - j * P);
  if (live <= 0) return;
  const int blk = paged_block(c, s, j, status);
  if (blk < 0) return;
  const int64_t at = (int64_t)blk * c.Hkv + h;
  const float inv = __fdiv_rn(1.f, c.key_step[h]);
  const int f = 8 * (tid % LANES);
  const __nv_bfloat16* k = (const __nv_bfloat16*)c.k + at * P * D + f;
  KeyBounds b[8];
#pragma unroll 8
  for (int r = tid / LANES; r < live; r += ROWS) {
    float x[8];
    unpack8(*reinterpret_cast<const uint4*>(k + (int64_t)r * D), x);
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e].take(x[e], inv);
  }
  const int lane = tid & 31, warp = tid >> 5;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1)
      b[e].merge(__shfl_xor_sync(0xffffffffu, b[e].mx, o), __shfl_xor_sync(0xffffffffu, b[e].mn, o));
    if (lane < LANES) bounds[0][warp][f + e] = b[e].mx, bounds[1][warp][f + e] = b[e].mn;
  }
  __syncthreads();
  if (tid < 2 * D / 4) {
    const int which = tid / (D / 4), d = 4 * (tid % (D / 4));
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = bounds[which][0][d + e];
#pragma unroll
      for (int w = 1; w < SUM_THREADS / 32; ++w)
        x[e] = which ? fminf(x[e], bounds[1][w][d + e]) : fmaxf(x[e], bounds[0][w][d + e]);
    }
    reinterpret_cast<uint32_t*>(c.summary + at * 2 * D)[tid] = pack_s8(x[0], x[1], x[2], x[3]);
  }
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
  // (Hkv is the y extent of a grid)
  if (c->Hkv > 65535 || (int64_t)c->num_blocks * c->Hkv >= (INT64_C(1) << 31) ||
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

template <bool ONE>
static cudaError_t launch_append(const AppendArgs& a, dim3 grid, int threads, cudaStream_t s) {
  return a.c.D == 128 ? launch_pdl(kv_append_kernel<128, ONE>, grid, threads, 0, s, a)
                      : launch_pdl(kv_append_kernel<64, ONE>, grid, threads, 0, s, a);
}

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
    const int threads = ((a.G + 2) * (c.D / 16) + 31) / 32 * 32;  // a unit for every head
    e = launch_append<true>(a, dim3(c.S, c.Hkv), threads, (cudaStream_t)stream);
  } else {
    // blocks touched: at most two more than whole ones for every sequence with tokens
    const int64_t items = (int64_t)T / c.block_rows + 2 * (int64_t)(T < c.S ? T : c.S);
    if (items >= (INT64_C(1) << 31)) return fail(PCED_ERR_UNSUPPORTED, "%s: too many tokens", fn);
    e = launch_append<false>(a, dim3((unsigned)items, c.Hkv), APP_THREADS, (cudaStream_t)stream);
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
  const int64_t gx = (int64_t)c.max_blocks * c.Hkv;
  if (gx >= (INT64_C(1) << 31)) return fail(PCED_ERR_UNSUPPORTED, "%s: max_blocks * Hkv >= 2^31", fn);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  const dim3 grid((unsigned)gx, c.S);
  const cudaError_t e =
      c.D == 128 ? launch_pdl(block_summaries_kernel<128>, grid, SUM_THREADS, 0, (cudaStream_t)stream, c, status)
                 : launch_pdl(block_summaries_kernel<64>, grid, SUM_THREADS, 0, (cudaStream_t)stream, c, status);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "block_summaries launch");
}
