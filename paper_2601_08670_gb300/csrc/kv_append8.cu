// kv_append8.cu -- new keys and values into a paged cache of e4m3 numbers with a scale
// for each block, kv-head and kind, rotated on the way (pced_kv_append8).
//
// A block's scale is the smallest power of two, from 2^-100 on, of which its largest
// number is at most 448 times: e4m3's steps are relative, so a finer scale would gain
// nothing, and with powers of two the products with scale and 1 / scale are exact.
// New rows that need a larger scale than their block has move the rows that it holds
// already: e4m3(b s0 / s), which shifts exponents and rounds only what falls below the
// smallest normal number.  Keys are rounded once, from the rotated fp32 ones.
//
// So every block and kv-head takes two passes over its new rows: their largest number,
// then the bytes.
//
// What bounds them (one GB300, GPU time in a graph): sixteen documents, 18,366 tokens of
// 32 + 16 heads of 128, 427 MB in 90 us (4.8 TB/s, 70 % of the copy rate): a CTA's loads wait
// for the block's largest number before the bytes can be written, with 16 warps an SM to
// fill the time; queries alone, which are most of the bytes, would take 50.  32 tokens
// behind each of 33 documents 8.9 us, nine sequences' next token 3.2 us (a launch and
// four round trips: length, table, scale, write).  Where every block's scale grows, the moves
// come on top: nine tokens behind 32 rows each 1.6 us, behind 247 rows of a block of 256 8.7
// (a CTA of 48 threads moves them), 272 tokens behind 55 rows 6.3, 32 tokens behind each document 1.4.
#include <cuda_fp8.h>

#include "kv_append.cuh"

namespace pced {

struct Append8Args : AppendArgs {
  float* scale;  // [num_blocks][Hkv][2]
};

constexpr int A8_LOWEST = -100;  // exponent of the smallest scale

// The smallest power of two, from 2^A8_LOWEST on, of which `top` is at most 448
// (e4m3's largest number, 7/8 2^9) times.
__device__ __forceinline__ float scale_for(float top) {
  const uint32_t b = __float_as_uint(top);  // 1.m 2^(x - 127) <= 1.75 2^8 2^e
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u);
  return __uint_as_float((uint32_t)(max(e, A8_LOWEST) + 127) << 23);
}
// The largest |x| of x, y and top; an infinity shows (what is no number does not).
__device__ __forceinline__ float largest(const float (&x)[8], const float (&y)[8], float top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(x[e]), fabsf(y[e])));
  return top;
}
// ... of the finite ones alone: infinities have no part in a scale
__device__ __forceinline__ float largest_finite(const float (&x)[8], const float (&y)[8], float top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (fabsf(x[e]) < INFINITY) top = fmaxf(top, fabsf(x[e]));
    if (fabsf(y[e]) < INFINITY) top = fmaxf(top, fabsf(y[e]));
  }
  return top;
}
// x inv as e4m3, rounded to nearest even.  An infinity would become the largest number: see drop_infinite.
__device__ __forceinline__ uint32_t e4m3_pair(float x, float y, float inv) {
  return __nv_cvt_float2_to_fp8x2(make_float2(x * inv, y * inv), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint2 e4m3_8(const float (&x)[8], float inv) {
  return make_uint2(e4m3_pair(x[0], x[1], inv) | e4m3_pair(x[2], x[3], inv) << 16,
                    e4m3_pair(x[4], x[5], inv) | e4m3_pair(x[6], x[7], inv) << 16);
}
// infinities become not-a-number
__device__ __forceinline__ void drop_infinite(float (&x)[8], float (&y)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (fabsf(x[e]) == INFINITY) x[e] = NAN;
    if (fabsf(y[e]) == INFINITY) y[e] = NAN;
  }
}
// four e4m3 numbers times `ratio`, rounded again
__device__ __forceinline__ uint32_t move4(uint32_t w, float ratio) {
  uint32_t lo, hi;
  e4m3_to_f16(w, lo, hi);
  const float2 a = unpack_f16(lo), b = unpack_f16(hi);
  return e4m3_pair(a.x, a.y, ratio) | e4m3_pair(b.x, b.y, ratio) << 16;
}
// Rows [0, rows) of a page (and pool) times `ratio`: thread `at` of `n`.
template <int D>
__device__ __forceinline__ void move_rows(uint8_t* page, int rows, float ratio, int at, int n) {
  constexpr int BATCH = 4;  // loads in flight
  uint4* p = reinterpret_cast<uint4*>(page);
  const int parts = rows * (D / 16);
  for (int i0 = at; i0 < parts; i0 += BATCH * n) {
    uint4 w[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (i0 + u * n < parts) w[u] = p[i0 + u * n];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (i0 + u * n < parts)
        p[i0 + u * n] = make_uint4(move4(w[u].x, ratio), move4(w[u].y, ratio), move4(w[u].z, ratio), move4(w[u].w, ratio));
  }
}

// max and min that not-a-number wins
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// eight channels' largest (up) or smallest keys as whole steps, a byte each
__device__ __forceinline__ uint2 bound_steps(const float (&k)[8], bool up, float inv) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    w[e / 4] |= ((uint32_t)(up ? steps_up(k[e], inv) : steps_down(k[e], inv)) & 0xFFu) << (8 * (e % 4));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 merge_steps(uint2 a, uint2 b, bool up) {
  return up ? make_uint2(__vmaxs4(a.x, b.x), __vmaxs4(a.y, b.y)) : make_uint2(__vmins4(a.x, b.x), __vmins4(a.y, b.y));
}
__device__ __forceinline__ void update_bound(int8_t* at, uint2 w, bool up, bool fresh) {
  uint2* p = reinterpret_cast<uint2*>(at);
  *p = fresh ? w : merge_steps(w, *p, up);
}

// The scale of a block after new rows whose largest number is `top`.
__device__ __forceinline__ float grown(float s0, float top, bool fresh) {
  const float need = scale_for(top);
  return fresh ? need : fmaxf(s0, need);  // (a scale that is not a number counts as none)
}

// One token per sequence: a CTA per (sequence, kv-head), D/16 lanes for each row of a
// head, as in kv_append.cu.
constexpr int A8_ONE_THREADS = 8 * (PAGED_MAX_G + 2);  // (D = 128)

template <int D>
__global__ void __launch_bounds__(A8_ONE_THREADS) kv_append8_one_kernel(Append8Args a) {
  constexpr int LANES = D / 16;
  const int tid = threadIdx.x, lane = tid & 31, s = blockIdx.y, h = blockIdx.x, G = a.G, P = a.c.block_rows;
  const int role = tid / LANES, f = 8 * (tid % LANES);  // role 0: key, 1: value, then queries
  __shared__ float ratio[2];                            // by which rows move (1: they stay)
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
  const int at = (n - 1) % P;
  const int blk = fits ? paged_block(a.c, s, (n - 1) / P, a.status) : -1;  // (the table's last row is another token's)
  const int64_t page = (int64_t)blk * a.c.Hkv + h;
  const bool stored = blk >= 0 && PCED_IN_BOUNDS(in_pool(a.c, page, at), a.status);
  float s0 = 0.f;
  if (stored && role < 2) s0 = a.scale[2 * page + role];
  float co[8], si[8];
  const bool rotated =
      a.rope && role != 1 && load_angles(a, D, a.positions ? a.positions[s] : n - 1, f, co, si);
  if (role >= 2) {
    if (rotated) r.rotate(co, si);
    r.store(dst, D / 2);
  }
  if (!stored) return;
  if (role < 2) {
    float x[8], y[8];
    unpack8(r.a, x);
    unpack8(r.b, y);
    if (rotated) rotate8(x, y, co, si);
    float top = largest(x, y, 0.f);
    const bool infinite = top == INFINITY;
    if (infinite) top = largest_finite(x, y, 0.f);
    const uint32_t unit = (LANES == 8 ? 0xFFu : 0xFu) << (lane & ~(LANES - 1));
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor_sync(unit, top, o));
    const float sc = grown(s0, top, at == 0), inv = __fdiv_rn(1.f, sc);
    if (f == 0) {
      if (sc != s0) a.scale[2 * page + role] = sc;
      ratio[role] = sc == s0 ? 1.f : __fdiv_rn(s0, sc);
    }
    if (role == 0 && a.c.summary) {
      const float step = __fdiv_rn(1.f, a.c.key_step[h]);
      int8_t* sum = a.c.summary + page * 2 * D + f;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        update_bound(sum + which * D, bound_steps(x, !which, step), !which, at == 0);
        update_bound(sum + which * D + D / 2, bound_steps(y, !which, step), !which, at == 0);
      }
    }
    if (infinite) drop_infinite(x, y);
    uint8_t* row = (uint8_t*)(role ? a.c.v : a.c.k) + (page * P + at) * D + f;
    *reinterpret_cast<uint2*>(row) = e4m3_8(x, inv);
    *reinterpret_cast<uint2*>(row + D / 2) = e4m3_8(y, inv);
  }
  if (at == 0) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (ratio[i] != 1.f)
      move_rows<D>((uint8_t*)(i ? a.c.v : a.c.k) + page * P * D, at, ratio[i], tid, blockDim.x);
}

// Any number of tokens: a CTA takes one item (the new rows of one block) and a kv-head,
// or `heads` of them where items have few rows; D/16 lanes (a unit) share a row of a
// kv-head and its group.  A thread keeps its parts of the first rows in shared memory
// between the passes (16 bytes beside those of its neighbours: no conflicts, and no
// barrier), so that blocks of 64 rows and less are read once.
// Sixteen documents: 115 us with the rows read again from L2, 111 kept, 104 with the kept
// rows' copies under way before the queries, 90 us with four query heads' loads in flight
// at 4 CTAs an SM instead of two at 6 (eight at 3: 107).
constexpr int A8_CTAS = 4;   // CTAs that an SM holds
constexpr int A8_HOLD = 4;   // rows of a unit that are kept
constexpr int A8_HEADS = 4;  // query heads whose loads a thread has in flight

template <int D>
__global__ void __launch_bounds__(APP_THREADS, A8_CTAS) kv_append8_kernel(Append8Args a) {
  constexpr int LANES = D / 16, UNITS = APP_THREADS / LANES;
  const int tid = threadIdx.x, unit = tid / LANES, G = a.G, P = a.c.block_rows;
  const int heads = a.heads, per_item = a.c.Hkv / heads;
  const int h0 = (int)(blockIdx.x % per_item) * heads, mine = unit & (heads - 1), h = h0 + mine;
  __shared__ uint4 kept[A8_HOLD][4][APP_THREADS];
  __shared__ uint2 bounds[UNITS][2][D / 8];  // largest, smallest keys of a unit, in steps
  __shared__ float tops[UNITS][2];
  pdl_wait();
  const AppendItem it = find_item(a, blockIdx.x / per_item);
  if (it.s < 0) return;
  const int blk = paged_block(a.c, it.s, it.r0 / P, a.status);
  const int64_t page = (int64_t)blk * a.c.Hkv + h;
  const int f = 8 * (tid % LANES), at = it.r0 % P;
  const bool fresh = at == 0;
  float s0[2] = {0.f, 0.f};
  if (blk >= 0) s0[0] = a.scale[2 * page], s0[1] = a.scale[2 * page + 1];
  const int i0 = unit / heads, step = UNITS / heads;
  // ---- the first rows on their way, a group of copies each
#pragma unroll
  for (int j = 0; j < A8_HOLD; ++j) {
    const int i = i0 + j * step;
    if (i < it.m) {
      const __nv_bfloat16* kp = a.k + (it.t0 + i) * a.k_stride + h * D + f;
      const __nv_bfloat16* vp = a.v + (it.t0 + i) * a.v_stride + h * D + f;
      copy_async_16(smem_u32(&kept[j][0][tid]), kp);
      copy_async_16(smem_u32(&kept[j][1][tid]), kp + D / 2);
      copy_async_16(smem_u32(&kept[j][2][tid]), vp);
      copy_async_16(smem_u32(&kept[j][3][tid]), vp + D / 2);
    }
    copy_async_commit();
  }
  // ---- queries, and the largest of the keys and the values
  float top[2] = {0.f, 0.f};
  bool infinite = false;  // among this thread's
  for (int i = i0, j = 0; i < it.m; i += step, ++j) {
    const int64_t t = it.t0 + i;
    HeadRow kr, vr;
    if (j >= A8_HOLD) {
      kr.load(a.k + t * a.k_stride + h * D + f, D / 2);
      vr.load(a.v + t * a.v_stride + h * D + f, D / 2);
    }
    float co[8], si[8];
    const bool rotated = a.rope && load_angles(a, D, a.positions ? a.positions[t] : it.r0 + i, f, co, si);
    const __nv_bfloat16* q = a.q + t * a.q_stride + (int64_t)h * G * D + f;
    __nv_bfloat16* qo = a.q_out + (t * a.Hq + h * G) * D + f;
    for (int g0 = 0; g0 < G; g0 += A8_HEADS) {
      HeadRow x[A8_HEADS];
#pragma unroll
      for (int u = 0; u < A8_HEADS; ++u)
        if (g0 + u < G) x[u].load(q + (g0 + u) * D, D / 2);
#pragma unroll
      for (int u = 0; u < A8_HEADS; ++u) {
        if (g0 + u >= G) break;
        if (rotated) x[u].rotate(co, si);
        if (PCED_IN_BOUNDS(t < a.T, a.status)) x[u].store(qo + (g0 + u) * D, D / 2);
      }
    }
    if (j < A8_HOLD) {  // (this thread's own copies: no barrier)
      static_assert(A8_HOLD == 4, "the groups to wait for");
      if (j == 0) copy_async_wait<3>();
      else if (j == 1) copy_async_wait<2>();
      else if (j == 2) copy_async_wait<1>();
      else copy_async_wait<0>();
      kr.a = kept[j][0][tid], kr.b = kept[j][1][tid], vr.a = kept[j][2][tid], vr.b = kept[j][3][tid];
    }
    float x[8], y[8];
    unpack8(vr.a, x);
    unpack8(vr.b, y);
    const float v = largest(x, y, 0.f);
    top[1] = fmaxf(top[1], v < INFINITY ? v : largest_finite(x, y, 0.f));
    unpack8(kr.a, x);
    unpack8(kr.b, y);
    if (rotated) rotate8(x, y, co, si);
    const float k = largest(x, y, 0.f);
    top[0] = fmaxf(top[0], k < INFINITY ? k : largest_finite(x, y, 0.f));
    infinite |= v == INFINITY || k == INFINITY;
  }
  copy_async_wait<0>();
  if (blk < 0) return;
  // ---- units of the same head meet
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
    if (f == 0) tops[unit][i] = top[i];
  }
  __syncthreads();
  float inv[2], ratio[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    for (int u = mine; u < UNITS; u += heads) top[i] = fmaxf(top[i], tops[u][i]);
    const float sc = grown(s0[i], top[i], fresh);
    inv[i] = __fdiv_rn(1.f, sc);
    ratio[i] = fresh || sc == s0[i] ? 1.f : __fdiv_rn(s0[i], sc);
    top[i] = sc;
  }
  // ---- the rows again, as bytes
  float mx[16], mn[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) mx[e] = -INFINITY, mn[e] = INFINITY;
  for (int i = i0, j = 0; i < it.m; i += step, ++j) {
    const int64_t t = it.t0 + i;
    HeadRow kr, vr;
    if (j < A8_HOLD) {
      kr.a = kept[j][0][tid], kr.b = kept[j][1][tid], vr.a = kept[j][2][tid], vr.b = kept[j][3][tid];
    } else {
      kr.load(a.k + t * a.k_stride + h * D + f, D / 2);
      vr.load(a.v + t * a.v_stride + h * D + f, D / 2);
    }
    float co[8], si[8];
    const bool rotated = a.rope && load_angles(a, D, a.positions ? a.positions[t] : it.r0 + i, f, co, si);
    if (!PCED_IN_BOUNDS(t < a.T && in_pool(a.c, page, at + i), a.status)) continue;
    const int64_t row = (page * P + at + i) * D + f;
    float x[8], y[8];
    unpack8(vr.a, x);
    unpack8(vr.b, y);
    if (infinite) drop_infinite(x, y);
    *reinterpret_cast<uint2*>((uint8_t*)a.c.v + row) = e4m3_8(x, inv[1]);
    *reinterpret_cast<uint2*>((uint8_t*)a.c.v + row + D / 2) = e4m3_8(y, inv[1]);
    unpack8(kr.a, x);
    unpack8(kr.b, y);
    if (rotated) rotate8(x, y, co, si);
    if (a.c.summary) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        mx[e] = max_nan(mx[e], x[e]), mn[e] = min_nan(mn[e], x[e]);
        mx[8 + e] = max_nan(mx[8 + e], y[e]), mn[8 + e] = min_nan(mn[8 + e], y[e]);
      }
    }
    if (infinite) drop_infinite(x, y);
    *reinterpret_cast<uint2*>((uint8_t*)a.c.k + row) = e4m3_8(x, inv[0]);
    *reinterpret_cast<uint2*>((uint8_t*)a.c.k + row + D / 2) = e4m3_8(y, inv[0]);
  }
  // ---- the rows that the block held already: the units of a head share them
  if (!PCED_IN_BOUNDS(in_pool(a.c, page, at), a.status)) return;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (ratio[i] != 1.f)
      move_rows<D>((uint8_t*)(i ? a.c.v : a.c.k) + page * P * D, at, ratio[i], i0 * LANES + tid % LANES, APP_THREADS / heads);
  if (a.c.summary) {  // (a unit without rows: bounds that change nothing)
    const float steps = __fdiv_rn(1.f, a.c.key_step[h]);
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float k[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = which ? mn[8 * half + e] : mx[8 * half + e];
        bounds[unit][which][(f + half * (D / 2)) / 8] = bound_steps(k, !which, steps);
      }
  }
  __syncthreads();  // (the bounds; and all have read the old scales)
  if (unit < heads && f == 0) a.scale[2 * page] = top[0], a.scale[2 * page + 1] = top[1];
  if (!a.c.summary) return;
  for (int i = tid; i < heads * 2 * (D / 8); i += APP_THREADS) {  // eight channels of a head
    const int hh = i / (2 * (D / 8)), which = i / (D / 8) % 2, d = i % (D / 8);
    uint2 w = bounds[hh][which][d];
    for (int u = hh + heads; u < UNITS; u += heads) w = merge_steps(w, bounds[u][which][d], !which);
    update_bound(a.c.summary + ((int64_t)blk * a.c.Hkv + h0 + hh) * 2 * D + which * D + 8 * d, w, !which, fresh);
  }
}

}  // namespace pced

using namespace pced;
using namespace pced_host;

extern "C" pced_status pced_kv_append8(const pced_paged_cache8* cache, const void* q, int64_t q_stride, const void* k,
                                       int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int32_t Hq,
                                       const int32_t* tok_start, int32_t T, const float* rope, int32_t rope_rows,
                                       const int32_t* positions, int32_t* status, void* stream) {
  const char* fn = "pced_kv_append8";
  if (cache && !cache->scale) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (cache && !aligned(cache->scale, 8)) return fail(PCED_ERR_INVALID_ARG, "%s: misaligned cache pointer", fn);
  Append8Args a;
  const pced_status st = append_args(cache ? &cache->pages : nullptr, q, q_stride, k, k_stride, v, v_stride, q_out, Hq,
                                     tok_start, T, rope, rope_rows, positions, status, fn, a);
  if (st != PCED_OK || T == 0) return st;
  a.scale = cache->scale;
  const pced_paged_cache& c = a.c;
  cudaError_t e;
  if (!tok_start) {
    const int threads = (a.G + 2) * (c.D / 16);
    e = launch_pdl(c.D == 128 ? kv_append8_one_kernel<128> : kv_append8_one_kernel<64>, dim3(c.Hkv, c.S), threads, 0,
                   (cudaStream_t)stream, a);
  } else {
    const int64_t items = append_items(a, APP_THREADS / (c.D / 16), 1);
    if (!items) return fail(PCED_ERR_UNSUPPORTED, "%s: too many tokens", fn);
    e = launch_pdl(c.D == 128 ? kv_append8_kernel<128> : kv_append8_kernel<64>,
                   dim3((unsigned)(items * (c.Hkv / a.heads))), APP_THREADS, 0, (cudaStream_t)stream, a);
  }
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "kv_append8 launch");
}
