// paged_attention.cu -- one layer of decode attention over a paged cache, over
// all blocks or the selected ones (pced_paged_attention).
//
// One CTA per (sequence, kv-head): its warps take the rows in turn, each with a
// running maximum and sum per query head, and meet in shared memory at the end.
#include <math.h>

#include "paged.cuh"

namespace pced {

constexpr int PATT_THREADS = 256;
constexpr int PATT_WARPS = PATT_THREADS / 32;

struct PagedAttArgs {
  pced_paged_cache c;
  const __nv_bfloat16* q;
  int64_t q_stride;
  int32_t Hq, G;
  const int32_t* sel;
  int32_t n_sel;
  float scale_log2;
  void* out;
  int32_t out_bf16;
  float* lse;
  int* status;
};

template <int D>
__global__ void __launch_bounds__(PATT_THREADS) paged_attention_kernel(PagedAttArgs a) {
  constexpr int E = D / 32;  // channels of a lane
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.x, s = blockIdx.y, G = a.G, P = a.c.block_rows;
  __shared__ float ms[PATT_WARPS][PAGED_MAX_G], ls[PATT_WARPS][PAGED_MAX_G];
  __shared__ float os[PATT_WARPS][PAGED_MAX_G][D];
  pdl_wait();
  const int n = paged_len(a.c, s, a.status);
  const int nb = (n + P - 1) / P;
  float q[PAGED_MAX_G][E], o[PAGED_MAX_G][E], m[PAGED_MAX_G], l[PAGED_MAX_G];
#pragma unroll
  for (int g = 0; g < PAGED_MAX_G; ++g) {
    m[g] = -INFINITY, l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      o[g][e] = 0.f;
      q[g][e] = g < G ? __bfloat162float(a.q[s * a.q_stride + (int64_t)(h * G + g) * D + lane + 32 * e]) : 0.f;
    }
  }
  const int blocks = a.sel ? a.n_sel : nb;
  for (int i = 0; i < blocks; ++i) {
    const int j = a.sel ? a.sel[((int64_t)s * a.c.Hkv + h) * a.n_sel + i] : i;
    if (j == -1) continue;
    if (j < 0 || j >= nb) {
      dev_flag(a.status, PCED_DEV_BAD_BLOCK);
      continue;
    }
    const int blk = paged_block(a.c, s, j, a.status);
    if (blk < 0) continue;
    const int64_t base = ((int64_t)blk * a.c.Hkv + h) * P * D;
    const int live = min(P, n - j * P);
    for (int r = warp; r < live; r += PATT_WARPS) {
      const __nv_bfloat16* k = (const __nv_bfloat16*)a.c.k + base + (int64_t)r * D + lane;
      const __nv_bfloat16* v = (const __nv_bfloat16*)a.c.v + base + (int64_t)r * D + lane;
      float kf[E], vf[E];
#pragma unroll
      for (int e = 0; e < E; ++e) kf[e] = __bfloat162float(k[32 * e]), vf[e] = __bfloat162float(v[32 * e]);
#pragma unroll
      for (int g = 0; g < PAGED_MAX_G; ++g) {
        if (g >= G) break;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x += q[g][e] * kf[e];
        x = warp_sum(x) * a.scale_log2;
        const float mn = fmaxf(m[g], x), f = m[g] == -INFINITY ? 0.f : exp2f(m[g] - mn);
        const float p = mn == -INFINITY ? 0.f : exp2f(x - mn);
        l[g] = l[g] * f + p;
        m[g] = mn;
#pragma unroll
        for (int e = 0; e < E; ++e) o[g][e] = o[g][e] * f + p * vf[e];
      }
    }
  }
#pragma unroll
  for (int g = 0; g < PAGED_MAX_G; ++g) {
    if (lane == 0) ms[warp][g] = m[g], ls[warp][g] = l[g];
#pragma unroll
    for (int e = 0; e < E; ++e) os[warp][g][lane + 32 * e] = o[g][e];
  }
  __syncthreads();
  for (int i = tid; i < G * D; i += PATT_THREADS) {
    const int g = i / D, d = i % D;
    float mx = -INFINITY, sum = 0.f, acc = 0.f;
    for (int w = 0; w < PATT_WARPS; ++w) mx = fmaxf(mx, ms[w][g]);
    for (int w = 0; w < PATT_WARPS; ++w) {
      const float f = ms[w][g] == -INFINITY ? 0.f : exp2f(ms[w][g] - mx);
      sum += ls[w][g] * f;
      acc += os[w][g][d] * f;
    }
    const float y = mx == -INFINITY ? 0.f : acc / sum;
    const int64_t at = ((int64_t)s * a.Hq + h * G + g) * D + d;
    if (a.out_bf16) ((__nv_bfloat16*)a.out)[at] = __float2bfloat16_rn(y);
    else ((float*)a.out)[at] = y;
    if (a.lse && d == 0)
      a.lse[(int64_t)s * a.Hq + h * G + g] = mx == -INFINITY ? -INFINITY : (mx + log2f(sum)) * 0.6931471805599453f;
  }
}

}  // namespace pced

using namespace pced;
using namespace pced_host;

extern "C" size_t pced_paged_attention_workspace_size(int32_t S, int32_t Hq, int32_t Hkv, int32_t D) {
  if (S < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || D < 1) return 0;
  return 256;
}

extern "C" pced_status pced_paged_attention(const pced_paged_cache* cache, const void* q, int64_t q_stride, int32_t Hq,
                                            const int32_t* sel, int32_t n_sel, int64_t total_rows, float scale,
                                            void* out, int32_t out_type, float* lse, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  const char* fn = "pced_paged_attention";
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
  if (!isfinite(scale) || total_rows < 0) return fail(PCED_ERR_INVALID_ARG, "%s: scale or total_rows", fn);
  if (!aligned(workspace, 256) || workspace_bytes < pced_paged_attention_workspace_size(c.S, Hq, c.Hkv, c.D))
    return fail(PCED_ERR_WORKSPACE, "%s: workspace too small or misaligned", fn);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  PagedAttArgs a;
  a.c = c;
  a.q = (const __nv_bfloat16*)q;
  a.q_stride = q_stride;
  a.Hq = Hq, a.G = Hq / c.Hkv;
  a.sel = sel, a.n_sel = n_sel;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.out = out, a.out_bf16 = out_type == PCED_OUT_BF16;
  a.lse = lse;
  a.status = (int*)workspace;
  const dim3 grid(c.Hkv, c.S);
  const cudaError_t e =
      c.D == 128 ? launch_pdl(paged_attention_kernel<128>, grid, PATT_THREADS, 0, (cudaStream_t)stream, a)
                 : launch_pdl(paged_attention_kernel<64>, grid, PATT_THREADS, 0, (cudaStream_t)stream, a);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "paged_attention launch");
}
