// logits.cu -- penalties for repeated tokens, biases and grammar masks on logits
// (pced_logits_process).
//
//   x <- (x > 0 ? x / t : x t) - (c f + p)   where the token is in the history c > 0 times
//   x <- x + bias;   x <- -inf where the mask's bit is clear
//
// A CTA takes LOG_CHUNK tokens of some of a query's rows.  It counts the
// history's tokens of the chunk in shared memory (whole numbers: the order does
// not matter) and marks the biased ones, then streams the rows, each asked for
// while the one before is processed; a thread keeps its tokens' mask bits, and a
// warp which of its places hold a repeated or biased token at all, in registers.
//
// What bounds it (one GB300, GPU time in a graph): HBM for many rows (272 rows of
// V = 151936, 331 MB in 60 us, 5.5 TB/s: 53 us without histories; with 4096 tokens
// each, counting them and the divisions of the first chunks, where the repeated
// tokens are, take 7), latency for few (nine rows of V = 128256 4.4 us).  Two rows in
// flight and none ahead: 69 us; per element tests for counts and biases: 94 us.
#include <math.h>

#include "common.cuh"

namespace pced {

constexpr int LOG_THREADS = 256;
constexpr int LOG_TOK = 8;  // tokens of a thread
constexpr int LOG_CHUNK = LOG_THREADS * LOG_TOK;
constexpr int LOG_CTAS = 4;  // CTAs that an SM holds
constexpr int LOG_HIST = 8;  // history tokens of a thread in flight

struct LogitsArgs {
  const float* x;
  float* y;
  int64_t stride;
  int32_t R, V, rows;  // rows: of a CTA
  const int32_t* history;
  int32_t history_stride;
  const int32_t* history_len;
  const float* penalties;
  const int32_t* bias_ids;
  const float* bias;
  int32_t n_bias;
  const uint32_t* mask;
  int32_t n_masks, mask_words;
  const int32_t* mask_row;
  int* status;
};

// Token e of this thread, from the chunk's first.  VEC: they are two runs of four,
// moved as 16 bytes.
template <bool VEC>
__device__ __forceinline__ int token_of(int e) {
  return VEC ? (e / 4 * LOG_THREADS + (int)threadIdx.x) * 4 + e % 4 : e * LOG_THREADS + (int)threadIdx.x;
}
template <bool VEC>
__device__ __forceinline__ void load_row(const LogitsArgs& a, int64_t at, int v0, float (&x)[LOG_TOK]) {
#pragma unroll
  for (int e = 0; e < LOG_TOK; e += VEC ? 4 : 1) {
    const int i = token_of<VEC>(e);
    if (v0 + i >= a.V) continue;
    if (VEC) *reinterpret_cast<float4*>(x + e) = *reinterpret_cast<const float4*>(a.x + at + i);
    else x[e] = a.x[at + i];
  }
}
template <bool VEC>
__device__ __forceinline__ void store_row(const LogitsArgs& a, int64_t at, int v0, const float (&x)[LOG_TOK]) {
#pragma unroll
  for (int e = 0; e < LOG_TOK; e += VEC ? 4 : 1) {
    const int i = token_of<VEC>(e);
    if (v0 + i >= a.V) continue;
    if (VEC) *reinterpret_cast<float4*>(a.y + at + i) = *reinterpret_cast<const float4*>(x + e);
    else a.y[at + i] = x[e];
  }
}

template <bool VEC>
__global__ void __launch_bounds__(LOG_THREADS, LOG_CTAS) logits_process_kernel(LogitsArgs a) {
  __shared__ __align__(16) int32_t count[LOG_CHUNK];
  __shared__ __align__(16) int32_t named[LOG_CHUNK];  // 1 + the last bias entry of the token; then the bias itself
  const int tid = threadIdx.x, b = blockIdx.x, v0 = blockIdx.z * LOG_CHUNK;
  const int r0 = blockIdx.y * a.rows, r1 = min(a.R, r0 + a.rows);
  const bool reports = blockIdx.z == 0 && blockIdx.y == 0;
  for (int i = tid; i < LOG_CHUNK / 4; i += LOG_THREADS) {
    reinterpret_cast<int4*>(count)[i] = make_int4(0, 0, 0, 0);
    reinterpret_cast<int4*>(named)[i] = make_int4(0, 0, 0, 0);
  }
  pdl_wait();
  const int64_t row0 = (int64_t)b * a.R * a.stride + v0;
  float x[LOG_TOK];  // the first row comes while the tokens are counted
  load_row<VEC>(a, row0 + r0 * a.stride, v0, x);
  int n = 0, m = -1;
  float rep = 1.f, freq = 0.f, pres = 0.f;
  if (a.history) {
    n = a.history_len[b];
    rep = a.penalties[3 * b], freq = a.penalties[3 * b + 1], pres = a.penalties[3 * b + 2];
  }
  if (a.mask) m = a.mask_row ? a.mask_row[b] : b;
  if (n < 0 || n > a.history_stride) {
    if (reports && tid == 0) dev_flag(a.status, PCED_DEV_BAD_LENGTH);
    n = n < 0 ? 0 : a.history_stride;
  }
  if (m < -1 || m >= a.n_masks) {
    if (reports && tid == 0) dev_flag(a.status, PCED_DEV_BAD_INDEX);
    m = -1;
  }
  __syncthreads();
  // bits to keep of this thread's tokens: none where the mask forbids them
  uint32_t keep[LOG_TOK];
#pragma unroll
  for (int e = 0; e < LOG_TOK; ++e) {
    const int v = v0 + token_of<VEC>(e);
    keep[e] = 0xFFFFFFFFu;
    if (m >= 0 && v < a.V) keep[e] = a.mask[(int64_t)m * a.mask_words + (v >> 5)] >> (v & 31) & 1u ? 0xFFFFFFFFu : 0u;
  }
  const int32_t* hist = a.history + (int64_t)b * a.history_stride;
  for (int i0 = tid; i0 < n; i0 += LOG_HIST * LOG_THREADS) {
    int t[LOG_HIST];
#pragma unroll
    for (int u = 0; u < LOG_HIST; ++u) t[u] = i0 + u * LOG_THREADS < n ? hist[i0 + u * LOG_THREADS] : -1;
#pragma unroll
    for (int u = 0; u < LOG_HIST; ++u) {
      if ((unsigned)(t[u] - v0) < (unsigned)LOG_CHUNK && t[u] < a.V) atomicAdd(&count[t[u] - v0], 1);
      if (reports && (t[u] < -1 || t[u] >= a.V)) dev_flag(a.status, PCED_DEV_BAD_TOKEN);
    }
  }
  for (int i = tid; i < a.n_bias; i += LOG_THREADS) {
    const int t = a.bias_ids[(int64_t)b * a.n_bias + i];
    if ((unsigned)(t - v0) < (unsigned)LOG_CHUNK && t < a.V) atomicMax(&named[t - v0], i + 1);
    if (reports && (t < -1 || t >= a.V)) dev_flag(a.status, PCED_DEV_BAD_TOKEN);
  }
  __syncthreads();
  // Which of the warp's places hold a repeated or a biased token: only there are
  // the counts and biases looked at again, row by row.
  uint32_t special = 0;
#pragma unroll
  for (int e = 0; e < LOG_TOK; ++e) {
    const int i = token_of<VEC>(e), w = named[i];
    if (w) named[i] = __float_as_int(a.bias[(int64_t)b * a.n_bias + w - 1]);  // (this thread's own from here on)
    if (__any_sync(0xffffffffu, w | count[i])) special |= 1u << e;
  }
  for (int r = r0; r < r1; ++r) {
    float next[LOG_TOK];  // ... and each other one while the one before it is processed
    if (r + 1 < r1) load_row<VEC>(a, row0 + (r + 1) * a.stride, v0, next);
#pragma unroll
    for (int e = 0; e < LOG_TOK; ++e) {
      if (special >> e & 1u) {
        const int i = token_of<VEC>(e);
        const float cnt = (float)count[i], add = __int_as_float(named[i]);
        if (cnt > 0.f)
          x[e] = __fsub_rn(x[e] > 0.f ? __fdiv_rn(x[e], rep) : __fmul_rn(x[e], rep),
                           __fadd_rn(__fmul_rn(cnt, freq), pres));
        if (add != 0.f) x[e] += add;
      }
      x[e] = __uint_as_float((__float_as_uint(x[e]) & keep[e]) | (~keep[e] & 0xFF800000u));  // or -inf
    }
    store_row<VEC>(a, row0 + r * a.stride, v0, x);
#pragma unroll
    for (int e = 0; e < LOG_TOK; ++e) x[e] = next[e];
  }
}

}  // namespace pced

using namespace pced;
using namespace pced_host;

extern "C" pced_status pced_logits_process(const float* x, float* y, int64_t stride, int32_t B, int32_t R, int32_t V,
                                           const int32_t* history, int32_t history_stride,
                                           const int32_t* history_len, const float* penalties,
                                           const int32_t* bias_ids, const float* bias, int32_t n_bias,
                                           const uint32_t* mask, int32_t n_masks, int32_t mask_words,
                                           const int32_t* mask_row, int32_t* status, void* stream) {
  const char* fn = "pced_logits_process";
  if (!x || !y) return fail(PCED_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (B < 1 || R < 1 || V < 1 || B > 65535 || R > 65535 || V > 65535 * LOG_CHUNK || stride < V) return fail(PCED_ERR_INVALID_ARG, "%s: bad sizes", fn);
  if (!history != !penalties || !history != !history_len || (history && history_stride < 1))
    return fail(PCED_ERR_INVALID_ARG, "%s: history, history_len and penalties go together", fn);
  if (n_bias < 0 || !bias_ids != !bias || (n_bias > 0) != (bias_ids != nullptr))
    return fail(PCED_ERR_INVALID_ARG, "%s: bias_ids, bias and n_bias go together", fn);
  if (mask ? n_masks < 1 || mask_words < (V - 1) / 32 + 1 || (!mask_row && n_masks < B) : mask_row != nullptr)
    return fail(PCED_ERR_INVALID_ARG, "%s: masks too few or too short", fn);
  const void* words[] = {x, y, history, history_len, penalties, bias_ids, bias, mask, mask_row, status};
  for (const void* p : words)
    if (((uintptr_t)p) & 3u) return fail(PCED_ERR_INVALID_ARG, "%s: misaligned pointer", fn);
  if (num_sms() <= 0) return fail(PCED_ERR_NO_DEVICE, "%s: no CUDA device", fn);
  LogitsArgs a;
  a.x = x, a.y = y, a.stride = stride;
  a.R = R, a.V = V;
  a.history = history, a.history_stride = history_stride, a.history_len = history_len;
  a.penalties = penalties;
  a.bias_ids = bias_ids, a.bias = bias, a.n_bias = n_bias;
  a.mask = mask, a.n_masks = n_masks, a.mask_words = mask_words, a.mask_row = mask_row;
  a.status = status;
  // Parts of a query's rows: no more than fill the SMs once, as each part counts its
  // chunk's tokens again (four queries of 17 rows 20 us; parts for three fillings 26,
  // and 23 against 18 with histories of 64 tokens)
  const int chunks = (V - 1) / LOG_CHUNK + 1;
  const int64_t parts = max((int64_t)1, min((int64_t)R, LOG_CTAS * (int64_t)num_sms() / ((int64_t)chunks * B)));
  a.rows = (int)((R + parts - 1) / parts);
  const bool vec = V % 4 == 0 && stride % 4 == 0 && (((uintptr_t)x | (uintptr_t)y) & 15u) == 0;
  // (the first chunks come first: low token numbers are the frequent ones, and repeated tokens cost time)
  const dim3 grid(B, (R - 1) / a.rows + 1, chunks);
  const cudaError_t e = vec ? launch_pdl(logits_process_kernel<true>, grid, LOG_THREADS, 0, (cudaStream_t)stream, a)
                            : launch_pdl(logits_process_kernel<false>, grid, LOG_THREADS, 0, (cudaStream_t)stream, a);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "logits_process launch");
}
