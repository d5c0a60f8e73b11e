// paged.cuh -- what the operators over a pced_paged_cache share: its checks on
// the host, and on the device lengths, table entries and key steps.
#pragma once
#include "common.cuh"

namespace pced {

constexpr int PAGED_MAX_S = 1024;  // sequences of a call (their lengths and prefixes lie in shared memory)
constexpr int PAGED_MAX_G = 8;     // query heads per kv-head

// live rows of sequence s, clipped into what its table can hold
__device__ __forceinline__ int paged_len(const pced_paged_cache& c, int s, int* status) {
  const int n = c.seq_len[s];
  const int cap = c.max_blocks * c.block_rows;
  if (n >= 0 && n <= cap) return n;
  dev_flag(status, PCED_DEV_BAD_LENGTH);
  return n < 0 ? 0 : cap;
}
// pool block of block j of sequence s, -1 where the entry is outside the pool
__device__ __forceinline__ int paged_block(const pced_paged_cache& c, int s, int j, int* status) {
  const int b = c.block_table[(int64_t)s * c.max_blocks + j];
  if (b >= 0 && b < c.num_blocks) return b;
  dev_flag(status, PCED_DEV_BAD_BLOCK);
  return -1;
}

// ------------------------------------------------------------- key summaries
// Largest and smallest key of a channel in whole steps: the bounds of what one
// thread has seen (fp32 holds these whole numbers exactly).
struct KeyBounds {
  float mx = -127.f, mn = 127.f;
  __device__ __forceinline__ void take(float k, float inv_step) {
    const float x = __fmul_rn(k, inv_step);
    // (fmaxf and fminf drop what is not a number)
    mx = x != x ? 127.f : fmaxf(mx, fminf(ceilf(x), 127.f));
    mn = x != x ? -127.f : fminf(mn, fmaxf(floorf(x), -127.f));
  }
  __device__ __forceinline__ void merge(float mx2, float mn2) {
    mx = fmaxf(mx, mx2);
    mn = fminf(mn, mn2);
  }
};
__device__ __forceinline__ uint32_t pack_s8(float a, float b, float c, float d) {
  return ((uint32_t)(int)a & 0xFFu) | ((uint32_t)(int)b & 0xFFu) << 8 | ((uint32_t)(int)c & 0xFFu) << 16 |
         ((uint32_t)(int)d & 0xFFu) << 24;
}
__device__ __forceinline__ float unpack_s8(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

}  // namespace pced

namespace pced_host {
// host-visible checks of a cache (all but its k, v, summary and key_step
// pointers, which differ from call to call)
pced_status check_paged_cache(const pced_paged_cache* c, const char* fn);
// ... and of a call's query heads over it
pced_status check_paged_heads(const pced_paged_cache* c, int32_t Hq, const char* fn);
// host.cu: make_tmap_kv with `blocks` of the D / 64 column blocks in a copy
pced_status make_tmap_kv_part(CUtensorMap* map, const void* base, uint64_t rows, uint32_t D, uint32_t box_rows,
                              uint32_t blocks);
// more than 48 KB of dynamic shared memory for a kernel: asked for once per device
template <typename K>
inline cudaError_t allow_smem(K kernel, size_t bytes, bool (&done)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (done[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  done[dev] = e == cudaSuccess;
  return e;
}
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
}  // namespace pced_host
