// paged.cuh -- what the operators over a pced_paged_cache share: its checks on
// the host, and on the device lengths, table entries and key steps.
#pragma once
#include "common.cuh"

namespace pced {

constexpr int PAGED_MAX_S = 1024;  // sequences of a call (their lengths and prefixes lie in shared memory)
constexpr int PAGED_MAX_G = 8;     // query heads per kv-head

// live rows of sequence s, clipped into what its table can hold; fits: they were not
__device__ __forceinline__ int paged_len(const pced_paged_cache& c, int s, int* status, bool& fits) {
  const int n = c.seq_len[s];
  const int cap = c.max_blocks * c.block_rows;
  fits = n >= 0 && n <= cap;
  if (fits) return n;
  dev_flag(status, PCED_DEV_BAD_LENGTH);
  return n < 0 ? 0 : cap;
}
__device__ __forceinline__ int paged_len(const pced_paged_cache& c, int s, int* status) {
  bool fits;
  return paged_len(c, s, status, fits);
}
// pool block of block j of sequence s, -1 where the entry is outside the pool
__device__ __forceinline__ int paged_block(const pced_paged_cache& c, int s, int j, int* status) {
  const int b = c.block_table[(int64_t)s * c.max_blocks + j];
  if (b >= 0 && b < c.num_blocks) return b;
  dev_flag(status, PCED_DEV_BAD_BLOCK);
  return -1;
}
// row r of page (block, kv-head) lies in the pool (guards of the bounds-checked build)
__device__ __forceinline__ bool in_pool(const pced_paged_cache& c, int64_t page, int r) {
  return page >= 0 && page < (int64_t)c.num_blocks * c.Hkv && r >= 0 && r < c.block_rows;
}

// ------------------------------------------------------------- key summaries
// Largest and smallest of two channels' keys, as bf16 pairs (one instruction for
// two keys each; not-a-number wins).  The product with 1 / key_step, rounded,
// and ceil, floor and the clipping are monotone, so they are taken of the bounds
// alone: counted per key they bound the summaries of 272 caches at 150 us.
struct KeyBounds2 {
  __nv_bfloat162 mx, mn;
  __device__ __forceinline__ void reset() {
    mx = __float2bfloat162_rn(-INFINITY);
    mn = __float2bfloat162_rn(INFINITY);
  }
  __device__ __forceinline__ void take(uint32_t k) { merge(k, k); }
  __device__ __forceinline__ void merge(uint32_t mx2, uint32_t mn2) {
    mx = __hmax2_nan(mx, *reinterpret_cast<const __nv_bfloat162*>(&mx2));
    mn = __hmin2_nan(mn, *reinterpret_cast<const __nv_bfloat162*>(&mn2));
  }
  __device__ __forceinline__ uint32_t top() const { return *reinterpret_cast<const uint32_t*>(&mx); }
  __device__ __forceinline__ uint32_t bottom() const { return *reinterpret_cast<const uint32_t*>(&mn); }
  // with the bounds of lane ^ o
  __device__ __forceinline__ void merge_xor(int o) {
    const uint32_t x = __shfl_xor_sync(0xffffffffu, top(), o), y = __shfl_xor_sync(0xffffffffu, bottom(), o);
    merge(x, y);
  }
};
// whole steps of a largest key, and of a smallest one
__device__ __forceinline__ int steps_up(float k, float inv_step) {
  const float x = __fmul_rn(k, inv_step);
  return x != x ? 127 : (int)fminf(fmaxf(ceilf(x), -127.f), 127.f);
}
__device__ __forceinline__ int steps_down(float k, float inv_step) {
  const float x = __fmul_rn(k, inv_step);
  return x != x ? -127 : (int)fminf(fmaxf(floorf(x), -127.f), 127.f);
}
// the steps of four channels (two words of bf16), a byte each
__device__ __forceinline__ uint32_t steps4(uint32_t a, uint32_t b, bool up, float inv) {
  const float k[4] = {bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b)};
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) w |= ((uint32_t)(up ? steps_up(k[i], inv) : steps_down(k[i], inv)) & 0xFFu) << (8 * i);
  return w;
}

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
// ... over a pool of `rows` rows of D bytes, box_rows whole rows in a copy, swizzled
// over D bytes (16-byte part c of row r lies at c ^ (r & 7), for D = 64 at c ^ (r >> 1 & 3))
pced_status make_tmap_bytes(CUtensorMap* map, const void* base, uint64_t rows, uint32_t D, uint32_t box_rows);
// more than 48 KB of dynamic shared memory for a kernel: asked for once per device (host
// threads call at the same time)
template <typename K>
inline cudaError_t allow_smem(K kernel, size_t bytes, std::atomic<bool> (&done)[64]) {
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
