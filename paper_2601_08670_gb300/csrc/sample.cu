// sample.cu -- pced_sample: a token for every row of logits; its kernel (sample.cuh) for fp32.
#include "sample.cuh"

namespace pced {
template cudaError_t launch_sample_t<float>(SampleArgs, int32_t, cudaStream_t);
}  // namespace pced

using namespace pced;
using namespace pced_host;

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
  const cudaError_t e = type == PCED_IN_F32 ? launch_sample_t<float>(a, rows, (cudaStream_t)stream)
                                             : launch_sample_t<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
  return e == cudaSuccess ? PCED_OK : cuda_status(e, "sample launch");
}
