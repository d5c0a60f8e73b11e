// sample_bf16.cu -- pced_sample's kernel (sample.cuh) for bf16.
#include "sample.cuh"

namespace pced {
template cudaError_t launch_sample_t<__nv_bfloat16>(SampleArgs, int32_t, cudaStream_t);
}  // namespace pced
