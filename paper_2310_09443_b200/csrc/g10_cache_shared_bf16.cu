// Attention of a batch behind a shared beginning: bf16.
#include "g10_cache_shared.cuh"

namespace g10 {

cudaError_t launch_cache_shared_bf16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s)
{
    return attend::launch_shared<__nv_bfloat16>(begin, rest, shared, s);
}

}  // namespace g10
