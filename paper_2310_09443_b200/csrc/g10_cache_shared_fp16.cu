// Attention of a batch behind a shared beginning: fp16, and the choice of the type.
#include "g10_cache_shared.cuh"

namespace g10 {

cudaError_t launch_cache_shared_fp16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s)
{
    return attend::launch_shared<__half>(begin, rest, shared, s);
}

cudaError_t launch_cache_shared_bf16(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, cudaStream_t s);
cudaError_t launch_cache_shared(const BeginArgs &begin, const RestArgs &rest, const int32_t *shared, int dtype, cudaStream_t s)
{
    return dtype == G10_BF16 ? launch_cache_shared_bf16(begin, rest, shared, s) : launch_cache_shared_fp16(begin, rest, shared, s);
}

}  // namespace g10
