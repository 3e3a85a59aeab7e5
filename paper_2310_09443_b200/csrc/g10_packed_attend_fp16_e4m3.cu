// Attention over rows of 8-bit codes: fp16 queries, e4m3 codes.
#include "g10_packed_attend.cuh"

namespace g10 {

cudaError_t launch_packed_fp16_e4m3(const PackedArgs &a, const AttendShape &z, cudaStream_t s) { return attend::launch_packed_type<__half, E4m3>(a, z, s); }

}  // namespace g10
