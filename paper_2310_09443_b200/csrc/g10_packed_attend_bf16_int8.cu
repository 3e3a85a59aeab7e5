// Attention over rows of 8-bit codes: bf16 queries, int8 codes.
#include "g10_packed_attend.cuh"

namespace g10 {

cudaError_t launch_packed_bf16_int8(const PackedArgs &a, const AttendShape &z, cudaStream_t s) { return attend::launch_packed_type<__nv_bfloat16, Int8>(a, z, s); }

}  // namespace g10
