// Attention over a paged cache: the variants for a bfloat16 cache.
#include "decode.cuh"

namespace cp {

CP_JOINS(, CP_BF16, 8, 16)

int launch_decode_bf16(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_BF16>(a, s); }

}  // namespace cp
