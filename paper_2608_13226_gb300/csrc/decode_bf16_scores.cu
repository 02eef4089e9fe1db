// Attention over a paged cache: the variants for a bfloat16 cache that leave the scores behind.
#include "decode.cuh"

namespace cp {

CP_JOINS(extern, CP_BF16, 8, 16)

int launch_decode_bf16_scores(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_BF16, true>(a, s); }

}  // namespace cp
