// Attention over a paged cache: the variants for a float32 cache that leave the scores behind.
#include "decode.cuh"

namespace cp {

CP_JOINS(extern, CP_F32, 4, 8)

int launch_decode_f32_scores(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_F32, true>(a, s); }

}  // namespace cp
