// Attention over a paged cache: the variants for a 4-bit cache that leave the scores behind.
#include "decode.cuh"

namespace cp {

CP_JOINS(extern, CP_I4, 8, 16)

int launch_decode_i4_scores(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_I4, true>(a, s); }

}  // namespace cp
