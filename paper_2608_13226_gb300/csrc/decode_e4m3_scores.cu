// Attention over a paged cache: the variants for a 8-bit cache that leave the scores behind.
#include "decode.cuh"

namespace cp {

CP_JOINS(extern, CP_E4M3, 8, 16)

int launch_decode_e4m3_scores(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_E4M3, true>(a, s); }

}  // namespace cp
