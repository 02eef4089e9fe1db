// Attention over a paged cache: the variants for a 8-bit cache.
#include "decode.cuh"

namespace cp {

int launch_decode_e4m3(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_E4M3>(a, s); }

}  // namespace cp
