// Attention over a paged cache: the variants for a 4-bit cache.
#include "decode.cuh"

namespace cp {

CP_JOINS(, CP_I4, 8, 16)

int launch_decode_i4(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_I4>(a, s); }

}  // namespace cp
