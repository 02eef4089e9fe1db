// Attention over a paged cache: the variants for a float32 cache.
#include "decode.cuh"

namespace cp {

int launch_decode_f32(const DecodeArgs& a, cudaStream_t s) { return launch_type<CP_F32>(a, s); }

}  // namespace cp
