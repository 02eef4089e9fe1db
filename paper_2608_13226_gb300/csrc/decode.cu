// Attention over a paged cache: the choice by the cache's type.  The kernels are in
// decode.cuh, a translation unit a type.
#include "serve.h"

namespace cp {

// What the attention leaves in its workspace: where query tiles begin, and two parts
// a block at most, each a maximum, a sum and an output a query.
size_t decode_ws_bytes(int64_t Hq, int64_t heads, int64_t D, int cache_dtype) {
  const size_t QT = decode_pass(cache_dtype, Hq / heads), DP = decode_width(D);
  return kDecodeBlocks * (sizeof(Begin) + 2 * sizeof(float) * QT * (DP + 2));
}

int launch_decode(const DecodeArgs& a, int cache_dtype, cudaStream_t s) {
  if (cache_dtype == CP_F32) return launch_decode_f32(a, s);
  if (cache_dtype == CP_BF16) return launch_decode_bf16(a, s);
  if (cache_dtype == CP_I4) return launch_decode_i4(a, s);
  return launch_decode_e4m3(a, s);
}

int launch_decode_scores(const DecodeArgs& a, int cache_dtype, cudaStream_t s) {
  if (cache_dtype == CP_F32) return launch_decode_f32_scores(a, s);
  if (cache_dtype == CP_BF16) return launch_decode_bf16_scores(a, s);
  if (cache_dtype == CP_I4) return launch_decode_i4_scores(a, s);
  return launch_decode_e4m3_scores(a, s);
}

}  // namespace cp
