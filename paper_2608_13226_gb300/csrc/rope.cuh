// Device side of the rotary positions: angles of any position, and the loads
// and stores of one element in the types of rows and caches.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "serve.h"

namespace cp {

// A pair's speed as the fraction of a turn that one position takes, in units
// of 2^-64 turns.  Whole turns drop out, and so they do of position * speed in
// 64-bit integers: the angle of any position is off by no more than the speed's
// own rounding (float64: 2^-54 of the turns made).
__device__ __forceinline__ uint64_t rope_turns(double inv_freq) {
  double t = inv_freq * 0.15915494309189533577;  // 1 / (2 pi)
  t -= floor(t);
  return __double2ull_rz(t * 18446744073709551616.0);
}

__device__ __forceinline__ void rope_unit(uint64_t turns, int64_t pos, const Rope& r, float* c,
                                          float* s) {
  const int64_t a = (int64_t)(turns * (uint64_t)pos);
  float sn, cs;
  sincospif(__ll2float_rn(a) * 0x1p-63f, &sn, &cs);  // 2 a / 2^64 half turns, in [-1, 1]
  *c = cs * r.scale;
  *s = (r.back ? -sn : sn) * r.scale;
}

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <> __device__ __forceinline__ __nv_fp8_e4m3 from_f32<__nv_fp8_e4m3>(float x) {
  return __nv_fp8_e4m3(x);  // to nearest even, saturating
}
__device__ __forceinline__ float to_f32(__nv_fp8_e4m3 x) { return (float)x; }

}  // namespace cp
