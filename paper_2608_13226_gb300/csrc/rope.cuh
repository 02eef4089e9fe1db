// Device side of the rotary positions: angles of any position, and the loads
// and stores of one element in the types of rows and caches.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "serve.h"

namespace cp {

// What ran before on the stream has ended and is seen from here on; what comes after
// may begin to wait likewise (launch_early), at once or from then on.  Every thread
// of the grid calls it before it reads or writes memory.
__device__ __forceinline__ void wait_for_stream(bool at_once = true) {
  if (at_once) asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (!at_once) asm volatile("griddepcontrol.launch_dependents;");
}

// A pair's speed as the fraction of a turn that one position takes, in units
// of 2^-64 turns.  Whole turns drop out, and so they do of position * speed in
// 64-bit integers: the angle of a position is off by 2^-64 turns for each of it.
// The float64's significand times 2^128 / (2 pi), cut to the units below a turn: integers, as a
// float64 product's two roundings would make 9e-5 rad at position 2^40.  (Three float64
// operations that keep what they round off would do as well, 0.1 us later: 1/64 of the
// float32 rate.)  Speeds of 2^53 and more, which are whole radians, count as 0.
__device__ __forceinline__ uint64_t rope_turns(double inv_freq) {
  constexpr uint64_t high = 0x28BE60DB9391054Aull, low = 0x7F09D5F47D4D3770ull;
  const uint64_t bits = (uint64_t)__double_as_longlong(inv_freq);
  const int s = (int)(bits >> 52 & 2047) - 1011;  // inv_freq = m 2^(s - 64)
  if (s > 64 || s < -63) return 0;
  const uint64_t m = (bits & (((uint64_t)1 << 52) - 1)) | (uint64_t)1 << 52;
  const unsigned __int128 p = (unsigned __int128)m * high + __umul64hi(m, low);  // m 2^64 / (2 pi)
  const uint64_t u = (uint64_t)(p >> (64 - s));
  return bits >> 63 ? 0 - u : u;
}

// (cos, sin) of the angle, times the scale.  The turn's fraction is cut to 32 bits
// (1.5e-9 rad), its nearest quarter taken off as an integer, and the rest, within
// pi / 4, goes into the series of sine and cosine up to x^9 / 9! and x^10 / 10!
// (what is left out is under 2e-9): about 6e-8 of error from roundings, in a third
// of the instructions of a call that reduces its argument itself.
__device__ __forceinline__ void rope_unit(uint64_t turns, int64_t pos, const Rope& r, float* c,
                                          float* s) {
  const uint32_t a = (uint32_t)((turns * (uint64_t)pos) >> 32);
  const uint32_t quarter = (a + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(a - (quarter << 30)) * (float)(1.57079632679489661923 / 1073741824.0);
  const float y = x * x;
  float sn = fmaf(y, 1.0f / 362880.0f, -1.0f / 5040.0f);
  sn = fmaf(y, sn, 1.0f / 120.0f);
  sn = fmaf(y, sn, -1.0f / 6.0f);
  sn = fmaf(x * y, sn, x);
  float cs = fmaf(y, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  cs = fmaf(y, cs, -1.0f / 720.0f);
  cs = fmaf(y, cs, 1.0f / 24.0f);
  cs = fmaf(y, cs, -0.5f);
  cs = fmaf(y, cs, 1.0f);
  const bool odd = quarter & 1;
  const float u = odd ? sn : cs, v = odd ? cs : sn;
  *c = ((quarter + 1) & 2 ? -u : u) * r.scale;
  *s = ((quarter & 2) != 0) != (r.back != 0) ? -v * r.scale : v * r.scale;
}

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <> __device__ __forceinline__ __nv_fp8_e4m3 from_f32<__nv_fp8_e4m3>(float x) {
  return __nv_fp8_e4m3(x);  // to nearest even, saturating
}

// The sequence that row t belongs to: how many of starts[1..B] are <= t.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int B, int64_t t) {
  int lo = 0, n = B;  // the first lo are, those from lo + n on are not
  while (n > 0) {
    const int h = n / 2;
    if (starts[1 + lo + h] <= t) {
      lo += h + 1;
      n -= h + 1;
    } else {
      n = h;
    }
  }
  return lo;
}

// Two float32 in a register pair, and products and sums of both at once.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  return (uint64_t)__float_as_uint(hi) << 32 | __float_as_uint(lo);
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// n / d for 0 <= n < 2^31 by a product: with 2^l >= d, mul = ceil(2^(31 + l) / d)
// is off by less than d / 2^(31 + l), and n times that by less than 1 / d.
struct Divisor {
  uint32_t d, mul, shift;
  __device__ __forceinline__ int of(int n) const { return (int)((uint64_t)(uint32_t)n * mul >> 31 >> shift); }
};
inline Divisor divisor(int d) {
  if (d < 1) d = 1;
  uint32_t l = 0;
  while (((int64_t)1 << l) < d) ++l;
  return Divisor{(uint32_t)d, (uint32_t)((((uint64_t)1 << (31 + l)) + d - 1) / d), l};
}

}  // namespace cp
