// The weights that cached keys got in an attention over them, added up: weight_j +=
// sum_h exp(s_hj - lse_h) for the visible keys j, from the scores that the attention left
// (decode.cuh, in units of log 2).
//
// HBM or L2 bounds it: 4 bytes a key and query head, 8 a key.  A thread has a key and goes over the columns of
// scores, whose keys lie side by side: loads are whole lines, and heads are added up in
// the same order every time, without atomics.
#include "common.cuh"
#include "rope.cuh"

namespace cp {

constexpr int kWeighThreads = 128;

// P floats of a key in a column.
template <int P>
__device__ __forceinline__ void load_scores(const float* p, float (&s)[P]) {
  if constexpr (P == 1) {
    s[0] = *p;
  } else if constexpr (P == 2) {
    const float2 x = *reinterpret_cast<const float2*>(p);
    s[0] = x.x;
    s[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < P; i += 4) {
      const float4 x = *reinterpret_cast<const float4*>(p + i);
      s[i] = x.x;
      s[i + 1] = x.y;
      s[i + 2] = x.z;
      s[i + 3] = x.w;
    }
  }
}

template <int P>
__global__ void __launch_bounds__(kWeighThreads) k_weigh(DecodeArgs a, float* weight, int64_t weight_stride, int tiles, int pass,
                                                         int64_t chunks, int64_t items) {
  constexpr int kSide = P >= 8 ? 4 : 8;  // columns whose loads are under way together
  wait_for_stream();
  const int G = a.Hq / a.cache.heads;
  const int64_t apart = (int64_t)a.cache.capacity * P;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int b = (int)(item / chunks);
    const int len = min(max(a.lens[b], 0), a.cache.capacity);
    const int first = a.window > 0 && a.window < len ? len - (int)a.window : 0;
    const int64_t j = first + (item - b * chunks) * kWeighThreads + threadIdx.x;
    if (j >= len || (a.keep && !a.keep[b * a.keep_stride + j])) continue;
    float* to = weight + b * weight_stride + j;
    const float before = *to;
    const float* lse = a.lse + (int64_t)b * a.Hq;  // of the tile at hand
    const float* scores = a.scores + (int64_t)b * a.score_cols * apart + j * P;
    float sum = 0.0f;
    int tile = 0;  // of its kv head
    for (int c0 = 0; c0 < a.score_cols; c0 += kSide) {
      float s[kSide][P];
#pragma unroll
      for (int i = 0; i < kSide; ++i)
        if (c0 + i < a.score_cols) load_scores<P>(scores + i * apart, s[i]);
      scores += kSide * apart;
#pragma unroll
      for (int i = 0; i < kSide; ++i) {
        if (c0 + i < a.score_cols) {
          const int n = min(pass, G - tile * pass);
#pragma unroll
          for (int q = 0; q < P; ++q)
            if (q < n) {
              // exp2 off by 2^-22 of itself; a head whose scores are all -infinity has no weights
              const float top = lse[q];
              float w;
              asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(fmaf(-top, 1.4426950408889634f, s[i][q])));
              sum += top == -INFINITY ? 0.0f : w;
            }
          lse += n;
          if (++tile == tiles) tile = 0;
        }
      }
    }
    *to = before + sum;
  }
}

int launch_weigh(const DecodeArgs& a, int cache_dtype, float* weight, int64_t weight_stride, cudaStream_t s) {
  const int64_t most = a.window > 0 && a.window < a.cache.capacity ? a.window : a.cache.capacity;
  const int64_t chunks = (most + kWeighThreads - 1) / kWeighThreads, items = chunks * a.B;
  if (items == 0) return CP_OK;
  const int pass = decode_pass(cache_dtype, a.Hq / a.cache.heads), tiles = a.score_cols / a.cache.heads;
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int64_t room = (int64_t)di.sm_count * 16;
  const dim3 grid((unsigned)(items < room ? items : room));
  auto launch = [&](auto kernel) {
    return cuda_status(launch_early(kernel, grid, kWeighThreads, 0, s, a, weight, weight_stride, tiles, pass, chunks, items), "weigh");
  };
  switch (a.score_pitch) {
    case 1: return launch(k_weigh<1>);
    case 2: return launch(k_weigh<2>);
    case 4: return launch(k_weigh<4>);
    case 8: return launch(k_weigh<8>);
    default: return launch(k_weigh<16>);
  }
}

}  // namespace cp
