// The weights that cached keys got in an attention over them, added up: weight_j +=
// sum_h exp(s_hj - lse_h) for the visible keys j, from the scores that the attention left
// (decode.cuh, in units of log 2).
//
// HBM or L2 bounds it: 4 bytes a key and query head, 8 a key.  A key's scores lie side by
// side, so lanes take its query heads (32 at most, of fewer heads several keys side by
// side) and add them up among themselves: the same order every time, no atomics.
#include "common.cuh"
#include "rope.cuh"

namespace cp {

constexpr int kWeighThreads = 256;
constexpr int kSide = 4;  // keys of a lane whose loads are under way together

__global__ void __launch_bounds__(kWeighThreads) k_weigh(DecodeArgs a, float* weight, int64_t weight_stride, int lanes,
                                                         int chunk, int64_t chunks, int64_t items) {
  wait_for_stream();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int keys = 32 / lanes, mine = lane / lanes, head = lane % lanes;  // keys side by side, this lane's
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int b = (int)(item / chunks);
    const int len = min(max(a.lens[b], 0), a.cache.capacity);
    const int first = a.window > 0 && a.window < len ? len - (int)a.window : 0;
    const int64_t begin = first + (item - b * chunks) * chunk;
    if (begin >= len) continue;
    const int end = (int)min((int64_t)len, begin + chunk);
    const float* scores = a.scores + (int64_t)b * a.cache.capacity * a.Hq;
    const float* lse = a.lse + (int64_t)b * a.Hq;
    float* to = weight + b * weight_stride;
    for (int j0 = (int)begin + warp * keys * kSide; j0 < end; j0 += kWeighThreads / 32 * keys * kSide) {
      float sum[kSide];
      bool seen[kSide];
#pragma unroll
      for (int i = 0; i < kSide; ++i) {
        const int j = j0 + i * keys + mine;
        seen[i] = j < end && (!a.keep || a.keep[b * a.keep_stride + j]);
        sum[i] = 0.0f;
      }
      for (int h = head; h < a.Hq; h += lanes) {
        const float top = lse[h];
        float s[kSide];
#pragma unroll
        for (int i = 0; i < kSide; ++i)
          s[i] = seen[i] ? scores[(int64_t)(j0 + i * keys + mine) * a.Hq + h] : -INFINITY;
#pragma unroll
        for (int i = 0; i < kSide; ++i)  // (a head whose scores are all -infinity has no weights)
          if (top != -INFINITY) sum[i] += exp2f(fmaf(-top, 1.4426950408889634f, s[i]));
      }
#pragma unroll
      for (int i = 0; i < kSide; ++i) {
        for (int d = 1; d < lanes; d *= 2) sum[i] += __shfl_xor_sync(~0u, sum[i], d);
        if (seen[i] && head == 0) to[j0 + i * keys + mine] += sum[i];
      }
    }
  }
}

int launch_weigh(const DecodeArgs& a, float* weight, int64_t weight_stride, cudaStream_t s) {
  int lanes = 1;
  while (lanes < 32 && lanes < a.Hq) lanes *= 2;
  const int64_t most = a.window > 0 && a.window < a.cache.capacity ? a.window : a.cache.capacity;
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int64_t room = (int64_t)di.sm_count * 8;
  // a block's keys: those that its lanes take at once, and more only where there are many
  int chunk = kWeighThreads / lanes * kSide;
  while (chunk < 4096 && (most + chunk - 1) / chunk * a.B > 4 * room) chunk *= 2;
  const int64_t chunks = (most + chunk - 1) / chunk, items = chunks * a.B;
  if (items == 0) return CP_OK;
  return cuda_status(launch_early(k_weigh, dim3((unsigned)(items < room ? items : room)), kWeighThreads, 0, s, a, weight,
                                  weight_stride, lanes, chunk, chunks, items),
                     "weigh");
}

}  // namespace cp
