// Attention of one query a sequence over a paged cache.
#include "rope.cuh"

namespace cp {

constexpr int kTile = 128;

// A block per query head: tiles of 128 keys, a running maximum and sum.
template <typename T, typename C>
__global__ void __launch_bounds__(kTile) k_decode(DecodeArgs a) {
  const Cache& ch = a.cache;
  const int b = blockIdx.y, h = blockIdx.x, hk = h / (a.Hq / ch.heads), D = ch.D, tid = threadIdx.x;
  __shared__ float q[256], p[kTile], red[4];
  __shared__ int64_t at[kTile];
  for (int d = tid; d < D; d += kTile) q[d] = to_f32(((const T*)a.q)[b * a.q_b + h * a.q_h + d]);
  const int len = min(max(a.lens[b], 0), ch.capacity);
  const int first = a.window > 0 && a.window < len ? len - (int)a.window : 0;
  const float scale = a.scale * (ch.k_scale ? ch.k_scale[hk] : 1.0f);
  float m = -INFINITY, l = 0.0f, o[2] = {0.0f, 0.0f};
  for (int j0 = first; j0 < len; j0 += kTile) {
    const int j = j0 + tid;
    float x = -INFINITY;
    int64_t row = -1;
    if (j < len && (!a.keep || a.keep[b * a.keep_stride + j])) {
      const int page = ch.table[b * ch.table_stride + j / ch.page_size];
      if (page < 0 || page >= ch.pages) {
        if (a.status) set_status(a.status, CP_EINVAL);
      } else {
        row = page * ch.page_stride + j % ch.page_size * ch.slot_stride + hk * ch.head_stride;
      }
    }
    __syncthreads();
    if (row >= 0) {
      x = 0.0f;
      for (int d = 0; d < D; ++d) x += q[d] * to_f32(((const C*)ch.k)[row + d]);
      x *= scale;
    }
    float top = x;
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (tid % 32 == 0) red[tid / 32] = top;
    at[tid] = row;
    __syncthreads();
    top = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
    const float base = top == -INFINITY ? 0.0f : top, f = expf(m - base);
    p[tid] = row >= 0 ? expf(x - base) : 0.0f;
    m = top;
    l *= f;
    o[0] *= f;
    o[1] *= f;
    __syncthreads();
    for (int i = 0; i < kTile; ++i) {
      if (at[i] < 0) continue;
      l += p[i];
      for (int n = 0; n < 2; ++n)
        if (tid + n * kTile < D) o[n] += p[i] * to_f32(((const C*)ch.v)[at[i] + tid + n * kTile]);
    }
  }
  const float inv = l == 0.0f ? 0.0f : (ch.v_scale ? ch.v_scale[hk] : 1.0f) / l;
  for (int n = 0; n < 2; ++n)
    if (tid + n * kTile < D)
      ((T*)a.out)[b * a.o_b + h * a.o_h + tid + n * kTile] = from_f32<T>(o[n] * inv);
  if (a.lse && tid == 0) a.lse[(int64_t)b * a.Hq + h] = l == 0.0f ? -INFINITY : logf(l) + m;
}

size_t decode_ws_bytes(int64_t, int64_t, int64_t, int64_t, int) { return 256; }

int launch_decode(const DecodeArgs& a, int cache_dtype, cudaStream_t s) {
  const dim3 grid(a.Hq, a.B);
  if (cache_dtype == CP_F32)
    k_decode<float, float><<<grid, kTile, 0, s>>>(a);
  else if (cache_dtype == CP_BF16)
    k_decode<__nv_bfloat16, __nv_bfloat16><<<grid, kTile, 0, s>>>(a);
  else
    k_decode<__nv_bfloat16, __nv_fp8_e4m3><<<grid, kTile, 0, s>>>(a);
  return last_launch_status();
}

}  // namespace cp
