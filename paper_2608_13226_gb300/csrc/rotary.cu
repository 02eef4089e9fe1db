// Rotary positions and the append of keys and values to a paged cache.
#include "rope.cuh"

namespace cp {

// One thread per pair of a row, and per component that passes through.
template <typename T>
__global__ void __launch_bounds__(256) k_rotary(RotaryArgs a) {
  const int per_row = a.D - a.rope.half;
  for (int n = 0; n < a.n; ++n) {
    const RowSet& x = a.set[n];
    const int64_t items = a.B * a.T * x.heads * per_row;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < items;
         i += (int64_t)gridDim.x * blockDim.x) {
      const int e = (int)(i % per_row);
      const int64_t row = i / per_row;
      const int h = (int)(row % x.heads);
      const int64_t tok = row / x.heads, t = tok % a.T, b = tok / a.T;
      const T* in = (const T*)x.in + b * x.in_b + t * x.in_t + h * x.in_h;
      T* out = (T*)x.out + b * x.out_b + t * x.out_t + h * x.out_h;
      if (e >= a.rope.half) {
        out[e + a.rope.half] = in[e + a.rope.half];
        continue;
      }
      float c, s;
      rope_unit(rope_turns(a.rope.inv_freq[e]), a.pos[b * a.pos_stride + t], a.rope, &c, &s);
      const int i0 = a.rope.interleaved ? 2 * e : e, i1 = a.rope.interleaved ? i0 + 1 : e + a.rope.half;
      const float u = to_f32(in[i0]), w = to_f32(in[i1]);
      out[i0] = from_f32<T>(u * c - w * s);
      out[i1] = from_f32<T>(w * c + u * s);
    }
  }
}

int launch_rotary(const RotaryArgs& a, int dtype, cudaStream_t s) {
  if (dtype == CP_BF16)
    k_rotary<__nv_bfloat16><<<608, 256, 0, s>>>(a);
  else
    k_rotary<float><<<608, 256, 0, s>>>(a);
  return last_launch_status();
}

// One block per token.
template <typename T, typename C>
__global__ void __launch_bounds__(128) k_cache_append(AppendArgs a) {
  const Cache& ch = a.cache;
  const int D = ch.D, half = a.rope.half, per_row = D - half;
  if (blockIdx.x == 0 && a.new_lens)
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
      const int64_t n = (int64_t)a.lens[b] + (a.starts ? a.starts[b + 1] - a.starts[b] : 1);
      a.new_lens[b] = (int32_t)min(n, (int64_t)ch.capacity);
    }
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    int b = (int)t, i = 0;
    if (a.starts) {
      b = 0;
      while (b < a.B && a.starts[b + 1] <= t) ++b;
      if (b == a.B) return;  // padding
      i = (int)(t - a.starts[b]);
    }
    const int64_t slot = (int64_t)a.lens[b] + i;
    const int64_t pos = a.pos ? a.pos[t] : slot;
    int page = -1;
    if (a.lens[b] >= 0 && slot < ch.capacity) page = ch.table[b * ch.table_stride + slot / ch.page_size];
    const bool fits = page >= 0 && page < ch.pages;
    if (!fits && threadIdx.x == 0 && a.status) set_status(a.status, CP_EINVAL);
    const int64_t row = fits ? page * ch.page_stride + slot % ch.page_size * ch.slot_stride : 0;
    const int rotated = a.q.heads + ch.heads;
    for (int i = threadIdx.x; i < rotated * per_row; i += blockDim.x) {
      const int e = i % per_row, h = i / per_row, hk = h - a.q.heads;
      const T* in = hk < 0 ? (const T*)a.q.in + t * a.q.in_t + h * a.q.in_h
                           : (const T*)a.k + t * a.k_t + hk * a.k_h;
      if (hk >= 0 && !fits) continue;
      auto put = [&](int at, float x) {
        if (hk < 0)
          ((T*)a.q.out)[t * a.q.out_t + h * a.q.out_h + at] = from_f32<T>(x);
        else
          ((C*)ch.k)[row + hk * ch.head_stride + at] =
              from_f32<C>(ch.k_scale ? x / ch.k_scale[hk] : x);
      };
      if (e >= half) {
        put(e + half, to_f32(in[e + half]));
        continue;
      }
      float c, s;
      rope_unit(rope_turns(a.rope.inv_freq[e]), pos, a.rope, &c, &s);
      const int i0 = a.rope.interleaved ? 2 * e : e, i1 = a.rope.interleaved ? i0 + 1 : e + half;
      const float u = to_f32(in[i0]), w = to_f32(in[i1]);
      put(i0, u * c - w * s);
      put(i1, w * c + u * s);
    }
    if (!fits) continue;
    for (int i = threadIdx.x; i < ch.heads * D; i += blockDim.x) {
      const int e = i % D, h = i / D;
      const float x = to_f32(((const T*)a.v)[t * a.v_t + h * a.v_h + e]);
      ((C*)ch.v)[row + h * ch.head_stride + e] = from_f32<C>(ch.v_scale ? x / ch.v_scale[h] : x);
    }
  }
}

int launch_cache_append(const AppendArgs& a, int dtype, int cache_dtype, cudaStream_t s) {
  const unsigned grid = (unsigned)(a.T < 1 ? 1 : a.T < 65536 ? a.T : 65536);
  if (cache_dtype == CP_F32)
    k_cache_append<float, float><<<grid, 128, 0, s>>>(a);
  else if (cache_dtype == CP_BF16)
    k_cache_append<__nv_bfloat16, __nv_bfloat16><<<grid, 128, 0, s>>>(a);
  else if (dtype == CP_F32)
    k_cache_append<float, __nv_fp8_e4m3><<<grid, 128, 0, s>>>(a);
  else
    k_cache_append<__nv_bfloat16, __nv_fp8_e4m3><<<grid, 128, 0, s>>>(a);
  return last_launch_status();
}

}  // namespace cp
