// The append to a 4-bit cache, and cached rows of any type read back.
//
// A row's 16 components share a scale: s = e4m3(min(max |x| / (7 h), 448)) with the head's
// factor h, and a component becomes n = round(x / (s h)), -7 to 7, held as n + 8.  Read
// back it is (n s) h.  Both calls read every element once and write it once: HBM
// bounds them.  A thread has 16 components of a row, a block some tokens: where their rows lie
// is looked up once a token, angles are computed once a token for all its heads.
// Nothing is staged: with 16 components (32 bytes of bfloat16, with their pairs' other halves 64)
// under way a thread, full SMs have 64 KB and more on their way.
#include <type_traits>

#include "rope.cuh"

namespace cp {

constexpr int kThreads = 256;
constexpr int kTokens = 8;  // of a block's turn, at most

// Where a token's rows lie: elements into the cache and bytes into its scales; there < 0: they are not.
struct Place {
  int64_t row, block;
  int there;  // 0; -1: no place, -2: padding
};

// The place of token t, of which sequence it is (starts NULL: t itself) and at which key.
__device__ __forceinline__ Place place_of(const Cache& ch, const int32_t* starts, const int32_t* lens, int B, int64_t t,
                                          int32_t* status, int64_t* key) {
  Place x{0, 0, -2};
  *key = 0;
  const int b = starts ? sequence_of(starts, B, t) : (int)t;
  const int64_t i = starts && b < B ? t - starts[b] : 0;  // below 0: before the first sequence's rows
  if (b >= B || i < 0) return x;
  const int len = lens[b];
  const int64_t slot = (int64_t)len + i;
  *key = slot;
  int page = -1;
  if (len >= 0 && slot >= 0 && slot < ch.capacity)
    page = ch.table[b * ch.table_stride + (uint32_t)slot / (uint32_t)ch.page_size];
  if (page >= 0 && page < ch.pages) {
    const int64_t r = (uint32_t)slot % (uint32_t)ch.page_size;
    x.row = page * ch.page_stride + r * ch.slot_stride;
    x.block = page * ch.block_page + r * ch.block_slot;
    x.there = 0;
  } else {
    x.there = -1;
    if (status) set_status(status, CP_EINVAL);
  }
  return x;
}

// N consecutive elements as float32; VEC: aligned to 16 bytes.
template <bool VEC, int N>
__device__ __forceinline__ void load_row(const float* p, float (&x)[N]) {
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 y = *reinterpret_cast<const float4*>(p + i);
      x[i] = y.x;
      x[i + 1] = y.y;
      x[i + 2] = y.z;
      x[i + 3] = y.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = p[i];
  }
}
template <bool VEC, int N>
__device__ __forceinline__ void load_row(const __nv_bfloat16* p, float (&x)[N]) {
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const uint4 y = *reinterpret_cast<const uint4*>(p + i);
      const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i + 2 * j] = __uint_as_float(w[j] << 16);
        x[i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __bfloat162float(p[i]);
  }
}
template <bool VEC, int N>
__device__ __forceinline__ void store_row(float* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    if constexpr (VEC) {
      *reinterpret_cast<float4*>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) p[i + j] = x[i + j];
    }
  }
}
template <bool VEC, int N>
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    if constexpr (VEC) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(x[i + 2 * j + 1]), "f"(x[i + 2 * j]));
      *reinterpret_cast<uint4*>(p + i) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[i + j] = __float2bfloat16_rn(x[i + j]);
    }
  }
}

// 16 components to 4 bits each and their scale's byte.
__device__ __forceinline__ uint2 to_fours(const float (&x)[16], float head, uint8_t* scale) {
  uint32_t top = 0;  // the largest size, a NaN above all numbers
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  const __nv_fp8_e4m3 s = from_f32<__nv_fp8_e4m3>(__fdiv_rn(__uint_as_float(top), __fmul_rn(7.0f, head)));
  *scale = s.__x;
  const float step = __fmul_rn((float)s, head);
  uint32_t w[2] = {};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float n = step == 0.0f ? 0.0f : fminf(fmaxf(rintf(__fdiv_rn(x[i], step)), -7.0f), 7.0f);
    w[i / 8] |= (uint32_t)((int)n + 8) << 4 * (i % 8);
  }
  return make_uint2(w[0], w[1]);
}

// 16 components from d0 on turned by interleaved pairs.
__device__ __forceinline__ void turn_neighbours(const Rope& r, int d0, float (&x)[16], const float* co, const float* si) {
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    const int p = (d0 + j) / 2;
    if (p < r.half) {
      const float u = x[j], w = x[j + 1];
      x[j] = fmaf(w, -si[p], __fmul_rn(u, co[p]));
      x[j + 1] = fmaf(u, si[p], __fmul_rn(w, co[p]));
    }
  }
}

// A piece of a query's row turned: 8 pairs of the half layout, or 16 components side by side, so that no
// thread reads what another writes where the result goes to the query's own place.
__device__ __forceinline__ int query_pieces(const Rope& r, int D) {
  return r.interleaved ? D / 16 : (r.half + 7) / 8 + (D - 2 * r.half + 15) / 16;
}
template <typename T, bool VEC>
__device__ __forceinline__ void turn_query(const Rope& r, int D, const T* in, T* out, int piece, const float* co, const float* si) {
  const int apart = r.interleaved ? 0 : (r.half + 7) / 8;
  if (piece < apart) {
    const int p = 8 * piece, n = VEC ? 8 : min(8, r.half - p);  // VEC: half is a multiple of 8
    float u[8] = {}, w[8] = {};
    if constexpr (VEC) {
      load_row<true>(in + p, u);
      load_row<true>(in + r.half + p, w);
    } else {
      for (int j = 0; j < n; ++j) {
        u[j] = (float)in[p + j];
        w[j] = (float)in[r.half + p + j];
      }
    }
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = VEC ? p + j : min(p + j, r.half - 1);
      x[j] = fmaf(w[j], -si[at], __fmul_rn(u[j], co[at]));
      y[j] = fmaf(u[j], si[at], __fmul_rn(w[j], co[at]));
    }
    if constexpr (VEC) {
      store_row<true>(out + p, x);
      store_row<true>(out + r.half + p, y);
    } else {
      for (int j = 0; j < n; ++j) {
        out[p + j] = from_f32<T>(x[j]);
        out[r.half + p + j] = from_f32<T>(y[j]);
      }
    }
    return;
  }
  const int d0 = (r.interleaved ? 0 : 2 * r.half) + 16 * (piece - apart);
  if (!VEC && D - d0 < 16) {  // what passes
    for (int d = d0; d < D; ++d) out[d] = in[d];
    return;
  }
  float x[16];
  load_row<VEC>(in + d0, x);
  if (r.interleaved) turn_neighbours(r, d0, x, co, si);
  store_row<VEC>(out + d0, x);
}

// VEC: rows come in vectors of 16 bytes, and so do the halves that pairs lie apart.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_append_fours(AppendArgs a, int tokens) {
  extern __shared__ __align__(16) char smem[];  // angles and speeds
  __shared__ Place s_place[kTokens];
  __shared__ int64_t s_pos[kTokens];
  wait_for_stream();
  const Cache& ch = a.cache;
  const int half = a.rope.half;
  float* s_cos = reinterpret_cast<float*>(smem);
  float* s_sin = s_cos + tokens * half;
  uint64_t* s_turns = reinterpret_cast<uint64_t*>(s_sin + tokens * half);
  if (a.new_lens)
    for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < a.B; b += (int64_t)gridDim.x * kThreads) {
      const int len = a.lens[b];
      const int64_t n = (int64_t)len + (a.starts ? (int64_t)a.starts[b + 1] - a.starts[b] : 1);
      a.new_lens[b] = len < 0 ? len : (int32_t)min(n, (int64_t)ch.capacity);
    }
  for (int i = threadIdx.x; i < half; i += kThreads) s_turns[i] = rope_turns(a.rope.inv_freq[i]);
  const int per_query = a.q.heads > 0 ? query_pieces(a.rope, ch.D) : 1, per_row = ch.D / 16;
  const int queries = a.q.heads * per_query, per_token = queries + 2 * ch.heads * per_row;
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < a.T; t0 += (int64_t)gridDim.x * tokens) {
    const int n = (int)min((int64_t)tokens, a.T - t0);
    __syncthreads();  // the tokens before are done with
    if (threadIdx.x < n) {
      int64_t key;
      s_place[threadIdx.x] = place_of(ch, a.starts, a.lens, a.B, t0 + threadIdx.x, a.status, &key);
      s_pos[threadIdx.x] = a.pos ? a.pos[t0 + threadIdx.x] : key;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * half; i += kThreads)
      rope_unit(s_turns[i % half], s_pos[i / half], a.rope, s_cos + i, s_sin + i);
    if (half > 0) __syncthreads();
    for (int i = threadIdx.x; i < n * per_token; i += kThreads) {
      const int tok = i / per_token;
      int r = i - tok * per_token;
      const Place at = s_place[tok];
      const int64_t t = t0 + tok;
      const float* co = s_cos + tok * half;
      const float* si = s_sin + tok * half;
      if (r < queries) {
        if (at.there == -2) continue;
        const int h = r / per_query;
        turn_query<T, VEC>(a.rope, ch.D, (const T*)a.q.in + t * a.q.in_t + h * a.q.in_h,
                           (T*)a.q.out + t * a.q.out_t + h * a.q.out_h, r - h * per_query, co, si);
        continue;
      }
      if (at.there < 0) continue;
      r -= queries;
      int h = r / per_row;
      const int d0 = 16 * (r - h * per_row);
      const bool key = h < ch.heads;
      if (!key) h -= ch.heads;
      const T* in = key ? (const T*)a.k + t * a.k_t + h * a.k_h : (const T*)a.v + t * a.v_t + h * a.v_h;
      float x[16];
      load_row<VEC>(in + d0, x);
      if (key && d0 < 2 * half) {
        if (a.rope.interleaved) {
          turn_neighbours(a.rope, d0, x, co, si);
        } else if constexpr (VEC) {  // half is a multiple of 8
#pragma unroll
          for (int g = 0; g < 16; g += 8) {
            const int d = d0 + g;
            if (d < 2 * half) {
              const bool front = d < half;
              const int p = front ? d : d - half;
              float y[8];
              load_row<true>(in + (front ? d + half : d - half), y);
#pragma unroll
              for (int j = 0; j < 8; ++j)
                x[g + j] = fmaf(y[j], front ? -si[p + j] : si[p + j], __fmul_rn(x[g + j], co[p + j]));
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int d = d0 + j;
            if (d < 2 * half) {
              const bool front = d < half;
              const int p = front ? d : d - half;
              const float y = (float)in[front ? d + half : d - half];
              x[j] = fmaf(y, front ? -si[p] : si[p], __fmul_rn(x[j], co[p]));
            }
          }
        }
      }
      const float* scales = key ? ch.k_scale : ch.v_scale;
      uint8_t s;
      const uint2 w = to_fours(x, scales ? scales[h] : 1.0f, &s);
      *reinterpret_cast<uint2*>((char*)(key ? ch.k : ch.v) + (at.row + h * ch.head_stride + d0) / 2) = w;
      uint8_t* to = (key ? ch.k_block : ch.v_block) + at.block + h * ch.block_head + d0 / 16;
      *to = s;
      if (d0 + 16 >= ch.D)  // the padding
        for (int j = d0 / 16 + 1; j < block_bytes(ch.D); ++j) *++to = 0;
    }
  }
}

template <typename T, bool VEC>
static int append_fours(const AppendArgs& a, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int64_t room = (int64_t)di.sm_count * 8;
  int tokens = 1;
  while (tokens < kTokens && tokens * room < a.T) tokens *= 2;
  const int64_t turns = (a.T + tokens - 1) / tokens;
  const size_t smem = (size_t)a.rope.half * (8 * (size_t)tokens + 8);
  return cuda_status(launch_early(k_append_fours<T, VEC>, dim3((unsigned)(turns < 1 ? 1 : turns < room ? turns : room)), kThreads,
                                  smem, s, a, tokens),
                     "cache append, 4 bits");
}

static bool vectors(const void* p, int64_t t, int64_t h, size_t e) {
  return (uintptr_t)p % 16 == 0 && t * (int64_t)e % 16 == 0 && h * (int64_t)e % 16 == 0;
}
template <typename T>
static int append_fours_of(const AppendArgs& a, cudaStream_t s) {
  const size_t e = sizeof(T);
  const bool vec = vectors(a.k, a.k_t, a.k_h, e) && vectors(a.v, a.v_t, a.v_h, e) && (a.rope.interleaved || a.rope.half % 8 == 0) &&
                   (a.q.heads == 0 || (vectors(a.q.in, a.q.in_t, a.q.in_h, e) && vectors(a.q.out, a.q.out_t, a.q.out_h, e)));
  return vec ? append_fours<T, true>(a, s) : append_fours<T, false>(a, s);
}
int launch_append_fours(const AppendArgs& a, int dtype, cudaStream_t s) {
  return dtype == CP_F32 ? append_fours_of<float>(a, s) : append_fours_of<__nv_bfloat16>(a, s);
}

// 16 cached components from `at` on (8 where a row has no more), as their element says, in float32.
template <int CT>
__device__ __forceinline__ void load_cached(const void* cache, int64_t at, uint8_t scale, float (&x)[16], bool whole) {
  if constexpr (CT == CP_I4) {
    const uint2 y = *reinterpret_cast<const uint2*>((const char*)cache + at / 2);
    __nv_fp8_e4m3 s;
    s.__x = scale;
    const float f = (float)s;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __fmul_rn((float)((int)((i < 8 ? y.x : y.y) >> 4 * (i % 8) & 15) - 8), f);
  } else if constexpr (CT == CP_E4M3) {
    const uint4 y = *reinterpret_cast<const uint4*>((const char*)cache + at);
    const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      __nv_fp8_e4m3 s;
      s.__x = (uint8_t)(w[i / 4] >> 8 * (i % 4));
      x[i] = (float)s;
    }
  } else {
    using C = typename std::conditional<CT == CP_F32, float, __nv_bfloat16>::type;
    float y[8] = {};
    load_row<true>((const C*)cache + at, *reinterpret_cast<float(*)[8]>(&x[0]));
    if (whole) load_row<true>((const C*)cache + at + 8, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[8 + i] = y[i];
  }
}

template <int CT, typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) k_cache_read(ReadArgs a, int tokens) {
  __shared__ Place s_place[kTokens];
  wait_for_stream();
  const Cache& ch = a.cache;
  const int per_row = (ch.D + 15) / 16, per_token = 2 * ch.heads * per_row;
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < a.T; t0 += (int64_t)gridDim.x * tokens) {
    const int n = (int)min((int64_t)tokens, a.T - t0);
    __syncthreads();
    int64_t key;
    if (threadIdx.x < n) s_place[threadIdx.x] = place_of(ch, a.starts, a.lens, a.B, t0 + threadIdx.x, a.status, &key);
    __syncthreads();
    for (int i = threadIdx.x; i < n * per_token; i += kThreads) {
      const int tok = i / per_token, r = (i - tok * per_token) / per_row, d0 = 16 * (i - tok * per_token - r * per_row);
      const Place at = s_place[tok];
      const bool key = r < ch.heads;
      const int h = key ? r : r - ch.heads;
      if (at.there == -2) continue;
      float x[16] = {};
      const int there = ch.D - d0;  // a multiple of 4
      if (at.there == 0) {
        const int64_t e = at.row + h * ch.head_stride + d0;
        const void* from = key ? ch.k : ch.v;
        if (CT == CP_F32 && there < 16) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j < there) x[j] = ((const float*)from)[e + j];
        } else {
          uint8_t s = 0;
          if (CT == CP_I4) s = (key ? ch.k_block : ch.v_block)[at.block + h * ch.block_head + d0 / 16];
          load_cached<CT>(from, e, s, x, there >= 16);
        }
        const float* scales = key ? ch.k_scale : ch.v_scale;
        if (scales) {
          const float f = scales[h];
#pragma unroll
          for (int j = 0; j < 16; ++j) x[j] = __fmul_rn(x[j], f);
        }
      }
      T* out = key ? (T*)a.k + (t0 + tok) * a.k_t + h * a.k_h + d0 : (T*)a.v + (t0 + tok) * a.v_t + h * a.v_h + d0;
      if (there >= 16) {
        store_row<VEC>(out, x);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (j < there) out[j] = from_f32<T>(x[j]);
      }
    }
  }
}

template <int CT, typename T, bool VEC>
static int cache_read(const ReadArgs& a, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int64_t room = (int64_t)di.sm_count * 8;
  int tokens = 1;
  while (tokens < kTokens && tokens * room < a.T) tokens *= 2;
  const int64_t turns = (a.T + tokens - 1) / tokens;
  return cuda_status(launch_early(k_cache_read<CT, T, VEC>, dim3((unsigned)(turns < room ? turns : room)), kThreads, 0, s, a, tokens),
                     "cache read");
}
template <int CT, typename T>
static int cache_read_of(const ReadArgs& a, cudaStream_t s) {
  const bool vec = vectors(a.k, a.k_t, a.k_h, sizeof(T)) && vectors(a.v, a.v_t, a.v_h, sizeof(T));
  return vec ? cache_read<CT, T, true>(a, s) : cache_read<CT, T, false>(a, s);
}
int launch_cache_read(const ReadArgs& a, int dtype, int cache_dtype, cudaStream_t s) {
  const bool wide = dtype == CP_F32;
  if (cache_dtype == CP_F32) return cache_read_of<CP_F32, float>(a, s);
  if (cache_dtype == CP_BF16) return cache_read_of<CP_BF16, __nv_bfloat16>(a, s);
  if (cache_dtype == CP_E4M3) return wide ? cache_read_of<CP_E4M3, float>(a, s) : cache_read_of<CP_E4M3, __nv_bfloat16>(a, s);
  return wide ? cache_read_of<CP_I4, float>(a, s) : cache_read_of<CP_I4, __nv_bfloat16>(a, s);
}

}  // namespace cp
