// The append to a 4-bit cache, and cached rows of any type read back.
//
// A row's 16 components share a scale: s = e4m3(min(max |x| / (7 h), 448)) with the head's
// factor h, and a component becomes n = round(x / (s h)), -7 to 7, held as n + 8.  Read
// back it is (n s) h.  Both calls read every element once and write it once: HBM
// bounds them.  A thread has 16 components of a row, a block some tokens: where their rows lie
// is looked up once a token, angles are computed once a token for all its heads.
// Nothing is staged: with 16 components (32 bytes of bfloat16, with their pairs' other halves 64)
// under way a thread, full SMs have 64 KB and more on their way.
#include <cuda_fp16.h>

#include "rope.cuh"

namespace cp {

constexpr int kThreads = 256;
constexpr int kTokens = 64;  // of a block's turn, at most

// Where a token's rows lie: elements into the cache and bytes into its scales; there < 0: they are not.
struct Place {
  int64_t row, block;
  int there;  // 0; -1: no place, -2: padding
};

// How many of starts[1..B] are <= t, by a warp: few of them are counted at once, of many a binary search ends.
__device__ __forceinline__ int sequence_by_warp(const int32_t* starts, int B, int64_t t) {
  if (B > 256) return sequence_of(starts, B, t);
  int n = 0;
  for (int b = threadIdx.x % 32; b < B; b += 32) n += starts[1 + b] <= t;
  return __reduce_add_sync(~0u, n);
}

// The places of tokens t0 to t0 + n - 1, a thread each (whole warps come here): which sequence each is of (starts NULL:
// it by itself), at which key.
__device__ __forceinline__ void find_places(const Cache& ch, const int32_t* starts, const int32_t* lens, int B, int64_t t0, int n,
                                            int32_t* status, Place* places, int64_t* keys) {
  const int i0 = threadIdx.x / 32 * 32;  // the warp's first
  if (i0 >= n) return;
  const int64_t t = t0 + threadIdx.x;
  int b = (int)min(t, (int64_t)B);
  if (starts) {  // between those of the warp's first token and of its last
    const int lo = sequence_by_warp(starts, B, t0 + i0), hi = sequence_by_warp(starts, B, t0 + min(i0 + 31, n - 1));
    b = lo + sequence_of(starts + lo, hi - lo, t);
  }
  if ((int)threadIdx.x >= n) return;
  Place x{0, 0, -2};
  int64_t key = 0;
  const int64_t at = starts && b < B ? t - starts[b] : 0;  // below 0: before the first sequence's rows
  if (b < B && at >= 0) {
    const int len = lens[b];
    key = (int64_t)len + at;
    int page = -1;
    if (len >= 0 && key >= 0 && key < ch.capacity)
      page = ch.table[b * ch.table_stride + (uint32_t)key / (uint32_t)ch.page_size];
    if (page >= 0 && page < ch.pages) {
      const int64_t r = (uint32_t)key % (uint32_t)ch.page_size;
      x.row = page * ch.page_stride + r * ch.slot_stride;
      x.block = page * ch.block_page + r * ch.block_slot;
      x.there = 0;
    } else {
      x.there = -1;
      if (status) set_status(status, CP_EINVAL);
    }
  }
  places[threadIdx.x] = x;
  if (keys) keys[threadIdx.x] = key;
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

// Four consecutive elements, aligned to as many bytes as they have.
__device__ __forceinline__ void load_quad(const float* p, float (&x)[4]) { load_row<true>(p, x); }
__device__ __forceinline__ void load_quad(const __nv_bfloat16* p, float (&x)[4]) {
  const uint2 y = *reinterpret_cast<const uint2*>(p);
  x[0] = __uint_as_float(y.x << 16);
  x[1] = __uint_as_float(y.x & 0xFFFF0000u);
  x[2] = __uint_as_float(y.y << 16);
  x[3] = __uint_as_float(y.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store_quad(float* p, const float (&x)[4]) { store_row<true>(p, x); }
__device__ __forceinline__ void store_quad(__nv_bfloat16* p, const float (&x)[4]) {
  uint32_t w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(x[2 * j + 1]), "f"(x[2 * j]));
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

__device__ __forceinline__ float max_nan(float a, float b) {  // a NaN is above all numbers
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// 16 components to 4 bits each and their scale's byte.
__device__ __forceinline__ uint2 to_fours(const float (&x)[16], float head, uint8_t* scale) {
  float top = fabsf(x[0]);
#pragma unroll
  for (int i = 1; i < 16; ++i) top = max_nan(top, fabsf(x[i]));
  const float want = __fdiv_rn(top, __fmul_rn(7.0f, head));
  const __nv_fp8_e4m3 s = from_f32<__nv_fp8_e4m3>(want);
  *scale = s.__x;
  const float step = __fmul_rn((float)s, head);
  uint32_t w[2] = {};
  // Quotients rounded as a division rounds them: with r = 1 / step rounded to nearest and q within a unit in the last
  // place of x / step, q + (x - q step) r rounds to the quotient (Markstein 1990, Computation of elementary functions on
  // the IBM RISC System/6000).  x r alone may be two units off, and once corrected is within one.  That within ranges
  // where nothing that counts under- or overflows, and where the scale is a normal number, so that no quotient is
  // above 7 (1 + 2^-4).  Else divisions.  38,400 tokens of 2 x 4 heads of 128 26.6 us, by divisions alone 46.8.
  if (want >= 0.015625f && want <= 448.0f && step > 1e-15f && step < 1e15f) {
    const float r = __frcp_rn(step);
    const uint64_t r2 = pair(r, r), less = pair(-step, -step), magic = pair(12582920.0f, 12582920.0f);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // a number's bits end in n + 8 once 1.5 2^23 + 8 is added, which rounds it to nearest even; what is
      // above them adds up to a constant
      uint32_t all = 0, above = 0;
#pragma unroll
      for (int i = 6; i >= 0; i -= 2) {
        const uint64_t v = pair(x[8 * h + i], x[8 * h + i + 1]);
        uint64_t y = mul2(v, r2);
        y = fma2(fma2(y, less, v), r2, y);
        y = fma2(fma2(y, less, v), r2, y);
        y = add2(y, magic);
        all = (all * 16 + (uint32_t)(y >> 32)) * 16 + (uint32_t)y;
        above = (above * 16 + 0x4B400000u) * 16 + 0x4B400000u;
      }
      w[h] = all - above;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float n = step == 0.0f ? 0.0f : fminf(fmaxf(rintf(__fdiv_rn(x[i], step)), -7.0f), 7.0f);
      w[i / 8] |= (uint32_t)((int)n + 8) << 4 * (i % 8);
    }
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
__host__ __device__ __forceinline__ int query_pieces(const Rope& r, int D) {
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

// The same for rows in vectors of 16 bytes, with halves of the layout that are not vectors apart: pairs go four by four where
// that divides them, and of what passes 16 components from a multiple of 16 on, but for the first.
// (38,400 tokens of 28 + 2 x 4 heads of 96 with 24 turned 154 us, one by one 675.)
template <typename T>
__device__ __forceinline__ void turn_query_apart(const Rope& r, const T* in, T* out, int piece, const float* co, const float* si) {
  const int apart = (r.half + 7) / 8;
  if (piece < apart) {
    const int p = 8 * piece, n = min(8, r.half - p);
    if (r.half % 4 == 0) {
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        if (i < n) {
          const int at = p + i;
          float u[4], w[4], x[4], y[4];
          load_quad(in + at, u);
          load_quad(in + r.half + at, w);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] = fmaf(w[j], -si[at + j], __fmul_rn(u[j], co[at + j]));
            y[j] = fmaf(u[j], si[at + j], __fmul_rn(w[j], co[at + j]));
          }
          store_quad(out + at, x);
          store_quad(out + r.half + at, y);
        }
      }
    } else {
      for (int j = p; j < p + n; ++j) {
        const float u = (float)in[j], w = (float)in[r.half + j];
        out[j] = from_f32<T>(fmaf(w, -si[j], __fmul_rn(u, co[j])));
        out[r.half + j] = from_f32<T>(fmaf(u, si[j], __fmul_rn(w, co[j])));
      }
    }
    return;
  }
  const int d0 = 16 * (r.half / 8 + piece - apart);
  if (d0 < 2 * r.half) {  // a part of it passes
    if (r.half % 2 == 0) {
      for (int d = 2 * r.half; d < d0 + 16; d += 4) {
        float x[4];
        load_quad(in + d, x);
        store_quad(out + d, x);
      }
    } else {
      for (int d = 2 * r.half; d < d0 + 16; ++d) out[d] = in[d];
    }
    return;
  }
  float x[16];
  load_row<true>(in + d0, x);
  store_row<true>(out + d0, x);
}

// How a block's threads share the items of one kind of a turn's tokens: `width` of a token's `count` side by side, and so
// `side` tokens; items beyond `width` in further rounds.  What an item is, a thread works out once a round.
struct Share {
  int count, per_row;  // items of a token, of a row
  int width, side;
};
static Share share_of(int rows, int per_row) {
  Share x;
  x.count = rows * per_row;
  x.per_row = per_row;
  const int rounds = x.count < 1 ? 1 : (x.count + kThreads - 1) / kThreads;
  x.width = x.count < 1 ? 1 : (x.count + rounds - 1) / rounds;
  x.side = kThreads / x.width;
  return x;
}
// Tokens of a turn: few go to as many blocks as there is room for.
static int tokens_of(int64_t T, int sms) {
  int n = 1;
  while (n < kTokens && n * (int64_t)sms * 4 < T) n *= 2;
  return n;
}
// body(item, first, step): the tokens first, first + step, .. of an item.
template <typename F>
__device__ __forceinline__ void each_item(const Share& x, F body) {
  const int first = threadIdx.x / x.width;
  if (first < x.side)
    for (int r = threadIdx.x - first * x.width; r < x.count; r += x.width) body(r, first, x.side);
}

// VEC: rows come in vectors of 16 bytes.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) k_append_fours(AppendArgs a, int tokens, Share queries, Share rows, Divisor by_half) {
  extern __shared__ __align__(16) char smem[];  // angles and speeds
  __shared__ Place s_place[kTokens];
  __shared__ int64_t s_pos[kTokens];
  wait_for_stream();
  const Cache& ch = a.cache;
  const int half = a.rope.half;
  const bool even = half % 8 == 0;  // a pair's halves are vectors apart
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
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < a.T; t0 += (int64_t)gridDim.x * tokens) {
    const int n = (int)min((int64_t)tokens, a.T - t0);
    __syncthreads();  // the tokens before are done with
    find_places(ch, a.starts, a.lens, a.B, t0, n, a.status, s_place, a.pos ? nullptr : s_pos);
    if (a.pos && threadIdx.x < n) s_pos[threadIdx.x] = a.pos[t0 + threadIdx.x];
    __syncthreads();
    for (int i = threadIdx.x; i < n * half; i += kThreads)
      rope_unit(s_turns[i - by_half.of(i) * half], s_pos[by_half.of(i)], a.rope, s_cos + i, s_sin + i);
    if (half > 0) __syncthreads();
    // 16 components from d0 on of head h's key or value
    each_item(rows, [&](int r, int first, int step) {
      int h = r / rows.per_row;
      const int d0 = 16 * (r - h * rows.per_row);
      const bool key = h < ch.heads;
      if (!key) h -= ch.heads;
      const T* row0 = (key ? (const T*)a.k + h * a.k_h : (const T*)a.v + h * a.v_h) + d0;
      const int64_t apart = key ? a.k_t : a.v_t;
      const float* scales = key ? ch.k_scale : ch.v_scale;
      const float head = scales ? scales[h] : 1.0f;
      char* codes = (char*)(key ? ch.k : ch.v) + (h * ch.head_stride + d0) / 2;
      uint8_t* blocks = (key ? ch.k_block : ch.v_block) + h * ch.block_head + d0 / 16;
      const bool turns = key && d0 < 2 * half;
#pragma unroll 1
      for (int tok = first; tok < n; tok += step) {
        const T* in = row0 + (t0 + tok) * apart;
        float x[16];
        load_row<VEC>(in, x);
        const Place at = s_place[tok];
        if (at.there < 0) continue;
        if (turns) {
          const float* co = s_cos + tok * half;
          const float* si = s_sin + tok * half;
          if (a.rope.interleaved) {
            turn_neighbours(a.rope, d0, x, co, si);
          } else if (VEC && even) {
#pragma unroll
            for (int g = 0; g < 16; g += 8) {
              const int d = d0 + g;
              if (d < 2 * half) {
                const bool front = d < half;
                const int p = front ? d : d - half;
                float y[8];
                load_row<true>(in + g + (front ? half : -half), y);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  x[g + j] = fmaf(y[j], front ? -si[p + j] : si[p + j], __fmul_rn(x[g + j], co[p + j]));
              }
            }
          } else if (VEC && half % 4 == 0) {
#pragma unroll
            for (int g = 0; g < 16; g += 4) {
              const int d = d0 + g;
              if (d < 2 * half) {
                const bool front = d < half;
                const int p = front ? d : d - half;
                float y[4];
                load_quad(in + g + (front ? half : -half), y);
#pragma unroll
                for (int j = 0; j < 4; ++j)
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
                const float y = (float)in[j + (front ? half : -half)];
                x[j] = fmaf(y, front ? -si[p] : si[p], __fmul_rn(x[j], co[p]));
              }
            }
          }
        }
        uint8_t s;
        const uint2 w = to_fours(x, head, &s);
        *reinterpret_cast<uint2*>(codes + at.row / 2) = w;
        uint8_t* to = blocks + at.block;
        *to = s;
        if (d0 + 16 >= ch.D)  // the padding
          for (int j = d0 / 16 + 1; j < block_bytes(ch.D); ++j) *++to = 0;
      }
    });
    each_item(queries, [&](int r, int first, int step) {
      const int h = r / queries.per_row, piece = r - h * queries.per_row;
      const T* in = (const T*)a.q.in + h * a.q.in_h;
      T* out = (T*)a.q.out + h * a.q.out_h;
#pragma unroll 1
      for (int tok = first; tok < n; tok += step) {
        if (s_place[tok].there == -2) continue;
        const int64_t t = t0 + tok;
        if (VEC && !even && !a.rope.interleaved)
          turn_query_apart(a.rope, in + t * a.q.in_t, out + t * a.q.out_t, piece, s_cos + tok * half, s_sin + tok * half);
        else
          turn_query<T, VEC>(a.rope, ch.D, in + t * a.q.in_t, out + t * a.q.out_t, piece, s_cos + tok * half, s_sin + tok * half);
      }
    });
  }
}

template <typename T, bool VEC>
static int append_fours(const AppendArgs& a, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int64_t room = (int64_t)di.sm_count * 8;
  const int tokens = tokens_of(a.T, di.sm_count);
  const int64_t turns = (a.T + tokens - 1) / tokens;
  const size_t smem = (size_t)a.rope.half * (8 * (size_t)tokens + 8);
  static std::atomic<uint64_t> allowed{0};
  CP_TRY_STATUS(allow_smem_once((const void*)k_append_fours<T, VEC>, 128 * (8 * kTokens + 8), "cache append: shared memory", &allowed));
  return cuda_status(launch_early(k_append_fours<T, VEC>, dim3((unsigned)(turns < 1 ? 1 : turns < room ? turns : room)), kThreads,
                                  smem, s, a, tokens, share_of(a.q.heads, query_pieces(a.rope, a.cache.D)),
                                  share_of(2 * a.cache.heads, a.cache.D / 16), divisor(a.rope.half)),
                     "cache append, 4 bits");
}

static bool vectors(const void* p, int64_t t, int64_t h, size_t e, int bytes = 16) {
  return (uintptr_t)p % bytes == 0 && t * (int64_t)e % bytes == 0 && h * (int64_t)e % bytes == 0;
}
template <typename T>
static int append_fours_of(const AppendArgs& a, cudaStream_t s) {
  const size_t e = sizeof(T);
  const bool vec = vectors(a.k, a.k_t, a.k_h, e) && vectors(a.v, a.v_t, a.v_h, e) &&
                   (a.q.heads == 0 || (vectors(a.q.in, a.q.in_t, a.q.in_h, e) && vectors(a.q.out, a.q.out_t, a.q.out_h, e)));
  return vec ? append_fours<T, true>(a, s) : append_fours<T, false>(a, s);
}
int launch_append_fours(const AppendArgs& a, int dtype, cudaStream_t s) {
  return dtype == CP_F32 ? append_fours_of<float>(a, s) : append_fours_of<__nv_bfloat16>(a, s);
}

// The same 16 components at a multiple of 32 bytes, which a thread stores whole: by 16 bytes, a warp's stores would fill
// half of every sector that they touch.
__device__ __forceinline__ void store_wide(__nv_bfloat16* p, const float (&x)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(x[2 * j + 1]), "f"(x[2 * j]));
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void store_wide(float* p, const float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + i), "r"(__float_as_uint(x[i])),
                 "r"(__float_as_uint(x[i + 1])), "r"(__float_as_uint(x[i + 2])), "r"(__float_as_uint(x[i + 3])),
                 "r"(__float_as_uint(x[i + 4])), "r"(__float_as_uint(x[i + 5])), "r"(__float_as_uint(x[i + 6])),
                 "r"(__float_as_uint(x[i + 7]))
                 : "memory");
}

// 16 cached components (8 where a row has no more), as they come.
template <int CT>
struct Held {
  static constexpr int kVecs = CT == CP_F32 ? 4 : CT == CP_BF16 ? 2 : 1;
  uint4 v[kVecs];
  uint8_t scale;
  // `there` of them; a row of float32 may end after 4, 8 or 12
  __device__ __forceinline__ void load(const char* p, const uint8_t* block, int there) {
    if constexpr (CT == CP_I4) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      v[0] = make_uint4(x.x, x.y, 0, 0);
      scale = *block;
    } else {
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        if (i * (16 / kVecs) < there) v[i] = reinterpret_cast<const uint4*>(p)[i];
    }
  }
  __device__ __forceinline__ void floats(float (&x)[16]) const {
    if constexpr (CT == CP_I4) {
      // Two numbers of a word at a time, four places apart: with bits 4-7 of a half 64 + n + 8 is a float16 as it is,
      // and (72 + n) s - 72 s rounds once to what float16 holds exactly.
      __nv_fp8_e4m3 s;
      s.__x = scale;
      const __half2 f = __half2half2(__half((float)s)), off = __hmul2(f, __half2half2(__half(-72.0f)));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t w = h ? v[0].y : v[0].x;
        const uint32_t at[4] = {w << 4, w, w >> 4, w >> 8};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bits = (at[i] & 0x00F000F0u) | 0x54005400u;
          const float2 y = __half22float2(__hfma2(*reinterpret_cast<const __half2*>(&bits), f, off));
          x[8 * h + i] = y.x;
          x[8 * h + i + 4] = y.y;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (CT == CP_F32) {
            x[4 * i + j] = __uint_as_float(w[j]);
          } else if constexpr (CT == CP_BF16) {
            x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
            x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              __nv_fp8_e4m3 s;
              s.__x = (uint8_t)(w[j] >> 8 * k);
              x[4 * j + k] = (float)s;
            }
          }
        }
      }
    }
  }
};

// ALIGN: bytes that the results' rows are aligned to, as far as it counts: 32, 16 or 0.
template <int CT, typename T, int ALIGN>
__global__ void __launch_bounds__(kThreads) k_cache_read(ReadArgs a, int tokens, Share rows) {
  __shared__ Place s_place[kTokens];
  wait_for_stream();
  const Cache& ch = a.cache;
  for (int64_t t0 = (int64_t)blockIdx.x * tokens; t0 < a.T; t0 += (int64_t)gridDim.x * tokens) {
    const int n = (int)min((int64_t)tokens, a.T - t0);
    __syncthreads();
    find_places(ch, a.starts, a.lens, a.B, t0, n, a.status, s_place, nullptr);
    __syncthreads();
    each_item(rows, [&](int r, int first, int step) {
      int h = r / rows.per_row;
      const int d0 = 16 * (r - h * rows.per_row), there = ch.D - d0;  // `there` components at least, a multiple of 4
      const bool key = h < ch.heads;
      if (!key) h -= ch.heads;
      const char* from = (const char*)(key ? ch.k : ch.v) + cache_bytes(CT, h * ch.head_stride + d0);
      const uint8_t* block = (key ? ch.k_block : ch.v_block) + h * ch.block_head + d0 / 16;
      const float* scales = key ? ch.k_scale : ch.v_scale;
      const float f = scales ? scales[h] : 1.0f;
      T* out0 = key ? (T*)a.k + h * a.k_h + d0 : (T*)a.v + h * a.v_h + d0;
      const int64_t apart = key ? a.k_t : a.v_t;
      // two tokens at a time: the second's loads do not wait for the first's stores
#pragma unroll 1
      for (int tok = first; tok < n; tok += 2 * step) {
        Held<CT> held[2];
        const int other = tok + step < n ? tok + step : tok;
        const Place at[2] = {s_place[tok], s_place[other]};
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (at[u].there == 0) held[u].load(from + cache_bytes(CT, at[u].row), block + at[u].block, there);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (at[u].there == -2 || (u == 1 && other == tok)) continue;
          float x[16] = {};
          if (at[u].there == 0) {
            held[u].floats(x);
            if (scales) {
#pragma unroll
              for (int j = 0; j < 16; ++j) x[j] = __fmul_rn(x[j], f);
            }
          }
          T* out = out0 + (t0 + (u ? other : tok)) * apart;
          if (there >= 16) {
            if constexpr (ALIGN == 32)
              store_wide(out, x);
            else
              store_row<ALIGN == 16>(out, x);
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < there) out[j] = from_f32<T>(x[j]);
          }
        }
      }
    });
  }
}

template <int CT, typename T, int ALIGN>
static int cache_read(const ReadArgs& a, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int64_t room = (int64_t)di.sm_count * 8;
  const int tokens = tokens_of(a.T, di.sm_count);
  const int64_t turns = (a.T + tokens - 1) / tokens;
  return cuda_status(launch_early(k_cache_read<CT, T, ALIGN>, dim3((unsigned)(turns < room ? turns : room)), kThreads, 0, s, a, tokens,
                                  share_of(2 * a.cache.heads, (a.cache.D + 15) / 16)),
                     "cache read");
}
template <int CT, typename T>
static int cache_read_of(const ReadArgs& a, cudaStream_t s) {
  if (vectors(a.k, a.k_t, a.k_h, sizeof(T), 32) && vectors(a.v, a.v_t, a.v_h, sizeof(T), 32)) return cache_read<CT, T, 32>(a, s);
  if (vectors(a.k, a.k_t, a.k_h, sizeof(T)) && vectors(a.v, a.v_t, a.v_h, sizeof(T))) return cache_read<CT, T, 16>(a, s);
  return cache_read<CT, T, 0>(a, s);
}
int launch_cache_read(const ReadArgs& a, int dtype, int cache_dtype, cudaStream_t s) {
  const bool wide = dtype == CP_F32;
  if (cache_dtype == CP_F32) return cache_read_of<CP_F32, float>(a, s);
  if (cache_dtype == CP_BF16) return cache_read_of<CP_BF16, __nv_bfloat16>(a, s);
  if (cache_dtype == CP_E4M3) return wide ? cache_read_of<CP_E4M3, float>(a, s) : cache_read_of<CP_E4M3, __nv_bfloat16>(a, s);
  return wide ? cache_read_of<CP_I4, float>(a, s) : cache_read_of<CP_I4, __nv_bfloat16>(a, s);
}

}  // namespace cp
