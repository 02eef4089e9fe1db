// Rotary positions, and the append of keys and values to a paged cache.
//
// Both read every row once and write it once, a few operations an element: HBM
// bounds them.  A block takes a few tokens at a time.  First its threads
// compute the tokens' cosines and sines into shared memory, one pair each, so that
// a token's angles are computed once for all of its heads; then a thread keeps
// the V pairs of one place of a row in registers and turns that place in row
// after row, two 16-byte loads and stores a row where alignment allows.
// Blocks stay for the whole call: the speeds' float64 arithmetic (1/64 of the
// float32 rate) is done once a block.
#include "rope.cuh"

namespace cp {

constexpr int kThreads = 256;
constexpr int kGroup = 16;  // tokens of a block at most
constexpr int kRows = 4;  // rows whose loads a thread has in flight

// Sizes of a launch that the kernels share.
struct Tiling {
  int nv, nvt;       // places of V pairs (and then of V components that pass) in a row; threads for them
  int lanes, group;  // rows side by side, tokens side by side: nvt * lanes * group threads at most
  int half;
};

// V consecutive elements in as few registers as they fill.
template <int BYTES> struct Words;
template <> struct Words<1> { using type = uint8_t; };
template <> struct Words<2> { using type = uint16_t; };
template <> struct Words<4> { using type = uint32_t; };
template <> struct Words<8> { using type = uint2; };
template <> struct Words<16> { using type = uint4; };

template <typename T, int V>
struct Pack {
  typename Words<sizeof(T) * V>::type w;
  __device__ __forceinline__ float operator[](int i) const {
    if (sizeof(T) == 4) return __uint_as_float(word(i));
    if (V == 1) return __uint_as_float((uint32_t)word(0) << 16);
    return __uint_as_float(i % 2 ? word(i / 2) & 0xFFFF0000u : word(i / 2) << 16);
  }

 private:
  __device__ __forceinline__ uint32_t word(int i) const {
    if constexpr (sizeof(w) == 16) return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    else if constexpr (sizeof(w) == 8) return i == 0 ? w.x : w.y;
    else return w;
  }
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load(const T* p, int at) {
  return Pack<T, V>{*reinterpret_cast<const typename Words<sizeof(T) * V>::type*>(p + at)};
}

// x rounded once to the type of p's elements.
template <typename C, int V>
__device__ __forceinline__ void store(C* p, int at, const float (&x)[V]) {
  uint32_t w[4] = {};
  if constexpr (sizeof(C) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = __float_as_uint(x[i]);
  } else if constexpr (V == 1) {
    p[at] = from_f32<C>(x[0]);
    return;
  } else if constexpr (sizeof(C) == 2) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i)
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      uint16_t h;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
      w[i / 2] = i % 2 ? w[i / 2] | (uint32_t)h << 16 : h;
    }
  }
  using W = typename Words<sizeof(C) * V>::type;
  W y;
  if constexpr (sizeof(W) == 16) y = W{w[0], w[1], w[2], w[3]};
  else if constexpr (sizeof(W) == 8) y = W{w[0], w[1]};
  else y = (W)w[0];
  *reinterpret_cast<W*>(p + at) = y;
}

// The two vectors of a place turned by its pairs: in the half layout a[i] with
// b[i], interleaved neighbours within a and within b.
template <typename T, int V>
__device__ __forceinline__ void turn(const Pack<T, V>& a, const Pack<T, V>& b, const float2 (&cs)[V],
                                     bool interleaved, float (&x)[V], float (&y)[V]) {
  if (interleaved) {
    float z[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      z[i] = a[i];
      z[V + i] = b[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float u = z[2 * i], w = z[2 * i + 1];
      z[2 * i] = fmaf(u, cs[i].x, -__fmul_rn(w, cs[i].y));
      z[2 * i + 1] = fmaf(w, cs[i].x, __fmul_rn(u, cs[i].y));
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = z[i];
      y[i] = z[V + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float u = a[i], w = b[i];
      x[i] = fmaf(u, cs[i].x, -__fmul_rn(w, cs[i].y));
      y[i] = fmaf(w, cs[i].x, __fmul_rn(u, cs[i].y));
    }
  }
}

// Speeds of all pairs, once a block.
__device__ __forceinline__ void speeds(const Rope& r, uint64_t* s_turns) {
  for (int i = threadIdx.x; i < r.half; i += kThreads) s_turns[i] = rope_turns(r.inv_freq[i]);
}

// The turned rows lane, lane + lanes, ... of one token.  `row(r, &in, &out,
// &scale)` says where row r lies and goes; a null `out` skips it.
template <typename T, typename C, int V, bool SCALED, int ROWS, typename Row>
__device__ __forceinline__ void turn_rows(const Tiling& tl, const Rope& rope, const float2* cs_of, int vec0, int lane,
                                          int rows, Row row) {
  for (int vec = vec0; vec < tl.nv; vec += tl.nvt) {
    const int turned = tl.half / V;
    const bool pass = vec >= turned;
    float2 cs[V];
    int at0, at1;
    if (pass) {
      at0 = at1 = 2 * tl.half + (vec - turned) * V;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) cs[i] = cs_of[vec * V + i];
      at0 = rope.interleaved ? 2 * vec * V : vec * V;
      at1 = rope.interleaved ? at0 + V : at0 + tl.half;
    }
    for (int r0 = lane; r0 < rows; r0 += ROWS * tl.lanes) {
      Pack<T, V> a[ROWS], b[ROWS];
      const T* in[ROWS];
      C* out[ROWS];
      float scale[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int r = r0 + i * tl.lanes;
        in[i] = nullptr;
        out[i] = nullptr;
        scale[i] = 1.0f;
        if (r < rows) row(r, &in[i], &out[i], &scale[i]);
        if (out[i]) {
          a[i] = load<T, V>(in[i], at0);
          if (!pass) b[i] = load<T, V>(in[i], at1);
        }
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        if (!out[i]) continue;
        float x[V], y[V];
        if (pass) {
#pragma unroll
          for (int j = 0; j < V; ++j) x[j] = a[i][j];
        } else {
          turn<T, V>(a[i], b[i], cs, rope.interleaved, x, y);
        }
        if (SCALED) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            x[j] = __fdiv_rn(x[j], scale[i]);
            if (!pass) y[j] = __fdiv_rn(y[j], scale[i]);
          }
        }
        store<C, V>(out[i], at0, x);
        if (!pass) store<C, V>(out[i], at1, y);
      }
    }
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) k_rotary(RotaryArgs a, Tiling tl, int rows) {
  extern __shared__ __align__(16) uint64_t s_turns[];  // [half], then the groups' (cos, sin), two of them
  float2* s_cs = (float2*)(s_turns + tl.half);
  speeds(a.rope, s_turns);
  const int vec = threadIdx.x % tl.nvt, lane = threadIdx.x / tl.nvt % tl.lanes;
  const int mine = threadIdx.x / tl.nvt / tl.lanes;
  const int64_t tokens = a.B * a.T;
  int flip = 0;
  __syncthreads();
  for (int64_t g = (int64_t)blockIdx.x * tl.group; g < tokens; g += (int64_t)gridDim.x * tl.group, flip ^= 1) {
    float2* cs = s_cs + flip * tl.group * tl.half;  // the other one may still be read
    for (int i = threadIdx.x; i < tl.group * tl.half; i += kThreads) {
      const int64_t tok = g + i / tl.half;
      if (tok >= tokens) break;
      const int64_t b = a.B == 1 ? 0 : tok / a.T;
      rope_unit(s_turns[i % tl.half], a.pos[b * a.pos_stride + (tok - b * a.T)], a.rope, &cs[i].x, &cs[i].y);
    }
    __syncthreads();
    const int64_t tok = g + mine;
    if (mine >= tl.group || tok >= tokens) continue;
    const int64_t b = a.B == 1 ? 0 : tok / a.T, t = tok - b * a.T;
    turn_rows<T, T, V, false, kRows>(tl, a.rope, cs + mine * tl.half, vec, lane, rows, [&](int r, const T** in, T** out, float*) {
      int n = 0;
      while (r >= a.set[n].heads) r -= a.set[n++].heads;
      const RowSet& x = a.set[n];
      *in = (const T*)x.in + b * x.in_b + t * x.in_t + r * x.in_h;
      *out = (T*)x.out + b * x.out_b + t * x.out_t + r * x.out_h;
    });
  }
}

// The sequence that row t belongs to: how many of starts[1..B] are <= t.  A
// warp's lanes look at 32 places at a time: two rounds for 1024 sequences.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int B, int64_t t, int lane) {
  int lo = 0, n = B;
  while (n > 0) {
    const int step = (n + 31) / 32, at = lo + (lane + 1) * step - 1;
    const bool before = at < lo + n && starts[1 + at] <= t;
    const int k = __popc(__ballot_sync(~0u, before));  // ascending: the first k lanes
    const int left = lo + n;
    lo += k * step;
    n = min(step - 1, left - lo);  // all places up to lo are <= t, the next probed one is not
  }
  return lo;
}

template <typename T, typename C, int V, bool SCALED>
__global__ void __launch_bounds__(kThreads, 2) k_cache_append(AppendArgs a, Tiling tl, int vecs) {
  extern __shared__ __align__(16) uint64_t s_turns[];
  __shared__ int64_t s_row[2][kGroup], s_pos[2][kGroup];  // a group's rows of the cache (-1: none) and positions
  __shared__ int s_seq[2][kGroup];
  const Cache& ch = a.cache;
  float2* s_cs = (float2*)(s_turns + tl.half);
  speeds(a.rope, s_turns);
  if (a.new_lens)
    for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < a.B; b += (int64_t)gridDim.x * kThreads) {
      const int64_t n = (int64_t)a.lens[b] + (a.starts ? a.starts[b + 1] - a.starts[b] : 1);
      a.new_lens[b] = (int32_t)min(n, (int64_t)ch.capacity);
    }
  const int vec = threadIdx.x % tl.nvt, lane = threadIdx.x / tl.nvt % tl.lanes;
  const int mine = threadIdx.x / tl.nvt / tl.lanes;
  const int wlane = threadIdx.x % 32;
  int flip = 0;
  for (int64_t g = (int64_t)blockIdx.x * tl.group; g < a.T; g += (int64_t)gridDim.x * tl.group, flip ^= 1) {
    // where the group's tokens go, a warp a token
    for (int i = threadIdx.x / 32; i < tl.group && g + i < a.T; i += kThreads / 32) {
      const int64_t t = g + i;
      const int b = a.starts ? sequence_of(a.starts, a.B, t, wlane) : (int)t;
      if (wlane == 0) {
        int64_t row = -1, pos = 0;
        if (b < a.B) {
          const int len = a.lens[b];
          const int64_t slot = (int64_t)len + (a.starts ? t - a.starts[b] : 0);
          int page = -1;
          if (len >= 0 && slot >= 0 && slot < ch.capacity) page = ch.table[b * ch.table_stride + (uint32_t)slot / (uint32_t)ch.page_size];
          if (page >= 0 && page < ch.pages)
            row = page * ch.page_stride + (int64_t)((uint32_t)slot % (uint32_t)ch.page_size) * ch.slot_stride;
          else if (a.status)
            set_status(a.status, CP_EINVAL);
          pos = a.pos ? a.pos[t] : slot;
        }
        s_row[flip][i] = row;
        s_pos[flip][i] = pos;
        s_seq[flip][i] = b;
      }
    }
    __syncthreads();
    float2* cs = s_cs + flip * tl.group * tl.half;
    for (int i = threadIdx.x; i < tl.group * tl.half; i += kThreads) {
      if (g + i / tl.half >= a.T) break;
      rope_unit(s_turns[i % tl.half], s_pos[flip][i / tl.half], a.rope, &cs[i].x, &cs[i].y);
    }
    __syncthreads();
    const int64_t t = g + mine;
    if (mine >= tl.group || t >= a.T || s_seq[flip][mine] >= a.B) continue;
    const int64_t row = s_row[flip][mine];
    if (a.q.heads)
      turn_rows<T, T, V, false, kRows>(tl, a.rope, cs + mine * tl.half, vec, lane, a.q.heads,
                                [&](int r, const T** in, T** out, float*) {
                                  *in = (const T*)a.q.in + t * a.q.in_t + r * a.q.in_h;
                                  *out = (T*)a.q.out + t * a.q.out_t + r * a.q.out_h;
                                });
    if (row < 0) continue;
    turn_rows<T, C, V, SCALED, 1>(tl, a.rope, cs + mine * tl.half, vec, lane, ch.heads,
                               [&](int r, const T** in, C** out, float* scale) {
                                 *in = (const T*)a.k + t * a.k_t + r * a.k_h;
                                 *out = (C*)ch.k + row + r * ch.head_stride;
                                 if (SCALED && ch.k_scale) *scale = ch.k_scale[r];
                               });
    // values as they are
    for (int r = lane; r < ch.heads; r += tl.lanes) {
      const float scale = SCALED && ch.v_scale ? ch.v_scale[r] : 1.0f;
      for (int i = vec; i < vecs; i += tl.nvt) {
        const Pack<T, V> p = load<T, V>((const T*)a.v + t * a.v_t + r * a.v_h, i * V);
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = SCALED ? __fdiv_rn(p[j], scale) : p[j];
        store<C, V>((C*)ch.v + row + r * ch.head_stride, i * V, x);
      }
    }
  }
}

// Whether every row of a tensor starts on a multiple of V elements.
static bool fits(const void* p, const int64_t* strides, int n, int V, size_t e) {
  if ((uintptr_t)p % (V * e) != 0) return false;
  for (int i = 0; i < n; ++i)
    if (strides[i] % V != 0) return false;
  return true;
}
static bool fits(const RowSet& r, int V, size_t e) {
  const int64_t s[6] = {r.in_b, r.in_t, r.in_h, r.out_b, r.out_t, r.out_h};
  return fits(r.in, s, 3, V, e) && fits(r.out, s + 3, 3, V, e);
}

// Threads to places, rows and tokens.  `rows` of a token run on as many lanes as
// leave each thread kRows of them, fewer tokens than blocks can be had are taken
// one at a time.
static Tiling tiling(int half, int D, int V, int rows, int64_t tokens, int sms) {
  Tiling t;
  t.half = half;
  t.nv = half / V + (D - 2 * half) / V;
  t.nvt = t.nv < kThreads ? t.nv : kThreads;
  const int most = kThreads / t.nvt;
  const bool few = tokens < 4 * sms;
  t.lanes = few ? rows : (rows + kRows - 1) / kRows;
  if (t.lanes > most) t.lanes = most;
  if (t.lanes < 1) t.lanes = 1;
  t.group = few ? 1 : most / t.lanes;
  if (t.group > kGroup) t.group = kGroup;
  // the angles of two groups within 32 KB
  while (t.group > 1 && 16 * t.group * half > 32 * 1024) --t.group;
  return t;
}
static size_t smem_of(const Tiling& t) { return (size_t)t.half * (8 + 2 * 8 * (size_t)t.group); }
static unsigned grid_of(const Tiling& t, int64_t tokens, int sms) {
  int64_t g = (tokens + t.group - 1) / t.group, most = 2 * (int64_t)sms;
  if (g > most) g = most;
  return (unsigned)(g < 1 ? 1 : g);
}

template <typename T, int V>
static int rotary(const RotaryArgs& a, int rows, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const Tiling t = tiling(a.rope.half, a.D, V, rows, a.B * a.T, di.sm_count);
  CP_TRY_STATUS(allow_smem((const void*)k_rotary<T, V>, smem_of(t), "rotary: shared memory"));
  k_rotary<T, V><<<grid_of(t, a.B * a.T, di.sm_count), kThreads, smem_of(t), s>>>(a, t, rows);
  return launch_status("rotary");
}

int launch_rotary(const RotaryArgs& args, int dtype, cudaStream_t s) {
  RotaryArgs a = args;
  int rows = 0, n = 0;
  for (int i = 0; i < args.n; ++i)
    if (args.set[i].heads) {
      a.set[n++] = args.set[i];
      rows += args.set[i].heads;
    }
  a.n = n;
  auto all = [&](int V) {
    if (a.rope.half % V || a.D % V) return false;
    for (int i = 0; i < n; ++i)
      if (!fits(a.set[i], V, dtype == CP_BF16 ? 2 : 4)) return false;
    return true;
  };
  if (dtype == CP_BF16) {
    if (all(8)) return rotary<__nv_bfloat16, 8>(a, rows, s);
    if (all(4)) return rotary<__nv_bfloat16, 4>(a, rows, s);
    if (all(2)) return rotary<__nv_bfloat16, 2>(a, rows, s);
    return rotary<__nv_bfloat16, 1>(a, rows, s);
  }
  if (all(4)) return rotary<float, 4>(a, rows, s);
  if (all(2)) return rotary<float, 2>(a, rows, s);
  return rotary<float, 1>(a, rows, s);
}

template <typename T, typename C, int V, bool SCALED>
static int append(const AppendArgs& a, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const int rows = a.q.heads > a.cache.heads ? a.q.heads : a.cache.heads;
  const Tiling t = tiling(a.rope.half, a.cache.D, V, rows, a.T, di.sm_count);
  auto kernel = k_cache_append<T, C, V, SCALED>;
  CP_TRY_STATUS(allow_smem((const void*)kernel, smem_of(t), "cache append: shared memory"));
  kernel<<<grid_of(t, a.T, di.sm_count), kThreads, smem_of(t), s>>>(a, t, a.cache.D / V);
  return launch_status("cache append");
}
template <typename T, typename C, int V>
static int append_scaled(const AppendArgs& a, cudaStream_t s) {
  return a.cache.k_scale || a.cache.v_scale ? append<T, C, V, true>(a, s) : append<T, C, V, false>(a, s);
}
template <typename T, typename C>
static int append_wide(const AppendArgs& a, cudaStream_t s) {
  auto all = [&](int V) {
    const int64_t k[2] = {a.k_t, a.k_h}, v[2] = {a.v_t, a.v_h};
    // a cache's rows start on 16 bytes and hold a multiple of it
    return a.rope.half % V == 0 && a.cache.D % V == 0 && fits(a.k, k, 2, V, sizeof(T)) && fits(a.v, v, 2, V, sizeof(T)) &&
           (a.q.heads == 0 || fits(a.q, V, sizeof(T)));
  };
  if (sizeof(T) == 2 && all(8)) return append_scaled<T, C, sizeof(T) == 2 ? 8 : 4>(a, s);
  if (all(4)) return append_scaled<T, C, 4>(a, s);
  if (all(2)) return append_scaled<T, C, 2>(a, s);
  return append_scaled<T, C, 1>(a, s);
}

int launch_cache_append(const AppendArgs& a, int dtype, int cache_dtype, cudaStream_t s) {
  if (cache_dtype == CP_F32) return append_wide<float, float>(a, s);
  if (cache_dtype == CP_BF16) return append_wide<__nv_bfloat16, __nv_bfloat16>(a, s);
  if (dtype == CP_F32) return append_wide<float, __nv_fp8_e4m3>(a, s);
  return append_wide<__nv_bfloat16, __nv_fp8_e4m3>(a, s);
}

}  // namespace cp
