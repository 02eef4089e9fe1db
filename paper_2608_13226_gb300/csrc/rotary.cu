// Rotary positions, and the append of keys and values to a paged cache.
//
// Both read every row once and write it once, a few operations an element: HBM
// bounds them, if about 50 KB an SM of it are on their way all the time.  So
//  - a block has a run of tokens for the whole call.  The speeds become fractions of a turn
//    once a block, and where the tokens go is looked up kChunk of them at a time, a
//    thread each;
//  - the rows of its tokens are one line, taken a stage of up to 2 (narrow ones 4)
//    rows a lane at a time.  Between two barriers the block notes where the rows of the
//    stage after next lie (a thread a row), computes the angles of the next
//    stage's tokens (a thread a pair, once for all heads), starts the next
//    stage's copies and turns this one's rows;
//  - a lane turns two places of a row (of a narrow one a place), each V pairs in two 16-byte vectors where
//    alignment allows.  It copies them into slots of its own, so a copy is
//    waited for by the lane that made it and the barrier never waits for one.
// The products are packed pairs of float32 (half the FMA instructions).
#include <type_traits>

#include "rope.cuh"

namespace cp {

constexpr int kThreads = 256;
// Blocks of an SM and rows of a stage that a lane has at most (narrow ones: twice that).  39,328 tokens of
// 28 + 4 bf16 heads of 128, us for rotary / append: 2 and 2 101 / 112, 2 and 1
// 105 / 130, 3 and 1 110 / 118, 4 and 1 116 / 122 (fewer bytes under way), 3 and 2
// 112 / 132 (two blocks fit).
constexpr int kBlocks = 2;
constexpr int kItems = 2;
constexpr int kChunk = 256;  // tokens looked up at a time
constexpr int64_t kTwoBlocks = 108 * 1024;  // dynamic shared memory of a block that leaves room for another
constexpr size_t kMostSmem = 160 * 1024;  // more than any launch takes

// Sizes of a launch that the kernels share.
struct Tiling {
  int places, wide;  // of V pairs (and then of 2 V components that pass) in a row; threads for them
  int parts;         // of a row: places / what those threads take at a time, rounded up
  Divisor rows_of;   // by the parts of a token's rows
  int lanes;         // rows side by side: wide * lanes threads at most
  int stage;         // parts of rows of a stage
  int held;          // tokens whose angles are held: those of two stages
  int half;
  int pairs, side;   // threads for the angles of a token, tokens side by side
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
template <typename T, int V, bool INTERLEAVED>
__device__ __forceinline__ void turn(const Pack<T, V>& a, const Pack<T, V>& b, const float (&c)[V], const float (&s)[V],
                                     float (&x)[V], float (&y)[V]) {
  float u[V], w[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (INTERLEAVED) {
      u[i] = 2 * i < V ? a[2 * i % V] : b[2 * i % V];
      w[i] = 2 * i + 1 < V ? a[(2 * i + 1) % V] : b[(2 * i + 1) % V];
    } else {
      u[i] = a[i];
      w[i] = b[i];
    }
  }
  float p[V], q[V];
  if constexpr (V == 1) {
    p[0] = fmaf(w[0], -s[0], __fmul_rn(u[0], c[0]));
    q[0] = fmaf(u[0], s[0], __fmul_rn(w[0], c[0]));
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const uint64_t u2 = pair(u[i], u[i + 1]), w2 = pair(w[i], w[i + 1]), c2 = pair(c[i], c[i + 1]);
      const uint64_t p2 = fma2(w2, pair(-s[i], -s[i + 1]), mul2(u2, c2));
      const uint64_t q2 = fma2(u2, pair(s[i], s[i + 1]), mul2(w2, c2));
      p[i] = __uint_as_float((uint32_t)p2);
      p[i + 1] = __uint_as_float((uint32_t)(p2 >> 32));
      q[i] = __uint_as_float((uint32_t)q2);
      q[i + 1] = __uint_as_float((uint32_t)(q2 >> 32));
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (INTERLEAVED) {
      (2 * i < V ? x : y)[2 * i % V] = p[i];
      (2 * i + 1 < V ? x : y)[(2 * i + 1) % V] = q[i];
    } else {
      x[i] = p[i];
      y[i] = q[i];
    }
  }
}

// V consecutive floats of shared memory, aligned to them.
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float* x) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 y = *reinterpret_cast<const float4*>(p + i);
      x[i] = y.x;
      x[i + 1] = y.y;
      x[i + 2] = y.z;
      x[i + 3] = y.w;
    }
  } else if constexpr (V == 2) {
    const float2 y = *reinterpret_cast<const float2*>(p);
    x[0] = y.x;
    x[1] = y.y;
  } else {
    x[0] = p[0];
  }
}

// Speeds of all pairs, once a block.
__device__ __forceinline__ void speeds(const Rope& r, uint64_t* s_turns) {
  for (int i = threadIdx.x; i < r.half; i += kThreads) s_turns[i] = rope_turns(r.inv_freq[i]);
}

// BYTES (4, 8 or 16) from global to shared memory, not waited for.
template <int BYTES>
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}

// A part of a token's row, as a thread notes it for the lanes.
constexpr int kThere = 1, kTurned = 2, kCached = 4;  // kCached: goes to the cache, in its type
struct Note {
  const void* in;
  void* out;
  int kind;    // 0: nothing to do
  int angles;  // where its token's angles are
  float scale;
  int part;
};

// A block's run of tokens.  The job says how many rows a token has (`rows`) and
// what row r of token tok is (`note`); `locate` looks up a chunk of tokens, a
// thread each, and gives a token's position.
template <typename T, typename C, int V, int SUBS, bool SCALED, typename Job>
__device__ __forceinline__ void run_rows(Job& job, const Rope& rope, const Tiling& tl, int D, int64_t tokens) {
  extern __shared__ __align__(16) char smem[];  // slots, notes of three stages, angles, speeds
  __shared__ int64_t s_pos[kChunk];
  constexpr int kBytes = V * (int)sizeof(T);
  constexpr int kRows = 2 * kItems / SUBS;  // rows of a stage that a lane has at most
  constexpr bool kSlots = kBytes >= 4;  // smaller vectors are loaded when they are turned
  using Vec = Pack<T, V>;
  Vec* slots = reinterpret_cast<Vec*>(smem);
  Note* notes = reinterpret_cast<Note*>(smem + (kSlots ? 8 * kItems * kThreads * kBytes : 0));
  float* s_cos = reinterpret_cast<float*>(notes + 3 * tl.stage);
  float* s_sin = s_cos + tl.held * tl.half;
  uint64_t* s_turns = reinterpret_cast<uint64_t*>(s_sin + tl.held * tl.half);
  speeds(rope, s_turns);

  const int64_t first = tokens * blockIdx.x / gridDim.x, last = tokens * (blockIdx.x + 1) / gridDim.x;
  const int vec0 = threadIdx.x % tl.wide, lane = threadIdx.x / tl.wide;
  const int rows = job.rows * tl.parts, turned_places = (tl.half + V - 1) / V;
  const bool works = lane < tl.lanes;
  // The pair whose angles a thread computes, and the first token (-1: none).
  const int p0 = threadIdx.x % tl.pairs, tok0 = threadIdx.x / tl.pairs < tl.side ? threadIdx.x / tl.pairs : -1;
  // The components of this lane's places in a row, two vectors each (`n` of them
  // there): of a row that turns and of one that passes whole, in the row's first
  // part.  Rows of several parts are rare and work theirs out.
  struct Place {
    int at0, at1, n;
    bool turned;
  };
  auto place_of = [&](bool turns, int part, int sub) {
    int vec = vec0 + (SUBS * part + sub) * tl.wide;
    Place p;
    p.turned = turns && vec < turned_places;
    // neighbouring lanes have neighbouring vectors, of the first and of the second
    // half of what turns or passes
    int from = 0, to = D;
    if (p.turned) {
      to = 2 * tl.half;
    } else if (turns) {
      from = 2 * tl.half;
      vec -= turned_places;
    }
    const int apart = (to - from + 2 * V - 1) / (2 * V);
    p.at0 = vec < apart ? from + vec * V : D;
    p.at1 = p.at0 + apart * V;
    if (V == 1 && p.turned && rope.interleaved) {  // a pair is not to be parted
      p.at0 = 2 * vec;
      p.at1 = p.at0 + 1;
    }
    p.n = !works || p.at0 >= D ? 0 : p.at1 < to ? 2 : 1;
    return p;
  };
  const Place turning[2] = {place_of(true, 0, 0), place_of(true, 0, SUBS - 1)};
  const Place passing[2] = {place_of(false, 0, 0), place_of(false, 0, SUBS - 1)};
  auto place = [&](int kind, int part, int sub) {
    if (tl.parts > 1 && part) return place_of(kind & kTurned, part, sub);
    return kind & kTurned ? turning[sub] : passing[sub];
  };

  for (int64_t c = first; c < last; c += kChunk) {
    const int n = (int)min((int64_t)kChunk, last - c);
    const int line = n * rows, stages = (line + tl.stage - 1) / tl.stage;
    __syncthreads();  // the chunk before is done with
    if (threadIdx.x < n) s_pos[threadIdx.x] = job.locate(c + threadIdx.x);
    __syncthreads();
    int known = 0, known_at = 0;  // tokens whose angles have been computed, where the next one's go
    for (int s = -2; s < stages; ++s) {
      if (s + 2 < stages) {  // notes of the stage after next
        Note* to = notes + (s + 2) % 3 * tl.stage;
        const int j = threadIdx.x;
        if (j < tl.stage) {
          const int f = (s + 2) * tl.stage + j, tok = tl.rows_of.of(f);
          Note x{};
          if (f < line) {
            const int rp = f - tok * rows, r = tl.parts == 1 ? rp : rp / tl.parts;
            x = job.note(r, c + tok, tok);
            x.part = rp - r * tl.parts;
            x.angles = tok % tl.held * tl.half;
          }
          to[j] = x;
        }
      }
      if (s >= -1 && s + 1 < stages) {
        // angles of the next stage's tokens
        const int upto = min(n, tl.rows_of.of((s + 2) * tl.stage + rows - 1));
        if (tok0 >= 0)
          for (int p = p0; p < tl.half; p += tl.pairs) {
            const uint64_t turns = s_turns[p];
#pragma unroll 2  // 40.3 us as below, one at a time 41.3
            for (int k = tok0; k < upto - known; k += tl.side) {
              const int at = (known_at + k >= tl.held ? known_at + k - tl.held : known_at + k) * tl.half + p;
              rope_unit(turns, s_pos[known + k], rope, s_cos + at, s_sin + at);
            }
          }
        known_at += upto - known;
        if (known_at >= tl.held) known_at -= tl.held;
        known = upto;
        // and its copies
        if (kSlots && works) {
          const Note* of = notes + (s + 1) % 3 * tl.stage;
          Vec* to = slots + (s + 1) % 2 * (kItems * 4 * kThreads) + threadIdx.x;
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            const int j = lane + k * tl.lanes;
            const int kind = j < tl.stage ? of[j].kind : 0;
            if (!kind) continue;
            const T* in = (const T*)of[j].in;
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
              const Place p = place(kind, of[j].part, sub);
              const uint32_t at = smem_addr(to + (SUBS * k + sub) * 2 * kThreads);
              if (p.n > 0) copy_ahead<kSlots ? kBytes : 4>(at, in + p.at0);
              if (p.n > 1) copy_ahead<kSlots ? kBytes : 4>(at + kThreads * kBytes, in + p.at1);
            }
          }
        }
      }
      if (kSlots) asm volatile("cp.async.commit_group;" ::: "memory");
      if (s >= 0 && works) {
        if (kSlots) asm volatile("cp.async.wait_group 1;" ::: "memory");
        const Note* of = notes + s % 3 * tl.stage;
        const Vec* from = slots + s % 2 * (kItems * 4 * kThreads) + threadIdx.x;
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          const int j = lane + k * tl.lanes;
          const int kind = j < tl.stage ? of[j].kind : 0;
          if (!kind) continue;
          const Note x = of[j];
#pragma unroll
          for (int sub = 0; sub < SUBS; ++sub) {
            const Place p = place(kind, x.part, sub);
            if (p.n == 0) continue;
            Vec a{}, b{};
            if (kSlots) {
              a = from[(SUBS * k + sub) * 2 * kThreads];
              b = from[((SUBS * k + sub) * 2 + 1) * kThreads];
            } else {
              a = load<T, V>((const T*)x.in, p.at0);
              if (p.n > 1) b = load<T, V>((const T*)x.in, p.at1);
            }
            float u[V], w[V];
            if (p.turned) {
              float co[V], si[V];
              if (rope.interleaved) {
                constexpr int H = V > 1 ? V / 2 : 1;  // pairs of a vector
                const int at = x.angles + p.at0 / 2, bt = p.n > 1 ? x.angles + p.at1 / 2 : at;
                load_floats<H>(s_cos + at, co);
                load_floats<H>(s_sin + at, si);
                load_floats<H>(s_cos + bt, co + V - H);
                load_floats<H>(s_sin + bt, si + V - H);
                turn<T, V, true>(a, b, co, si, u, w);
              } else {
                load_floats<V>(s_cos + x.angles + p.at0, co);
                load_floats<V>(s_sin + x.angles + p.at0, si);
                turn<T, V, false>(a, b, co, si, u, w);
              }
            } else {
#pragma unroll
              for (int i = 0; i < V; ++i) {
                u[i] = a[i];
                w[i] = p.n > 1 ? b[i] : 0.0f;
              }
            }
            if (!(kind & kCached)) {
              store<T, V>((T*)x.out, p.at0, u);
              if (p.n > 1) store<T, V>((T*)x.out, p.at1, w);
            } else {
              if (SCALED) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                  u[i] = __fdiv_rn(u[i], x.scale);
                  w[i] = __fdiv_rn(w[i], x.scale);
                }
              }
              store<C, V>((C*)x.out, p.at0, u);
              if (p.n > 1) store<C, V>((C*)x.out, p.at1, w);
            }
          }
        }
      }
      __syncthreads();
    }
  }
}

template <typename T>
struct RotaryJob {
  const RotaryArgs& a;
  int rows;
  __device__ int64_t locate(int64_t tok) const {
    const int64_t b = a.B == 1 ? 0 : tok / a.T;
    return a.pos[b * a.pos_stride + (tok - b * a.T)];
  }
  __device__ Note note(int r, int64_t tok, int) const {
    const int64_t b = a.B == 1 ? 0 : tok / a.T, t = tok - b * a.T;
    int i = 0;
    while (r >= a.set[i].heads) r -= a.set[i++].heads;
    const RowSet& x = a.set[i];
    return Note{(const T*)x.in + b * x.in_b + t * x.in_t + r * x.in_h,
                (T*)x.out + b * x.out_b + t * x.out_t + r * x.out_h, kThere | kTurned, 0, 1.0f, 0};
  }
};

template <typename T, int V, int SUBS>
__global__ void __launch_bounds__(kThreads, kBlocks) k_rotary(RotaryArgs a, Tiling tl, int rows) {
  wait_for_stream();
  RotaryJob<T> job{a, rows};
  run_rows<T, T, V, SUBS, false>(job, a.rope, tl, a.D, a.B * a.T);
}

// Rows of a token: its queries, keys and values.
template <typename T, typename C>
struct AppendJob {
  const AppendArgs& a;
  int rows;
  int64_t* s_row;  // [kChunk]: a token's row of the cache; -1 none, -2 it is padding
  __device__ int64_t locate(int64_t t) const {
    const Cache& ch = a.cache;
    const int b = a.starts ? sequence_of(a.starts, a.B, t) : (int)t;
    int64_t row = -2, pos = 0;
    const int64_t i = a.starts && b < a.B ? t - a.starts[b] : 0;  // below 0: before the first sequence's rows
    if (b < a.B && i >= 0) {
      const int len = a.lens[b];
      const int64_t slot = (int64_t)len + i;
      pos = a.pos ? a.pos[t] : slot;
      int page = -1;
      if (len >= 0 && slot >= 0 && slot < ch.capacity)
        page = ch.table[b * ch.table_stride + (uint32_t)slot / (uint32_t)ch.page_size];
      row = -1;
      if (page >= 0 && page < ch.pages)
        row = page * ch.page_stride + (int64_t)((uint32_t)slot % (uint32_t)ch.page_size) * ch.slot_stride;
      else if (a.status)
        set_status(a.status, CP_EINVAL);
    }
    s_row[threadIdx.x] = row;
    return pos;
  }
  __device__ Note note(int r, int64_t t, int i) const {
    const Cache& ch = a.cache;
    const int64_t row = s_row[i];
    if (r < a.q.heads) {
      if (row == -2) return Note{};
      return Note{(const T*)a.q.in + t * a.q.in_t + r * a.q.in_h, (T*)a.q.out + t * a.q.out_t + r * a.q.out_h,
                  kThere | kTurned, 0, 1.0f, 0};
    }
    if (row < 0) return Note{};
    r -= a.q.heads;
    if (r < ch.heads)
      return Note{(const T*)a.k + t * a.k_t + r * a.k_h, (C*)ch.k + row + r * ch.head_stride,
                  kThere | kTurned | kCached, 0, ch.k_scale ? ch.k_scale[r] : 1.0f, 0};
    r -= ch.heads;
    return Note{(const T*)a.v + t * a.v_t + r * a.v_h, (C*)ch.v + row + r * ch.head_stride,
                kThere | kCached, 0, ch.v_scale ? ch.v_scale[r] : 1.0f, 0};
  }
};

template <typename T, typename C, int V, int SUBS, bool SCALED>
__global__ void __launch_bounds__(kThreads, kBlocks) k_cache_append(AppendArgs a, Tiling tl) {
  __shared__ int64_t s_row[kChunk];
  wait_for_stream();
  if (a.new_lens)
    for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < a.B; b += (int64_t)gridDim.x * kThreads) {
      const int len = a.lens[b];
      const int64_t n = (int64_t)len + (a.starts ? (int64_t)a.starts[b + 1] - a.starts[b] : 1);
      a.new_lens[b] = len < 0 ? len : (int32_t)min(n, (int64_t)a.cache.capacity);
    }
  AppendJob<T, C> job{a, a.q.heads + 2 * a.cache.heads, s_row};
  run_rows<T, C, V, SUBS, SCALED>(job, a.rope, tl, a.cache.D, a.T);
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

static size_t slots_of(int bytes) { return bytes >= 4 ? 8 * kItems * kThreads * (size_t)bytes : 0; }
static int places_of(int half, int D, int V) { return (half + V - 1) / V + (D - 2 * half + 2 * V - 1) / (2 * V); }
// Whether rows come in vectors of V: in the half layout a pair's second components are
// vectors of their own, interleaved both are in one vector.
static bool vectors(const Rope& r, int D, int V) {
  return (r.interleaved && V > 1 ? 2 * r.half : r.half) % V == 0 && D % V == 0;
}
static Tiling tiling(int half, int D, int V, int subs, int rows, int bytes) {
  Tiling t;
  t.half = half;
  t.places = places_of(half, D, V);
  t.wide = (t.places + subs - 1) / subs < kThreads ? (t.places + subs - 1) / subs : kThreads;
  t.parts = (t.places + subs * t.wide - 1) / (subs * t.wide);
  t.lanes = kThreads / t.wide;
  rows *= t.parts;
  t.stage = 2 * kItems / subs * t.lanes < kThreads ? 2 * kItems / subs * t.lanes : kThreads;  // a thread notes one row
  // Where angles take much room, heads of few rows and tokens of wide rotations, a
  // stage is as short as leaves two blocks on an SM: 115,255 tokens of two heads of 128
  // 40 us, with one block and longer ones 64.
  const int64_t room = kTwoBlocks - (int64_t)slots_of(bytes) - 8 * half * (int64_t)4;
  const int64_t most = room * rows / (3 * (int64_t)sizeof(Note) * rows + 16 * half);
  if (t.stage > most) t.stage = most < 1 ? 1 : (int)most;
  t.held = (2 * t.stage + rows - 1) / rows + 1;
  t.rows_of = divisor(rows);
  t.pairs = half < 1 ? 1 : half < kThreads ? half : kThreads;
  t.side = kThreads / t.pairs;
  return t;
}
static size_t smem_of(const Tiling& t, int bytes) {
  return slots_of(bytes) + 3 * (size_t)t.stage * sizeof(Note) +
         (size_t)t.half * (8 + 8 * (size_t)t.held);
}
static unsigned grid_of(int64_t tokens, int sms) {
  const int64_t most = kBlocks * (int64_t)sms;
  return (unsigned)(tokens < 1 ? 1 : tokens < most ? tokens : most);
}

// Rows of at most so many places give a lane one place of twice as many rows: the
// lanes of a warp then read longer pieces of fewer rows, and odd numbers of places
// leave no lane idle.  us with two places / with one, bf16: append of 32,000 tokens'
// 8 + 2 x 8 heads of 64 (4 places) 48 / 37, 28 + 2 x 4 to 8 bits 87 / 67, 16 + 2 x 4
// of 80 (5) 60 / 54, of 96 (6) 67 / 57, of 128 of which 64 turn (8) 72 / 65, all (8)
// 111.2 / 110.2 (39,328 tokens of 28 + 2 x 4); of 256 (16) 29.1 / 29.5; float32 of 64
// (8) 71.6 / 72.4.  Rotary of 16 + 4 heads of 80 (5) 48 / 44, of 128 (8) 53.8 / 55.0.
constexpr int kNarrowRotary = 7, kNarrowAppend = 8;
template <typename T, int V, int SUBS = 2>
static int rotary(const RotaryArgs& a, int rows, cudaStream_t s) {
  if constexpr (SUBS == 2 && V * sizeof(T) == 16)
    if (places_of(a.rope.half, a.D, V) <= kNarrowRotary) return rotary<T, V, 1>(a, rows, s);
  static std::atomic<uint64_t> allowed{0};
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const unsigned grid = grid_of(a.B * a.T, di.sm_count);
  const Tiling t = tiling(a.rope.half, a.D, V, SUBS, rows, V * sizeof(T));
  const size_t smem = smem_of(t, V * sizeof(T));
  CP_TRY_STATUS(allow_smem_once((const void*)k_rotary<T, V, SUBS>, kMostSmem, "rotary: shared memory", &allowed));
  return cuda_status(launch_early(k_rotary<T, V, SUBS>, dim3(grid), kThreads, smem, s, a, t, rows), "rotary");
}

int launch_rotary(const RotaryArgs& args, int dtype, cudaStream_t s) {
  RotaryArgs a = args;
  // a batch whose entries follow one another like tokens is one long entry
  bool one = a.pos_stride == a.T;
  for (int i = 0; i < a.n; ++i)
    one = one && (!a.set[i].heads || (a.set[i].in_b == a.T * a.set[i].in_t && a.set[i].out_b == a.T * a.set[i].out_t));
  if (one) {
    a.T *= a.B;
    a.B = 1;
  }
  int rows = 0, n = 0;
  for (int i = 0; i < args.n; ++i)
    if (args.set[i].heads) {
      a.set[n++] = args.set[i];
      rows += args.set[i].heads;
    }
  a.n = n;
  auto all = [&](int V) {
    if (!vectors(a.rope, a.D, V)) return false;
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

template <typename T, typename C, int V, bool SCALED, int SUBS = 2>
static int append(const AppendArgs& a, cudaStream_t s) {
  if constexpr (SUBS == 2 && V * sizeof(T) == 16)
    if (places_of(a.rope.half, a.cache.D, V) <= kNarrowAppend) return append<T, C, V, SCALED, 1>(a, s);
  static std::atomic<uint64_t> allowed{0};
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const unsigned grid = grid_of(a.T, di.sm_count);
  const Tiling t = tiling(a.rope.half, a.cache.D, V, SUBS, a.q.heads + 2 * a.cache.heads, V * sizeof(T));
  auto kernel = k_cache_append<T, C, V, SUBS, SCALED>;
  CP_TRY_STATUS(allow_smem_once((const void*)kernel, kMostSmem, "cache append: shared memory", &allowed));
  return cuda_status(launch_early(kernel, dim3(grid), kThreads, smem_of(t, V * sizeof(T)), s, a, t), "cache append");
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
    return vectors(a.rope, a.cache.D, V) && fits(a.k, k, 2, V, sizeof(T)) && fits(a.v, v, 2, V, sizeof(T)) &&
           (a.q.heads == 0 || fits(a.q, V, sizeof(T)));
  };
  if (sizeof(T) == 2 && all(8)) return append_scaled<T, C, sizeof(T) == 2 ? 8 : 4>(a, s);
  if (all(4)) return append_scaled<T, C, 4>(a, s);
  if (all(2)) return append_scaled<T, C, 2>(a, s);
  return append_scaled<T, C, 1>(a, s);
}

int launch_cache_append(const AppendArgs& a, int dtype, int cache_dtype, cudaStream_t s) {
  if (cache_dtype == CP_I4) return launch_append_fours(a, dtype, s);
  if (cache_dtype == CP_F32) return append_wide<float, float>(a, s);
  if (cache_dtype == CP_BF16) return append_wide<__nv_bfloat16, __nv_bfloat16>(a, s);
  if (dtype == CP_F32) return append_wide<float, __nv_fp8_e4m3>(a, s);
  return append_wide<__nv_bfloat16, __nv_fp8_e4m3>(a, s);
}

}  // namespace cp
