// Attention of one query a sequence over a paged cache: out = softmax(scale q K^T) V
// for every query head, where a group of query heads shares a kv head's keys
// and values.
//
// Each visible key and value row is read once for up to 16 query heads (of a float32
// cache 8), and a bf16 cache gives 1 flop a byte and query head: the kernel is bound by HBM as
// long as enough bytes are in flight (about 1 us of it, 45 KB an SM) whatever
// the lengths.  In a block every warp runs on its own: it copies tiles of 16 keys
// (16 rows of K and of V, wherever their pages are; 8 of float32) into a ring in
// shared memory by 16-byte asynchronous copies, several tiles ahead, and keeps its
// own running maximum, sum and output; no barrier between warps until the block's
// part of one sequence and kv head ends, and no lengths have to be known on the
// host.  How the keys of the B sequences and their kv heads are dealt out
// (launch() has the rule and both sides of each of its lines):
//  - k_decode, one line: the keys of all of them are one line of units of 64
//    keys, cut evenly among as many blocks as the device holds at a time, so that
//    one long sequence and a batch of ragged ones fill it alike.  What is whole in
//    a block is written out, a part goes to the workspace, and k_decode_join adds
//    the parts in the order of the blocks: 32 sequences of 8192 to 8704
//    keys and 4 kv heads of 128 90 us (0.91 of the HBM's rate), one of 200,001 and 8
//    heads 129 us (0.94).
//  - k_decode_cluster: few sequences have a cluster of blocks each, whose parts
//    meet in shared memory: no second launch.  One sequence of 1500 keys 6.7 us,
//    with parts through the workspace 7.7.
//  - k_decode, uncut: sequences of at most 256 keys, a block each.
//  - k_decode_short: many short ones, or hardly any keys, a warp each; nothing is
//    to be merged.
// The products run on mma.sync with keys as rows: S^T = K Q^T (16 keys x 8
// queries) and O^T = V^T P^T, so a group of 8 query heads wastes nothing and
// the columns of S and O lie in the same lanes.  One tile of 16 keys costs 24
// MMAs of a warp (head 128, 8 queries; a third of them for the weights' second
// term) for 8 KB: a sixth of the tensor pipe at the full rate of HBM, where
// tcgen05's 128 rows would be 7 of 8 empty.
#pragma once

#include "rope.cuh"

namespace cp {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kUnit = 64;   // keys of a unit
constexpr int kChunk = 64;  // keys whose marks a warp looks at together
constexpr int kMaxCluster = 16;
constexpr int kMarks = 4;   // of them under way, so that few marks in a chunk hold nothing up
constexpr int kQueue = 128;
// A running maximum follows the scores only when one is more than `slack` above it
// (in units of log 2): weights up to 2^8 are as good as those up to 1, and most
// tiles then need no maximum over their keys.  Beside an 8-bit cache weights become
// float16, which ends at 2^16 and has 11 bits down to 2^-14, then 2^-25 absolute: there
// it stays `under` the largest score, so that a weight keeps its 11 bits down to
// 2^-(14 + under) of the largest and is off by 2^-(25 + under) of it at most below.  With
// `under` 11 and 15 maxima follow more often: 64 sequences of 8192 keys and sharp scores
// 54.2 and 55.0 us, with 7 53.9; 128 ragged ones 94.9 and 97.2, with 7 94.9.
template <int CT> struct Maximum { static constexpr float slack = 8.0f, under = 0.0f; };
template <> struct Maximum<CP_E4M3> { static constexpr float slack = 15.0f, under = 7.0f; };
// A maximum before any score: finite, so that differences of two are, and below no
// finite score (of weight 1 beside it).
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// What a cache's type changes: bytes an element, keys a tile.
template <int CT> struct Type;
template <> struct Type<CP_BF16> { static constexpr int e = 2, tk = 16; using Row = __nv_bfloat16; };
template <> struct Type<CP_E4M3> { static constexpr int e = 1, tk = 16; using Row = __nv_bfloat16; };
template <> struct Type<CP_F32> { static constexpr int e = 4, tk = 8; using Row = float; };

// Shape of one variant: CT cache type, DP head width it is laid out for, QT query
// heads a pass, SHORT whether each warp has sequences of its own (k_decode_short).
template <int CT, int DP, int QT, bool SHORT = false>
struct Shape {
  static constexpr int e = Type<CT>::e;
  // Keys of a tile: 4 of float32 heads of 256, whose rings leave room for two blocks then:
  // 102 sequences of 574 to 1149 keys and 6 query tiles 242 us, with 8 keys and one block
  // 283; 47 of up to 125 15.0, 18.3.
  static constexpr int tk = CT == CP_F32 && DP == 256 ? 4 : Type<CT>::tk;
  static constexpr int row = DP * e;                  // bytes of a row in shared memory
  static constexpr int cpr = row / 16;                // 16-byte chunks of it
  static constexpr int tile = 2 * tk * row;           // K and V of a tile
  // Ring: as many tiles as keep two blocks on an SM, 3 at least.  Three blocks of
  // shorter rings leave the join no room beside them and wait longer: 128 ragged
  // 8-bit sequences 101 us with two, 115 with three; four 125.
  // Short sequences: three blocks, as registers allow, as there is more to begin
  // than to copy.
  static constexpr int fit = (SHORT ? 64 : 100) * 1024 / (kWarps * tile);
  static constexpr int least = SHORT ? 2 : 3;
  static constexpr int stages = fit < least ? least : fit > 8 ? 8 : fit;
  static constexpr int ring = kWarps * stages * tile;
  // float32 queries, the block's or each warp's, and each warp's weights of a tile
  static constexpr int queries = SHORT ? kWarps : 1;
  static constexpr int extra = CT == CP_F32 ? (queries * QT * DP + kWarps * tk * QT) * 4 : 0;
  static constexpr int smem = ring + extra;
  // (Registers allow them but for some spills, 4 to 84 bytes a thread: 16 queries and heads of
  // 256 (255 registers), an 8-bit cache's 8 queries and heads of 64, float32's of 4 queries and
  // heads of 128 and 256 and, for short sequences, of 8 and 128.)
  static constexpr int per_sm = SHORT && smem <= 70 * 1024 ? 3 : smem <= 110 * 1024 ? 2 : 1;
  static constexpr int part = QT * (DP + 2);  // floats of a partial result
  // What beginning and merging a segment costs, in units of 64 keys: about 3 us, in
  // which a block takes 72 KB.
  static constexpr int setup = 72 * 1024 / (2 * kUnit * row) < 1 ? 1 : 72 * 1024 / (2 * kUnit * row);
  static constexpr int pitch = DP + 4;        // floats of a query in the merge: the lanes' banks differ
  static_assert(SHORT || (kWarps * pitch + DP) * QT * 4 <= ring, "the merge reuses the ring");
};

// Rows of the cache in 32 bits: row r of page p starts (p * page + r * slot) << shift
// bytes into K and V.
struct Rows {
  uint32_t page, slot;
  uint32_t scale;  // 1 << shift
  uint32_t mul, div_shift;  // key / page_size = key * mul >> 31 >> div_shift
};

// Where a chunk of a row lies, chunk c at c ^ swizzle(r): rows that are read
// together fall on other banks.  Bits of r only, so that swizzle(r ^ s) is
// swizzle(r) ^ swizzle(s).
template <int CT, int CPR>
__host__ __device__ constexpr int swizzle(int r) {
  return CT == CP_F32 ? (r & 1) << 2 : CPR >= 8 ? r & 7 : (r >> 1) & 3;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  const int n = there ? 16 : 0;  // 0: nothing is read, zeros are written
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                              uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
      "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Four 8-bit elements as two pairs of float16 (exact).
__device__ __forceinline__ void e4m3_f16x2(uint32_t x, uint32_t* lo, uint32_t* hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(*lo), "=r"(*hi)
      : "r"(x));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}

// a / b of non-negative numbers, mostly small ones.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Keys of sequence b: [first, len).
__device__ __forceinline__ void keys_of(const DecodeArgs& a, int b, int* first, int* len) {
  const int n = min(max(a.lens[b], 0), a.cache.capacity);
  *len = n;
  *first = a.window > 0 && a.window < n ? n - (int)a.window : 0;
}
__device__ __forceinline__ int units_of(const DecodeArgs& a, int b, int unit) {
  int first, len;
  keys_of(a, b, &first, &len);
  return max(1, (int)(((int64_t)(len - first) + unit - 1) / unit));
}

// The keys that a warp takes from its part [lo, hi) of a segment, a tile at a
// time: every SIDE-th run of `tk` keys, or of the marked ones among them (SIDE warps
// share a segment).
template <int TK, int SIDE>
struct Keys {
  int next, hi, lane;
  const uint8_t* keep;  // the sequence's marks, or null
  int* queue;           // marked keys that are still to be taken
  int head, count;
  uint32_t mark[kMarks][2];  // of the next chunks

  __device__ void load(int i, int at) {
    mark[i][0] = at + lane < hi ? keep[at + lane] : 0;
    mark[i][1] = at + 32 + lane < hi ? keep[at + 32 + lane] : 0;
  }
  __device__ void start(int lo, int hi_, int warp) {
    hi = hi_;
    head = count = 0;
    next = lo + warp * (keep ? kChunk : TK);
    if (keep) {
#pragma unroll
      for (int i = 0; i < kMarks; ++i) load(i, next + i * SIDE * kChunk);
    }
  }
  // How many keys the next tile has (0: no more); this lane's, or -1.
  __device__ int take(int* key) {
    if (!keep) {
      const int n = min(max(hi - next, 0), TK);
      *key = lane < n ? next + lane : -1;
      next += SIDE * TK;
      return n;
    }
    while (count < TK && next < hi) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t all = __ballot_sync(~0u, mark[0][h] != 0);
        if (mark[0][h])
          queue[(head + count + __popc(all & ((1u << lane) - 1))) % kQueue] = next + 32 * h + lane;
        count += __popc(all);
      }
#pragma unroll
      for (int i = 0; i + 1 < kMarks; ++i) {
        mark[i][0] = mark[i + 1][0];
        mark[i][1] = mark[i + 1][1];
      }
      load(kMarks - 1, next + kMarks * SIDE * kChunk);
      next += SIDE * kChunk;
    }
    __syncwarp();
    const int n = min(count, TK);
    *key = lane < n ? queue[(head + lane) % kQueue] : -1;
    head = (head + n) % kQueue;
    count -= n;
    __syncwarp();
    return n;
  }
};

// A warp's running softmax and output of one segment on the tensor cores.
// Lane (g, t) = (lane / 4, lane % 4) has the scores of keys g and g + 8 and
// queries 2 t, 2 t + 1 of each group of 8, and the same queries' outputs at
// components 16 i + g, + 8 (8-bit caches: 16 i + 2 g, + 1).
template <int CT, int DP, int QT, bool SHORT>
struct Math {
  using S = Shape<CT, DP, QT, SHORT>;
  static constexpr int NT = QT / 8, KS = DP / 16;
  uint32_t q[NT][KS][2];
  float o[NT][KS][4];
  float m[NT][2], l[NT][2];
  float sc[NT][2];  // score = sc * product, in units of log 2
  int g, t;
  uint32_t k_at, v_at;  // this lane's rows in a tile's K and V, first chunk: chunk c is ^ 16 c

  __device__ __forceinline__ void start(const DecodeArgs& a, int b, int hk, int h0, int nq, char*,
                                        int, int lane) {
    g = lane / 4;
    t = lane % 4;
    {
      const int r = lane % 16, key = CT == CP_BF16 ? lane % 8 + lane / 16 * 8 : r;
      const int kc = lane / 16, vc = CT == CP_BF16 ? lane / 8 % 2 : kc;
      k_at = r * S::row + 16 * (kc ^ swizzle<CT, S::cpr>(r));
      v_at = key * S::row + 16 * (vc ^ swizzle<CT, S::cpr>(key));
    }
    const int D = a.cache.D;
    const float scale = a.scale * (a.cache.k_scale ? a.cache.k_scale[hk] : 1.0f) * kLog2e;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = 8 * n + g;
      const uint16_t* src = (const uint16_t*)a.q + b * a.q_b + (int64_t)(h0 + row) * a.q_h;
      // components of a place: bf16 2 t, 2 t + 1 and the same + 8; 8 bits 4 t .. 4 t + 3, as its
      // keys come.  A head is even, so a pair is there or not as one.
      const bool row_there = row < nq;
      const bool pairs = (((uint64_t)a.q | (uint64_t)(2 * a.q_b) | (uint64_t)(2 * a.q_h)) & 3) == 0;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int d = 16 * s + (CT == CP_E4M3 ? 4 * t + 2 * i : 2 * t + 8 * i);
          uint32_t x = 0;
          if (row_there && d < D) {
            if (pairs)
              x = *(const uint32_t*)(src + d);
            else
              x = src[d] | (uint32_t)src[d + 1] << 16;
          }
          q[n][s][i] = x;
        }
      int ex = 0;
      if (CT == CP_E4M3) {
        // keys enter as float16, exactly, and so do queries once their largest
        // component is brought to [2^8, 2^9) by a power of two (bf16 has fewer bits;
        // what lies 2^22 below the largest component loses some; below 2^-92 the
        // largest itself does, and every score is as good as 0)
        float top = 0.0f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            top = fmaxf(top, fmaxf(fabsf(__uint_as_float(q[n][s][i] << 16)),
                                   fabsf(__uint_as_float(q[n][s][i] & 0xFFFF0000u))));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        ex = min(max((int)(__float_as_uint(top) >> 23) - 127 - 8, -100), 100);
        const float f = power(-ex);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            q[n][s][i] = pack_f16(__uint_as_float(q[n][s][i] << 16) * f, __uint_as_float(q[n][s][i] & 0xFFFF0000u) * f);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // the two queries whose scores this lane has
        sc[n][i] = scale;
        if (CT == CP_E4M3) sc[n][i] *= power(__shfl_sync(~0u, ex, 4 * (2 * t + i)));
        m[n][i] = kLowest;
        l[n][i] = 0.0f;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][s][i] = 0.0f;
    }
  }

  __device__ __forceinline__ void tile(uint32_t at, uint32_t valid, char*, int, int) {
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
    if (CT == CP_BF16) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t x[4];
        ldmatrix4(x, (at + k_at) ^ (32 * k));
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16_16816(s[n], x[0], x[1], x[2], x[3], q[n][k][0], q[n][k][1]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < KS; k += 2) {
        uint32_t x[4];
        ldmatrix4(x, (at + k_at) ^ (16 * k));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t a0, a1, a2, a3;
          e4m3_f16x2(x[2 * j], &a0, &a2);
          e4m3_f16x2(x[2 * j + 1], &a1, &a3);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16_16816(s[n], a0, a1, a2, a3, q[n][k + j][0], q[n][k + j][1]);
        }
      }
    }
    const bool full = valid == (1u << S::tk) - 1;
    if (!full) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)  // scores are multiplied by sc, of either sign, next
          if (!(valid >> (g + 8 * (i / 2)) & 1)) s[n][i] = __int_as_float(0x7fffffff);
    }
    bool above = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i)  // fmaxf passes over the NaN of a key that is not there
        above |= fmaxf(s[n][i] * sc[n][i], s[n][i + 2] * sc[n][i]) > m[n][i] + Maximum<CT>::slack;
    if (__any_sync(~0u, above)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float top = fmaxf(fmaxf(s[n][i] * sc[n][i], s[n][i + 2] * sc[n][i]) - Maximum<CT>::under, m[n][i]);
#pragma unroll
          for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
          const float f = exp2_fast(m[n][i] - top);
          m[n][i] = top;
          l[n][i] *= f;
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            o[n][k][i] *= f;
            o[n][k][i + 2] *= f;
          }
        }
    }
    uint32_t p[NT][2], rest[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = exp2_fast(fmaf(s[n][i], sc[n][i & 1], -m[n][i & 1]));
      if (!full) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(valid >> (g + 8 * (i / 2)) & 1)) x[i] = 0.0f;
      }
      l[n][0] += x[0] + x[2];
      l[n][1] += x[1] + x[3];
      // A weight goes on in 11 bits beside an 8-bit cache, float16's (see Maximum).  bfloat16's 8 would
      // add as much error as the output's own rounding (0.0024 of its norm against
      // 0.0017), so what they leave goes on as well, in a second product.  The first term
      // is the largest bfloat16 below the weight: what it leaves is above 0 then, never 0
      // or less, and an infinite value stays that infinity in both products (but for weights
      // below 2^-100, whose second term may be none).
      if (CT == CP_BF16) {
        uint32_t below[4];
        float left[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          below[i] = (uint32_t)max(__float_as_int(x[i]) - 1, 0);  // 0 stays 0
          left[i] = x[i] - __uint_as_float(below[i] & 0xFFFF0000u);
        }
        p[n][0] = movmatrix_trans(__byte_perm(below[0], below[1], 0x7632));
        p[n][1] = movmatrix_trans(__byte_perm(below[2], below[3], 0x7632));
        rest[n][0] = movmatrix_trans(pack_bf16(left[0], left[1]));
        rest[n][1] = movmatrix_trans(pack_bf16(left[2], left[3]));
      } else {
        p[n][0] = movmatrix_trans(pack_f16(x[0], x[1]));
        p[n][1] = movmatrix_trans(pack_f16(x[2], x[3]));
      }
    }
    at += S::tk * S::row;
    if (CT == CP_BF16) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t x[4];
        ldmatrix4_trans(x, (at + v_at) ^ (32 * k));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_bf16_16816(o[n][k], x[0], x[1], x[2], x[3], p[n][0], p[n][1]);
          mma_bf16_16816(o[n][k], x[0], x[1], x[2], x[3], rest[n][0], rest[n][1]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < KS; k += 2) {
        uint32_t x[4];
        ldmatrix4_trans(x, (at + v_at) ^ (16 * k));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          // bytes: key 2 t's components 2 g, 2 g + 1, then key 2 t + 1's
          uint32_t a0, a1, a2, a3;
          e4m3_f16x2(__byte_perm(x[2 * j], 0, 0x3120), &a0, &a1);
          e4m3_f16x2(__byte_perm(x[2 * j + 1], 0, 0x3120), &a2, &a3);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16_16816(o[n][k + j], a0, a1, a2, a3, p[n][0], p[n][1]);
        }
      }
    }
  }

  // The outputs over their sums, for a warp that has all keys: out(query, component,
  // value), and lse(query, value).
  template <typename Out, typename Lse>
  __device__ __forceinline__ void write(float vs, Out out, Lse lse) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[n][i] += __shfl_xor_sync(~0u, l[n][i], d);
        const int query = 8 * n + 2 * t + i;
        const float by = vs / l[n][i];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          out(query, 16 * k + (CT == CP_E4M3 ? 2 * g : g), l[n][i] == 0.0f ? 0.0f : o[n][k][i] * by);
          out(query, 16 * k + (CT == CP_E4M3 ? 2 * g + 1 : g + 8), l[n][i] == 0.0f ? 0.0f : o[n][k][i + 2] * by);
        }
        if (g == 0) lse(query, l[n][i] == 0.0f ? -INFINITY : (m[n][i] + log2f(l[n][i])) * kLn2);
      }
  }

  // This warp's maximum and sum of each query.
  __device__ __forceinline__ void finish(float* sm, float* sl) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[n][i] += __shfl_xor_sync(~0u, l[n][i], d);
        if (g == 0) {
          sm[8 * n + 2 * t + i] = m[n][i];
          sl[8 * n + 2 * t + i] = l[n][i];
        }
      }
  }
  // Its outputs by the common maximum: buf[query][component] = o * f[query].
  __device__ __forceinline__ void put(float* buf, const float* f) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int query = 8 * n + 2 * t + (i & 1);
          const int d = 16 * k + (CT == CP_E4M3 ? 2 * g + i / 2 : g + 8 * (i / 2));
          buf[query * S::pitch + d] = o[n][k][i] * f[query];
        }
  }
};

// The same in float32 on the FMA units: 4 lanes a key for the scores, then the
// components spread over the lanes.
template <int DP, int QT, bool SHORT>
struct Math<CP_F32, DP, QT, SHORT> {
  using S = Shape<CP_F32, DP, QT, SHORT>;
  static constexpr int V = DP / 32;  // components of a lane
  static constexpr int L = 32 / S::tk;  // lanes of a key
  float o[QT][V];
  float m[QT], l[QT];
  float sc;

  __device__ __forceinline__ void start(const DecodeArgs& a, int b, int hk, int h0, int nq, char* extra,
                                        int warp, int lane) {
    float* sq = queries(extra, warp);  // the block's, of which each warp fills a part, or the warp's
    const float* src = (const float*)a.q + b * a.q_b + (int64_t)h0 * a.q_h;
    const bool quads = (((uint64_t)a.q | (uint64_t)(4 * a.q_b) | (uint64_t)(4 * a.q_h)) & 15) == 0;
#pragma unroll 4
    for (int i = SHORT ? lane : warp * 32 + lane; i < QT * (DP / 4); i += SHORT ? 32 : kThreads) {
      const int n = i / (DP / 4), d = 4 * (i % (DP / 4));  // heads are a multiple of 4
      float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (n < nq && d < a.cache.D) {
        const float* from = src + n * a.q_h + d;
        x = quads ? *(const float4*)from : make_float4(from[0], from[1], from[2], from[3]);
      }
      *(float4*)(sq + 4 * i) = x;
    }
    if (SHORT)
      __syncwarp();
    else
      __syncthreads();
    sc = a.scale * (a.cache.k_scale ? a.cache.k_scale[hk] : 1.0f) * kLog2e;
#pragma unroll
    for (int n = 0; n < QT; ++n) {
      m[n] = kLowest;
      l[n] = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) o[n][i] = 0.0f;
    }
  }

  __device__ static float* queries(char* extra, int warp) { return (float*)extra + (SHORT ? warp * QT * DP : 0); }
  // Component of this lane's i-th: consecutive float4 (float2 for heads of 64).
  __device__ static int component(int i, int lane) {
    return V == 2 ? 2 * lane + i : 128 * (i / 4) + 4 * lane + i % 4;
  }

  __device__ __forceinline__ void tile(uint32_t at, uint32_t valid, char* extra, int warp,
                                       int lane) {
    const float* sq = queries(extra, warp);
    float* sp = (float*)extra + S::queries * QT * DP + warp * S::tk * QT;
    const char* smem = extra - S::ring;
    const char* keys = smem + (at - smem_addr(smem));
    const int r = lane / L, sub = lane % L;
    float s[QT];
#pragma unroll
    for (int n = 0; n < QT; ++n) s[n] = 0.0f;
    // Chunks of the key in flight at a time: 32 sequences of 1000 to 4000 keys and 32
    // heads of 64 246 us, one by one 292.
    constexpr int kHeld = S::cpr / L < 8 ? S::cpr / L : 8;
#pragma unroll
    for (int j0 = 0; j0 < S::cpr / L; j0 += kHeld) {
      float4 k[kHeld];
#pragma unroll
      for (int j = 0; j < kHeld; ++j)
        k[j] = *(const float4*)(keys + r * S::row +
                                16 * ((L * (j0 + j) + sub) ^ swizzle<CP_F32, S::cpr>(r)));
#pragma unroll
      for (int j = 0; j < kHeld; ++j)
#pragma unroll
        for (int n = 0; n < QT; ++n) {
          const float4 x = *(const float4*)(sq + n * DP + 4 * (L * (j0 + j) + sub));
          s[n] = fmaf(x.x, k[j].x, fmaf(x.y, k[j].y, fmaf(x.z, k[j].z, fmaf(x.w, k[j].w, s[n]))));
        }
    }
    const bool there = valid >> r & 1;
    bool above = false;
#pragma unroll
    for (int n = 0; n < QT; ++n) {
#pragma unroll
      for (int d = 1; d < L; d *= 2) s[n] += __shfl_xor_sync(~0u, s[n], d);
      above |= there && s[n] * sc > m[n] + Maximum<CP_F32>::slack;
    }
    if (__any_sync(~0u, above)) {
#pragma unroll
      for (int n = 0; n < QT; ++n) {
        float top = there ? fmaxf(s[n] * sc, m[n]) : m[n];
#pragma unroll
        for (int d = L; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        const float f = exp2f(m[n] - top);
        m[n] = top;
        l[n] *= f;
#pragma unroll
        for (int i = 0; i < V; ++i) o[n][i] *= f;
      }
    }
#pragma unroll
    for (int n = 0; n < QT; ++n) {
      const float p = there ? exp2f(fmaf(s[n], sc, -m[n])) : 0.0f;
      l[n] += p;
      if (sub == 0) sp[r * QT + n] = p;
    }
    __syncwarp();
    const char* values = keys + S::tk * S::row;
#pragma unroll
    for (int k = 0; k < S::tk; ++k) {
      float v[V], p[QT];
      if (V == 2) {
        const float2 x = *(const float2*)(values + k * S::row + 8 * (lane % 2) +
                                          16 * (lane / 2 ^ swizzle<CP_F32, S::cpr>(k)));
        v[0] = x.x;
        v[V > 1 ? 1 : 0] = x.y;
      } else {
#pragma unroll
        for (int j = 0; j < V / 4; ++j) {
          const float4 x = *(const float4*)(values + k * S::row +
                                            16 * (32 * j + lane ^ swizzle<CP_F32, S::cpr>(k)));
          v[4 * j] = x.x;
          v[4 * j + 1] = x.y;
          v[4 * j + 2] = x.z;
          v[4 * j + 3] = x.w;
        }
      }
#pragma unroll
      for (int n = 0; n < QT; n += 4) {
        const float4 x = *(const float4*)(sp + k * QT + n);
        p[n] = x.x;
        p[n + 1] = x.y;
        p[n + 2] = x.z;
        p[n + 3] = x.w;
      }
#pragma unroll
      for (int n = 0; n < QT; ++n)
#pragma unroll
        for (int i = 0; i < V; ++i) o[n][i] = fmaf(p[n], v[i], o[n][i]);
    }
    __syncwarp();
  }

  template <typename Out, typename Lse>
  __device__ __forceinline__ void write(float vs, Out out, Lse lse) {
#pragma unroll
    for (int n = 0; n < QT; ++n) {
#pragma unroll
      for (int d = L; d < 32; d *= 2) l[n] += __shfl_xor_sync(~0u, l[n], d);
      const float by = vs / l[n];
#pragma unroll
      for (int i = 0; i < V; ++i) out(n, component(i, threadIdx.x % 32), l[n] == 0.0f ? 0.0f : o[n][i] * by);
      if (threadIdx.x % 32 == 0) lse(n, l[n] == 0.0f ? -INFINITY : (m[n] + log2f(l[n])) * kLn2);
    }
  }
  __device__ __forceinline__ void finish(float* sm, float* sl) {
#pragma unroll
    for (int n = 0; n < QT; ++n) {
#pragma unroll
      for (int d = L; d < 32; d *= 2) l[n] += __shfl_xor_sync(~0u, l[n], d);
      if (threadIdx.x % 32 == 0) {
        sm[n] = m[n];
        sl[n] = l[n];
      }
    }
  }
  __device__ __forceinline__ void put(float* buf, const float* f) {
#pragma unroll
    for (int n = 0; n < QT; ++n)
#pragma unroll
      for (int i = 0; i < V; ++i) buf[n * S::pitch + component(i, threadIdx.x % 32)] = o[n][i] * f[n];
  }
};

// A warp's keys [lo, hi) of sequence b for the queries from h0 on: their tiles through
// its ring into `math`.
template <int CT, int DP, int QT, bool SHORT, typename K>
__device__ __forceinline__ void math_of_keys(const DecodeArgs& a, const Rows& rows, K& keys, const int32_t* table, int lo,
                                             int hi, int hk, int b, int h0, int nq, int warp, int lane, uint32_t ring,
                                             uint32_t* s_valid, char* extra, Math<CT, DP, QT, SHORT>& math) {
  using S = Shape<CT, DP, QT, SHORT>;
  const Cache& ch = a.cache;
  const int chunks = ch.D * S::e / 16;  // of a row that is there
  const char* kp = (const char*)ch.k + (int64_t)hk * ch.head_stride * S::e;
  const char* vp = (const char*)ch.v + (int64_t)hk * ch.head_stride * S::e;
  if (chunks < S::cpr)  // components beyond the head's: the products run over zeros
    for (int i = lane; i < S::stages * S::tk * (S::cpr - chunks); i += 32) {
      const int c = chunks + i % (S::cpr - chunks), r = i / (S::cpr - chunks);
      const uint32_t at = ring + r / S::tk * S::tile + r % S::tk * S::row + 16 * (c ^ swizzle<CT, S::cpr>(r % S::tk));
      asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
    }

  keys.start(lo, hi, SHORT ? 0 : warp);
  int key, n_next = keys.take(&key), page = -1, slot_of = 0, issued = 0;
  auto look = [&] {
    const int p = (int)((uint64_t)(uint32_t)key * rows.mul >> 31 >> rows.div_shift);
    page = key >= 0 ? table[p] : -1;
    slot_of = key - p * ch.page_size;
  };
  auto issue = [&] {
    if (n_next > 0) {
      const int slot = issued % S::stages;
      bool ok = key >= 0;
      if (ok && (page < 0 || page >= ch.pages)) {
        if (a.status) set_status(a.status, CP_EINVAL);
        ok = false;
      }
      const uint32_t mine = ok ? (uint32_t)page * rows.page + (uint32_t)slot_of * rows.slot : 0;
      const uint32_t valid = __ballot_sync(~0u, ok);
      if (lane == 0) s_valid[slot] = valid;
      // 32 chunks at a time: some rows side by side, or a part of one
      constexpr int side = S::cpr >= 32 ? 1 : 32 / S::cpr;
      const int c = lane % S::cpr, r0 = lane / S::cpr;
      const uint32_t to = ring + slot * S::tile + r0 * S::row + 16 * (c ^ swizzle<CT, S::cpr>(r0));
      auto each = [&](auto copy) {
#pragma unroll
        for (int i = 0; i < S::tk * S::cpr / 32; ++i) {
          constexpr int turns = S::cpr > 32 ? S::cpr / 32 : 1;  // copies of a row
          const int r = i / turns * side, more = i % turns * 512;
          const uint64_t off = (uint64_t)__shfl_sync(~0u, mine, r + r0) * rows.scale + (16 * c + more);
          const uint32_t at = (to ^ (16 * swizzle<CT, S::cpr>(r))) + r * S::row + more;
          copy(at, off, r + r0, c + more / 16);
        }
      };
      if (valid == (1u << S::tk) - 1 && chunks == S::cpr) {
        each([&](uint32_t at, uint64_t off, int, int) {
          copy16(at, kp + off);
          copy16(at + S::tk * S::row, vp + off);
        });
      } else {
        each([&](uint32_t at, uint64_t off, int r, int c) {
          const bool there = valid >> r & 1;
          if (c < chunks) {
            copy16(at, kp + (there ? off : 0), there);
            copy16(at + S::tk * S::row, vp + (there ? off : 0), there);
          }
        });
      }
      ++issued;
      n_next = keys.take(&key);
      look();
    }
    copy_commit();
  };
  look();
  __syncwarp();
#pragma unroll 1
  for (int i = 0; i < S::stages - 1; ++i) issue();
  math.start(a, b, hk, h0, nq, extra, warp, lane);
  for (int i = 0; i < issued; ++i) {
    copy_wait<S::stages - 2>();
    __syncwarp();  // tile i is there for every lane, and tile i - 1 done with
    issue();
    const int slot = i % S::stages;
    math.tile(ring + slot * S::tile, s_valid[slot], extra, warp, lane);
  }
}

// Query n's maximum and sum of all warps, and what each warp's output is to be
// multiplied by.
template <int QT>
__device__ __forceinline__ void merge_sums(const float (&s_m)[kWarps][QT], const float (&s_l)[kWarps][QT],
                                           float (&s_f)[kWarps][QT], int n, float* top_of, float* sum_of) {
  float top = kLowest, sum = 0.0f;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][n]);
  for (int w = 0; w < kWarps; ++w) {
    const float f = exp2f(s_m[w][n] - top);
    s_f[w][n] = f;
    sum += s_l[w][n] * f;
  }
  *top_of = top;
  *sum_of = sum;
}

// Four components of a query added over the warps, quad i of [QT][DP / 4].
template <int DP, int QT, int PITCH>
__device__ __forceinline__ float4 merge_quad(const float* buf, int i) {
  const float* at = buf + i / (DP / 4) * PITCH + 4 * (i % (DP / 4));
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const float4 y = *(const float4*)(at + w * QT * PITCH);
    x.x += y.x;
    x.y += y.y;
    x.z += y.z;
    x.w += y.w;
  }
  return x;
}

// A float of another block of the cluster, at the place of this block's *p.
__device__ __forceinline__ float remote(const float* p, int rank) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(map_rank(smem_addr(p), (uint32_t)rank)) : "memory");
  return x;
}

template <int CT, int DP, int QT>
__global__ void __launch_bounds__(kThreads) k_decode(DecodeArgs a, Rows rows, int unit, int tiles, float* parts,
                                                     Begin* begins, int by_column) {
  using S = Shape<CT, DP, QT>;
  using Row = typename Type<CT>::Row;
  extern __shared__ __align__(1024) char smem[];  // addresses of rows are put together by exclusive or
  __shared__ int s_queue[kWarps][kQueue];
  __shared__ uint32_t s_valid[kWarps][S::stages];
  __shared__ float s_m[kWarps][QT], s_l[kWarps][QT], s_f[kWarps][QT], s_top[QT], s_sum[QT];
  wait_for_stream();
  const Cache& ch = a.cache;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int G = a.Hq / ch.heads, cols = ch.heads * tiles;

  // this block's units of the line
  const int64_t mine = lane < a.B ? units_of(a, lane, unit) : 0;
  int64_t total = mine;
#pragma unroll 4
  for (int b = 32 + lane; b < a.B; b += 32) total += units_of(a, b, unit);
#pragma unroll
  for (int d = 16; d; d /= 2) total += __shfl_xor_sync(~0u, total, d);
  total *= cols;
  // Where blocks have many units, a query tile counts for `setup` more, so that one
  // with several short ones does not end last.
  const int setup = total >= 8 * (int64_t)gridDim.x ? S::setup : 0;
  total += (int64_t)setup * a.B * cols;
  const int64_t blocks = min((int64_t)gridDim.x, total);  // each of these has a unit at least
  if (begins && !by_column && threadIdx.x == 0) begins[blockIdx.x] = Begin{0, 0, 0, 0};
  if (blockIdx.x >= blocks) return;
  // the first `longer` of them one more than the others
  const int64_t share = quotient(total, blocks), longer = total - share * blocks;
  int64_t u = share * blockIdx.x + min((int64_t)blockIdx.x, longer);
  const int64_t end = u + share + (blockIdx.x < longer);
  // the sequence they start in
  int b = 0;
  int64_t before = 0;
#pragma unroll 1
  for (int b0 = 0;; b0 += 32) {
    const int64_t units = b0 == 0 ? mine : b0 + lane < a.B ? units_of(a, b0 + lane, unit) : 0;
    const int64_t own = b0 + lane < a.B ? (units + setup) * cols : 0;
    int64_t upto = own;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int64_t x = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += x;
    }
    const uint32_t past = __ballot_sync(~0u, before + upto > u);
    if (past) {
      const int i = __ffs(past) - 1;
      b = b0 + i;
      before += __shfl_sync(~0u, upto - own, i);
      break;
    }
    before += __shfl_sync(~0u, upto, 31);
  }

  const uint32_t ring = smem_addr(smem) + warp * S::stages * S::tile;
  char* extra = smem + S::ring;
  Keys<S::tk, kWarps> keys;
  keys.lane = lane;
  keys.queue = s_queue[warp];

  for (; u < end; ++b) {
    int first, len;
    keys_of(a, b, &first, &len);
    const int nu = max(1, (int)(((int64_t)(len - first) + unit - 1) / unit));
    const int32_t* table = ch.table + (int64_t)b * ch.table_stride;
    keys.keep = a.keep ? a.keep + (int64_t)b * a.keep_stride : nullptr;
    const int long_nu = nu + setup;
    for (; u < end && u < before + (int64_t)long_nu * cols;) {
      // the segment: units [k0, k1) of sequence b, query tile `col`, on the line after its setup
      const int col = (int)quotient(u - before, long_nu);
      const int64_t at = before + (int64_t)col * long_nu + setup;  // its unit 0
      const int k0 = (int)max(u - at, (int64_t)0), k1 = (int)min((int64_t)nu, end - at);
      u = min(end, at + nu);
      if (k1 <= 0) continue;  // the block ends before unit 0
      const int hk = col / tiles, h0 = hk * G + col % tiles * QT;
      const int nq = min(QT, G - col % tiles * QT);
      const int lo = first + k0 * unit, hi = (int)min((int64_t)len, first + (int64_t)k1 * unit);
      Math<CT, DP, QT, false> math;
      math_of_keys<CT, DP, QT, false>(a, rows, keys, table, lo, hi, hk, b, h0, nq, warp, lane, ring, s_valid[warp], extra,
                                      math);
      math.finish(s_m[warp], s_l[warp]);
      copy_wait<0>();
      __syncthreads();
      // the warps' results by a common maximum
      if (threadIdx.x < QT) merge_sums<QT>(s_m, s_l, s_f, threadIdx.x, &s_top[threadIdx.x], &s_sum[threadIdx.x]);
      __syncthreads();
      float* buf = (float*)smem;
      math.put(buf + warp * QT * S::pitch, s_f[warp]);
      __syncthreads();
      const bool whole = k0 == 0 && k1 == nu;
      const float vs = ch.v_scale ? ch.v_scale[hk] : 1.0f;
      float* part = whole ? nullptr : parts + (2 * (int64_t)blockIdx.x + (k0 == 0)) * S::part;
      for (int i = threadIdx.x; i < nq * (DP / 4); i += kThreads) {
        const float4 x = merge_quad<DP, QT, S::pitch>(buf, i);
        const int n = i / (DP / 4), d = 4 * (i % (DP / 4));
        if (!whole) {
          *(float4*)(part + 2 * QT + 4 * i) = x;
        } else if (d < ch.D) {
          const float sum = s_sum[n], by = vs / sum;
          Row* out = (Row*)a.out + b * a.o_b + (int64_t)(h0 + n) * a.o_h + d;
          out[0] = from_f32<Row>(sum == 0.0f ? 0.0f : x.x * by);
          out[1] = from_f32<Row>(sum == 0.0f ? 0.0f : x.y * by);
          out[2] = from_f32<Row>(sum == 0.0f ? 0.0f : x.z * by);
          out[3] = from_f32<Row>(sum == 0.0f ? 0.0f : x.w * by);
        }
      }
      if (threadIdx.x < nq) {
        const int n = threadIdx.x;
        if (!whole) {
          part[n] = s_top[n];
          part[QT + n] = s_sum[n];
        } else if (a.lse) {
          a.lse[(int64_t)b * a.Hq + h0 + n] = s_sum[n] == 0.0f ? -INFINITY : (s_top[n] + log2f(s_sum[n])) * kLn2;
        }
      }
      if (begins && k0 == 0 && (by_column || !whole) && threadIdx.x == 0) {
        // the block that has the query tile's last unit
        const int64_t last = at + nu - 1, split = longer * (share + 1);
        const int to = (int)(last < split ? quotient(last, share + 1) : longer + quotient(last - split, share));
        begins[by_column ? b * cols + col : (int)blockIdx.x] =
            Begin{(int)blockIdx.x, whole ? 0 : to - (int)blockIdx.x + 1, b, col};
      }
      __syncthreads();  // the ring and the sums are free
    }
    before += (int64_t)long_nu * cols;
  }
}

// Few query tiles of a few units a block: a cluster of blocks shares each, and adds its
// parts from one another's shared memory, an element a thread, so that no launch has
// to follow.
template <int CT, int DP, int QT>
__global__ void __launch_bounds__(kThreads) k_decode_cluster(DecodeArgs a, Rows rows, int tiles, int size) {
  using S = Shape<CT, DP, QT>;
  using Row = typename Type<CT>::Row;
  extern __shared__ __align__(1024) char smem[];
  __shared__ int s_queue[kWarps][kQueue];
  __shared__ uint32_t s_valid[kWarps][S::stages];
  __shared__ float s_m[kWarps][QT], s_l[kWarps][QT], s_f[kWarps][QT];
  __shared__ float s_top[QT], s_sum[QT];          // this block's, for the others
  __shared__ float s_w[QT][kMaxCluster], s_all[QT];  // the blocks' weights and the whole sum
  wait_for_stream();
  const Cache& ch = a.cache;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int G = a.Hq / ch.heads, cols = ch.heads * tiles;
  const int rank = (int)cluster_ctarank(), column = blockIdx.x / size;
  const int b = column / cols, col = column - b * cols;
  const int hk = col / tiles, h0 = hk * G + col % tiles * QT;
  const int nq = min(QT, G - col % tiles * QT);
  int first, len;
  keys_of(a, b, &first, &len);
  // this block's tiles of the keys
  const int n = (len - first + S::tk - 1) / S::tk;
  const int lo = first + (int)((int64_t)n * rank / size) * S::tk;
  const int hi = min(len, first + (int)((int64_t)n * (rank + 1) / size) * S::tk);
  Keys<S::tk, kWarps> keys;
  keys.lane = lane;
  keys.queue = s_queue[warp];
  keys.keep = a.keep ? a.keep + (int64_t)b * a.keep_stride : nullptr;
  Math<CT, DP, QT, false> math;
  math_of_keys<CT, DP, QT, false>(a, rows, keys, ch.table + (int64_t)b * ch.table_stride, lo, hi, hk, b, h0, nq, warp, lane,
                                  smem_addr(smem) + warp * S::stages * S::tile, s_valid[warp], smem + S::ring, math);
  math.finish(s_m[warp], s_l[warp]);
  copy_wait<0>();
  __syncthreads();
  if (threadIdx.x < QT) merge_sums<QT>(s_m, s_l, s_f, threadIdx.x, &s_top[threadIdx.x], &s_sum[threadIdx.x]);
  __syncthreads();
  float* buf = (float*)smem;
  math.put(buf + warp * QT * S::pitch, s_f[warp]);
  __syncthreads();
  float* mine = buf + kWarps * QT * S::pitch;  // [nq][DP]
  for (int i = threadIdx.x; i < nq * (DP / 4); i += kThreads)
    *(float4*)(mine + 4 * i) = merge_quad<DP, QT, S::pitch>(buf, i);
  __syncwarp();
  hw_cluster_sync();
  // every block weighs the parts, and adds its share of the elements
  for (int q = warp; q < nq; q += kWarps) {
    const float m = lane < size ? remote(&s_top[q], lane) : kLowest, l = lane < size ? remote(&s_sum[q], lane) : 0.0f;
    float top = m;
#pragma unroll
    for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    const float f = exp2f(m - top), sum = warp_sum(l * f);
    if (lane < size) s_w[q][lane] = f;
    if (lane == 0) {
      s_all[q] = sum;
      if (rank == 0 && a.lse)
        a.lse[(int64_t)b * a.Hq + h0 + q] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
  }
  __syncthreads();
  const float vs = ch.v_scale ? ch.v_scale[hk] : 1.0f;
  for (int i = rank * kThreads + threadIdx.x; i < nq * DP; i += size * kThreads) {
    const int q = i / DP, d = i % DP;
    float x = 0.0f;
    float y[kMaxCluster];
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) y[r] = r < size ? remote(&mine[i], r) : 0.0f;
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r)
      if (r < size) x = fmaf(s_w[q][r], y[r], x);
    if (d < ch.D)
      ((Row*)a.out)[b * a.o_b + (int64_t)(h0 + q) * a.o_h + d] =
          from_f32<Row>(s_all[q] == 0.0f ? 0.0f : x * (vs / s_all[q]));
  }
  __syncwarp();
  hw_cluster_sync();  // no block's memory goes while it is read
}

// Many short sequences: a warp takes a query tile alone, and then another, so that one's beginning (table, keys, queries: three trips
// to memory) runs beside the others' and nothing is merged.
template <int CT, int DP, int QT>
__global__ void __launch_bounds__(kThreads) k_decode_short(DecodeArgs a, Rows rows, int tiles, int64_t columns) {
  using S = Shape<CT, DP, QT, true>;
  using Row = typename Type<CT>::Row;
  extern __shared__ __align__(1024) char smem[];
  __shared__ int s_queue[kWarps][kQueue];
  __shared__ uint32_t s_valid[kWarps][S::stages];
  wait_for_stream();
  const Cache& ch = a.cache;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int G = a.Hq / ch.heads, cols = ch.heads * tiles;
  const uint32_t ring = smem_addr(smem) + warp * S::stages * S::tile;
  Keys<S::tk, 1> keys;
  keys.lane = lane;
  keys.queue = s_queue[warp];
  for (int64_t c = (int64_t)blockIdx.x * kWarps + warp; c < columns; c += (int64_t)gridDim.x * kWarps) {
    const int b = (int)quotient(c, cols), col = (int)(c - (int64_t)b * cols);
    const int hk = col / tiles, h0 = hk * G + col % tiles * QT;
    const int nq = min(QT, G - col % tiles * QT);
    int first, len;
    keys_of(a, b, &first, &len);
    keys.keep = a.keep ? a.keep + (int64_t)b * a.keep_stride : nullptr;
    Math<CT, DP, QT, true> math;
    math_of_keys<CT, DP, QT, true>(a, rows, keys, ch.table + (int64_t)b * ch.table_stride, first, len, hk, b, h0, nq, warp,
                                   lane, ring, s_valid[warp], smem + S::ring, math);
    copy_wait<0>();
    math.write(
        ch.v_scale ? ch.v_scale[hk] : 1.0f,
        [&](int n, int d, float x) {
          if (n < nq && d < ch.D) ((Row*)a.out)[b * a.o_b + (int64_t)(h0 + n) * a.o_h + d] = from_f32<Row>(x);
        },
        [&](int n, float x) {
          if (n < nq && a.lse) a.lse[(int64_t)b * a.Hq + h0 + n] = x;
        });
    __syncwarp();  // the ring is free
  }
}

// Adds the parts of the query tiles that several blocks shared: part 1 of the block
// that the tile begins in, then part 0 of the following ones, weighed by a common
// maximum.  A block takes `side` queries of one tile, several warps each where
// there are many parts; a lane has DP / 32 components.
constexpr int kJoinWarps = 8;
template <int V>
__device__ __forceinline__ void load_part(const float* p, float (&x)[V]) {
  if constexpr (V == 2) {
    const float2 y = *reinterpret_cast<const float2*>(p);
    x[0] = y.x;
    x[1] = y.y;
  } else {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float4 y = *reinterpret_cast<const float4*>(p + j);
      x[j] = y.x;
      x[j + 1] = y.y;
      x[j + 2] = y.z;
      x[j + 3] = y.w;
    }
  }
}
template <int CT, int DP, int QT>
__global__ void __launch_bounds__(32 * kJoinWarps) k_decode_join(DecodeArgs a, int tiles, int side, const float* parts,
                                                                 const Begin* begins) {
  using S = Shape<CT, DP, QT>;
  using Row = typename Type<CT>::Row;
  constexpr int V = DP / 32;
  constexpr int kFirst = 4;  // parts that a warp loads before it knows their weights
  __shared__ float s_o[kJoinWarps][DP];
  // What follows comes to the SMs once the parts are there: while they are being
  // made, its blocks would be in their way (one scene 7.7 us a call, else 8.7).
  wait_for_stream(false);
  const Begin x = begins[blockIdx.x];
  if (x.blocks == 0) return;
  const int G = a.Hq / a.cache.heads, hk = x.col / tiles, h0 = hk * G + x.col % tiles * QT;
  const int nq = min(QT, G - x.col % tiles * QT);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int warps = kJoinWarps / side, n = min((int)blockIdx.y * side + warp / warps, nq - 1), own = warp % warps;
  auto part = [&](int i) { return parts + (2 * ((int64_t)x.block + i) + (i == 0)) * S::part; };
  float m0 = kLowest, l0 = 0.0f;  // the first 32 parts' maxima and sums are kept
  if (lane < x.blocks) {
    m0 = part(lane)[n];
    l0 = part(lane)[QT + n];
  }
  float y[kFirst][V];
#pragma unroll
  for (int k = 0; k < kFirst; ++k)
    if (own + k * warps < min(32, x.blocks)) load_part<V>(part(own + k * warps) + 2 * QT + n * DP + V * lane, y[k]);
  float top = m0;
  for (int i = 32 + lane; i < x.blocks; i += 32) top = fmaxf(top, part(i)[n]);
#pragma unroll
  for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  float f = exp2f(m0 - top), sum = l0 * f, o[V];
#pragma unroll
  for (int j = 0; j < V; ++j) o[j] = 0.0f;
#pragma unroll
  for (int k = 0; k < kFirst; ++k) {
    const int i = own + k * warps;
    const float w = __shfl_sync(~0u, f, i % 32);
    if (i < min(32, x.blocks)) {
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = fmaf(w, y[k][j], o[j]);
    }
  }
  for (int i0 = 0; i0 < x.blocks; i0 += 32) {
    if (i0 > 0) {
      const bool there = i0 + lane < x.blocks;
      f = there ? exp2f(part(i0 + lane)[n] - top) : 0.0f;
      sum += there ? part(i0 + lane)[QT + n] * f : 0.0f;
    }
    const int here = min(32, x.blocks - i0);
#pragma unroll 4
    for (int i = own + (i0 == 0 ? kFirst * warps : 0); i < here; i += warps) {
      const float w = __shfl_sync(~0u, f, i);
      float z[V];
      load_part<V>(part(i0 + i) + 2 * QT + n * DP + V * lane, z);
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = fmaf(w, z[j], o[j]);
    }
  }
  sum = warp_sum(sum);  // the same in every warp of a query
  if (warps > 1) {
#pragma unroll
    for (int j = 0; j < V; ++j) s_o[warp][V * lane + j] = o[j];
    __syncthreads();
    if (own != 0) return;
#pragma unroll
    for (int j = 0; j < V; ++j)
      for (int w = 1; w < warps; ++w) o[j] += s_o[warp + w][V * lane + j];
  }
  if ((int)blockIdx.y * side + warp / warps >= nq) return;
  const float by = sum == 0.0f ? 0.0f : (a.cache.v_scale ? a.cache.v_scale[hk] : 1.0f) / sum;
  Row* out = (Row*)a.out + x.b * a.o_b + (int64_t)(h0 + n) * a.o_h;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (V * lane + j < a.cache.D) out[V * lane + j] = from_f32<Row>(sum == 0.0f ? 0.0f : o[j] * by);
  if (lane == 0 && a.lse) a.lse[(int64_t)x.b * a.Hq + h0 + n] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// The largest clusters of which `columns` run at the same time, 2 to kMaxCluster blocks
// (1: there are none): at most `all` blocks, and no more clusters than the device
// holds, which is asked once a device and size.
template <int CT, int DP, int QT>
static int cluster_size(int64_t columns, int64_t all, int* size) {
  using S = Shape<CT, DP, QT>;
  static std::atomic<uint64_t> allowed{0};
  static std::atomic<int> held[64][5];  // a device's clusters of 2^i blocks, and one more (0: not asked yet)
  *size = 1;
  if (columns * 2 > all) return CP_OK;
  const void* kernel = (const void*)k_decode_cluster<CT, DP, QT>;
  int dev = 0;
  CP_TRY_STATUS(cuda_status(cudaGetDevice(&dev), "decode: device"));
  if (!(allowed.load(std::memory_order_acquire) >> (dev & 63) & 1))
    CP_TRY_STATUS(cuda_status(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1),
                              "decode: cluster"));
  CP_TRY_STATUS(allow_smem_once(kernel, S::smem, "decode: shared memory", &allowed));
  int most = kMaxCluster, i = 4;
  for (; most > 1; most /= 2, --i) {
    if (columns * most > all) continue;
    int n = held[dev & 63][i].load(std::memory_order_relaxed) - 1;
    if (n < 0) {
      cudaLaunchAttribute with{};
      with.id = cudaLaunchAttributeClusterDimension;
      with.val.clusterDim = {(unsigned)most, 1, 1};
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3((unsigned)most);
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = S::smem;
      cfg.attrs = &with;
      cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&n, k_decode_cluster<CT, DP, QT>, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();  // a size that the device does not take
        n = 0;
      }
      held[dev & 63][i].store(n + 1, std::memory_order_relaxed);
    }
    if (columns <= n) break;
  }
  *size = most;
  return CP_OK;
}

template <int CT, int DP, int QT>
static int launch(const DecodeArgs& a, cudaStream_t s) {
  using S = Shape<CT, DP, QT>;
  const int G = a.Hq / a.cache.heads, tiles = (G + QT - 1) / QT;
  // What a table's row or the window holds stands for the longest sequence, which only the
  // device knows: a row far wider than that goes as one line.  Exact rows / rows of 32,768
  // keys, us: one sequence of 1500 keys 6.7 / 8.2, 32 of 1229 to 1741 22.9 / 23.7, 160 of
  // 100 to 300 23.4 / 25.6, 16 of 8192 to 8704 with 15% marked 16.3 / 19.4.
  // Sequences of at most 4 units are not cut: the join would cost more.
  const int64_t most = a.window > 0 && a.window < a.cache.capacity ? a.window : a.cache.capacity;  // keys of one
  const bool cut = most > 4 * kUnit;
  const int unit = cut ? kUnit : 4 * kUnit;
  const int64_t line = (int64_t)a.B * a.cache.heads * tiles * (most < 1 ? 1 : (most + unit - 1) / unit);
  if (line > (int64_t)1 << 52) return CP_EUNSUPPORTED;  // units times blocks stay within 64 bits

  // rows of the cache in units that fit 32 bits
  const Cache& ch = a.cache;
  const uint64_t page = (uint64_t)ch.page_stride * S::e, slot = (uint64_t)ch.slot_stride * S::e;
  int shift = 4;
  while (shift < 31 && (page | slot) != 0 && ((page | slot) >> shift & 1) == 0) ++shift;
  const uint64_t far = (uint64_t)(ch.pages > 0 ? ch.pages - 1 : 0) * (page >> shift) +
                       (uint64_t)(ch.page_size - 1) * (slot >> shift);
  if (far > 0xFFFFFFFFu) return CP_EUNSUPPORTED;
  Rows rows{(uint32_t)(page >> shift), (uint32_t)(slot >> shift), (uint32_t)1 << shift, 0, 0};
  while (((int64_t)1 << rows.div_shift) < ch.page_size) ++rows.div_shift;
  rows.mul = (uint32_t)((((uint64_t)1 << (31 + rows.div_shift)) + ch.page_size - 1) / ch.page_size);

  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  int64_t grid = (int64_t)di.sm_count * S::per_sm;
  if (grid > kDecodeBlocks) grid = kDecodeBlocks;
  const int64_t all = grid;
  if (grid > line) grid = line;
  const int64_t columns = (int64_t)a.B * ch.heads * tiles;
  const bool by_column = columns <= grid;
  Begin* begins = (Begin*)a.ws;
  float* parts = (float*)((char*)a.ws + kDecodeBlocks * sizeof(Begin));
  static std::atomic<uint64_t> allowed{0};
  CP_TRY_STATUS(allow_smem_once((const void*)k_decode<CT, DP, QT>, S::smem, "decode: shared memory", &allowed));
  // Many short sequences: a warp a query tile, up to 64 keys for every third of the
  // blocks' number that there are tiles, and 64 more.  us with blocks / with warps,
  // 7 queries a head of 128: 320 tiles of up to 300 keys 17 / 16, of 500 18 / 26; 640
  // of 300 26 / 17, of 500 38 / 38, of 1000 62 / 69; 1600 of 300 46 / 28, of 500 79 /
  // 65, of 1000 138 / 122; 8 bits: 640 of 500 30 / 27, of 1000 45 / 50; 1600 of 1000
  // 97 / 67.  Longer ones have not been measured.  float32 computes longer on a key: up
  // to 48 keys for every blocks' number that there are tiles; 320 of 300 keys 39 / 40, 468 of up to 155
  // 30 / 36, 640 of 64 27 / 22, of 300 68 / 80, 1600 of 150 100 / 85, of up to 300 103 /
  // 128, 6400 (heads of 64) of 300 240 / 178, of 900 582 / 491.
  // Of marked keys, which may be few, twice that (float32: five times): 10% / 50% marked,
  // 1000 tiles of up to 1000 keys 31 / 16, 50 / 48, 8 bits 30 / 14, 45 / 35, float32 of up
  // to 600 41 / 24, 89 / 81; beyond it what some gain others lose: 1000 of up to 2000 37 /
  // 31, 76 / 90, float32 of up to 1000 50 / 34, 122 / 129.
  // Few tiles too, when two tiles of keys (one of float32) are all there is: one sequence
  // of 4 tiles and 16 keys 5.5 / 3.8, of 50 5.5 / 6.2; 60 of 4, 16 keys 6.5 / 4.1, 50 keys
  // 7.2 / 6.5; float32, 8 keys 8.9 / 7.4, 16 keys 9.0 / 8.6 and, for one sequence, 7.9 /
  // 8.2.
  constexpr int kFew = CT == CP_F32 ? 8 : 32;
  const int64_t reach = CT == CP_F32 ? (a.keep ? 240 : 48) * columns : (a.keep ? 2 : 1) * kUnit * (3 * columns + all);
  if (most <= kFew || (columns > all && most <= (a.keep ? 32 : 16) * kUnit && most * all <= reach)) {
    using Short = Shape<CT, DP, QT, true>;
    static std::atomic<uint64_t> short_allowed{0};
    CP_TRY_STATUS(allow_smem_once((const void*)k_decode_short<CT, DP, QT>, Short::smem, "decode: shared memory",
                                  &short_allowed));
    const int64_t room = (int64_t)di.sm_count * Short::per_sm, wanted = (columns + kWarps - 1) / kWarps;
    return cuda_status(launch_early(k_decode_short<CT, DP, QT>, dim3((unsigned)(wanted < room ? wanted : room)), kThreads,
                                    Short::smem, s, a, rows, tiles, columns),
                       "decode: short");
  }
  // Few query tiles: a cluster each, if all run at once.  That saves 4 us of joining,
  // and costs what the blocks that get no tile would have done (at most 8 units' time
  // a block) and, where sequences differ in length more than the table's width
  // tells, the longest one's time: at most 16 units a block, of marked keys thrice
  // that.  us as one line / with clusters, 7 queries a head of 128: 4 tiles of 500 keys
  // 7.5 / 6.0, of 1500 7.7 / 6.7, of 8000 15.2 / 11.1, of 16000 16.2 / 17.3; 64 of 1500
  // 15.4 / 11.3, of 4000 29.9 / 26.2, of 8000 with 15% marked 19.8 / 16.2; 128 of 1229
  // to 1741 24.1 / 22.8.
  // float32 computes longer on a unit: half of the longest one's time and a quarter of
  // what idles; 64 tiles of 500 to 3000 keys 46 / 67 (heads of 256), 27 / 34 (128), 19 /
  // 25 (64), of 1500 41 / 40, 23.2 / 21.4, 17.4 / 15.7; 4 of 4000 16.1 / 19.5, 12.3 / 12.6,
  // 10.6 / 11.6, of 1500 12.0 / 11.0, 9.3 / 8.2, 8.1 / 7.4.
  const int64_t n64 = (most + kUnit - 1) / kUnit;
  int size = 0;
  if (cut) CP_TRY_STATUS((cluster_size<CT, DP, QT>(columns, all, &size)));
  const bool slow = CT == CP_F32 && !a.keep;
  if (size > 1 && n64 <= (a.keep ? 48 : slow ? 8 : 16) * size &&
      n64 * (all - columns * size) <= (slow ? 2 : 8) * size * all)
    return cuda_status(launch_early_cluster(k_decode_cluster<CT, DP, QT>, dim3((unsigned)(columns * size)), kThreads, S::smem,
                                            s, size, a, rows, tiles, size),
                       "decode: cluster");
  CP_TRY_STATUS(cuda_status(launch_early(k_decode<CT, DP, QT>, dim3((unsigned)grid), kThreads, S::smem, s, a, rows, unit,
                                         tiles, parts, cut ? begins : nullptr, (int)by_column),
                            "decode"));
  if (!cut) return CP_OK;
  // about so many parts a query tile, and the join's queries side by side for it
  const int64_t share = grid / columns + 1;
  const int queries = G < QT ? G : QT;
  int side = share <= 4 ? 8 : share <= 12 ? 2 : 1;
  while (side > 1 && side / 2 >= queries) side /= 2;
  const dim3 joins((unsigned)(by_column ? columns : grid), (unsigned)(queries + side - 1) / side);
  return cuda_status(launch_early(k_decode_join<CT, DP, QT>, joins, 32 * kJoinWarps, 0, s, a, tiles, side, parts, begins),
                     "decode: join");
}

template <int CT, int DP>
static int launch_pass(const DecodeArgs& a, cudaStream_t s) {
  constexpr int one = CT == CP_F32 ? 4 : 8;
  return decode_pass(CT, a.Hq / a.cache.heads) == one ? launch<CT, DP, one>(a, s) : launch<CT, DP, 2 * one>(a, s);
}
template <int CT>
static int launch_type(const DecodeArgs& a, cudaStream_t s) {
  switch (decode_width(a.cache.D)) {
    case 64: return launch_pass<CT, 64>(a, s);
    case 128: return launch_pass<CT, 128>(a, s);
    default: return launch_pass<CT, 256>(a, s);
  }
}

}  // namespace cp
