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
//
// A 4-bit cache is bound by instructions: of the 850 of a warp for 32 keys (head 128, 8 queries) 450 turn 4 bits and
// scales into float16 operands (14 for 8 numbers: a mask and a fused product each two, their scale), and
// the SM's four schedulers issue 2.4 a cycle together however many warps there are.  32 sequences of 8192 to 8704
// keys 47.7 us (0.48 of the HBM's rate), the copies alone 34, all but the copies 43.
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
template <> struct Maximum<CP_I4> : Maximum<CP_E4M3> {};
// A maximum before any score: finite, so that differences of two are, and below no
// finite score (of weight 1 beside it).
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// What a cache's type changes: keys a tile (a lane has a key's page and row, so 32 at
// most), the type of queries and outputs.
template <int CT> struct Type;
template <> struct Type<CP_BF16> { static constexpr int tk = 16; using Row = __nv_bfloat16; };
template <> struct Type<CP_E4M3> { static constexpr int tk = 16; using Row = __nv_bfloat16; };
template <> struct Type<CP_I4> { static constexpr int tk = 32; using Row = __nv_bfloat16; };
template <> struct Type<CP_F32> { static constexpr int tk = 8; using Row = float; };

// Shape of one variant: CT cache type, DP head width it is laid out for, QT query
// heads a pass, SHORT whether each warp has sequences of its own (k_decode_short).
template <int CT, int DP, int QT, bool SHORT = false>
struct Shape {
  // Keys of a tile: 4 of float32 heads of 256, whose rings leave room for two blocks then:
  // 102 sequences of 574 to 1149 keys and 6 query tiles 242 us, with 8 keys and one block
  // 283; 47 of up to 125 15.0, 18.3.
  static constexpr int tk = CT == CP_F32 && DP == 256 ? 4 : Type<CT>::tk;
  static constexpr uint32_t all = tk == 32 ? ~0u : (1u << tk % 32) - 1;  // every key of a tile
  static constexpr int row = (int)cache_bytes(CT, DP);  // bytes of a row in shared memory
  static constexpr int cpr = row / 16;                // 16-byte chunks of it
  static constexpr int sb = CT == CP_I4 ? DP / 16 : 0;  // bytes of its scales
  static constexpr int tile = 2 * tk * (row + sb);    // K and V of a tile, and their scales
  // Ring: as many tiles as keep two blocks on an SM, 3 at least.  Three blocks of
  // shorter rings leave the join no room beside them and wait longer: 128 ragged
  // 8-bit sequences 101 us with two, 115 with three; four 125.
  // Short sequences: three blocks, as registers allow, as there is more to begin
  // than to copy.
  // 4 bits: instructions bound it, and 2, 3 and 4 blocks of 128 threads do 32 sequences of 8448 keys in 48.6, 47.8
  // and 49.7 us.  (100 KB, not 112, leave two blocks of 16 queries and heads of 128 room for the keys whose scores they leave behind:
  // 32 sequences of 8448 keys, 64 heads and weights 91 us, by one block 128.)
  static constexpr int blocks = CT != CP_I4 ? (SHORT ? 3 : 2) : DP == 256 || (DP == 128 && QT == 16) ? 2 : DP == 128 || QT == 16 ? 3 : 4;
  static constexpr int bound = CT == CP_I4 ? blocks : 0;  // of the registers
  static constexpr int room = CT != CP_I4 ? (SHORT ? 64 : 100) : blocks == 4 ? 50 : blocks == 3 ? 68 : DP == 256 ? 112 : 100;  // KB of a block
  static constexpr int fit = room * 1024 / (kWarps * tile);
  static constexpr int least = SHORT || CT == CP_I4 ? 2 : 3;
  static constexpr int stages = fit < least ? least : fit > 8 ? 8 : fit;
  static constexpr int ring = kWarps * stages * tile;
  // float32 queries, the block's or each warp's, and each warp's weights of a tile
  static constexpr int queries = SHORT ? kWarps : 1;
  static constexpr int extra = CT == CP_F32 ? (queries * QT * DP + kWarps * tk * QT) * 4 : 0;
  static constexpr int smem = ring + extra;
  // (Registers allow them but for some spills, 4 to 32 bytes of stores a thread: 4 and 8 bits' heads of
  // 64, float32's of 128 and 256, 4 bits' of 256 with weights.  Heads of 256 with 16 queries, whose outputs
  // and queries are 192 registers, spill more: 16 to 108 bytes of 16 or 8 bits, of 4 bits, where decoding
  // needs its own, 248 to 516, and wait for that: 16 sequences of 8448 keys and 2 heads 52 us, with 8 queries 31.)
  static constexpr int per_sm = CT == CP_I4 ? blocks
                                : SHORT && smem <= 70 * 1024 ? 3 : smem <= 110 * 1024 ? 2 : 1;
  static constexpr int part = QT * (DP + 2);  // floats of a partial result
  // What beginning and merging a segment costs, in units of 64 keys: about 3 us, in
  // which a block takes 72 KB (of 4 bits, which take longer to decode, less: 128 ragged
  // sequences of heads of 128 with 0, 2, 4 and 9 units 84.4, 82.6, 81.4, 83.1 us; of 4 heads of 64 117, 111, 108, 103, of
  // 8 with 2 queries each 192, 188, 187, 189).
  static constexpr int setup = CT == CP_I4 ? (DP == 64 ? 9 : 4) : 72 * 1024 / (2 * kUnit * row) < 1 ? 1 : 72 * 1024 / (2 * kUnit * row);
  static constexpr int pitch = DP + 4;        // floats of a query in the merge: the lanes' banks differ
  static_assert(SHORT || (kWarps * pitch + DP) * QT * 4 <= ring, "the merge reuses the ring");
  static_assert(sb == 0 || tk == 32, "a lane copies the scales of a key");
};

// Rows of the cache in 32 bits: row r of page p starts (p * page + r * slot) << shift
// bytes into K and V.
// Its scales start (p * block_page + r * block_slot) * 4 bytes into theirs, and are copied
// `piece` bytes at a time.
struct Rows {
  uint32_t page, slot;
  uint32_t scale;  // 1 << shift
  uint32_t mul, div_shift;  // key / page_size = key * mul >> 31 >> div_shift
  uint32_t block_page, block_slot;
  int piece;
};

// Where a chunk of a row lies, chunk c at c ^ swizzle(r): rows that are read
// together fall on other banks.  Bits of r only, so that swizzle(r ^ s) is
// swizzle(r) ^ swizzle(s).
template <int CT, int CPR>
__host__ __device__ constexpr int swizzle(int r) {
  return CT == CP_F32 ? (r & 1) << 2 : CPR >= 8 ? r & 7 : CPR == 4 ? (r >> 1) & 3 : (r >> 2) & 1;
}

// 16 bytes of a row; L2 fetches the 128 around them (which marked keys of 32-byte rows do not fill, at no cost: 2 sequences of
// 180,876 keys with 15% marked 36 us with the hint and without).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  const int n = there ? 16 : 0;  // 0: nothing is read, zeros are written
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// 4, 8 or 16 bytes, or as many zeros.
template <int BYTES>
__device__ __forceinline__ void copy_few(uint32_t dst, const void* src, bool there) {
  const int n = there ? BYTES : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
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
// Numbers n + 8 in bits 4-7 of each half of x become n s in float16: 64 + n + 8 is a float16 as its bits
// are, and (72 + n) s - 72 s rounds once to what float16 holds exactly; `off` is -72 s.
__device__ __forceinline__ uint32_t i4_f16x2(uint32_t x, uint32_t s, uint32_t off) {
  uint32_t y;
  asm("{\n\t.reg .b32 a;\n\tlop3.b32 a, %1, 0x00F000F0, 0x54005400, 0xEA;\n\tfma.rn.f16x2 %0, a, %2, %3;\n\t}"
      : "=r"(y)
      : "r"(x), "r"(s), "r"(off));
  return y;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t y;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
constexpr uint32_t kOff = 0xD480D480u;  // -72
// Bytes of a and b picked by `sel`, as two 8-bit elements, in float16 (exact).
__device__ __forceinline__ uint32_t scales_f16x2(uint32_t a, uint32_t b, uint32_t sel) {
  uint32_t y;
  asm("{\n\t.reg .b32 p;\n\t.reg .b16 l, h;\n\tprmt.b32 p, %1, %2, %3;\n\tmov.b32 {l, h}, p;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\t}"
      : "=r"(y)
      : "r"(a), "r"(b), "r"(sel));
  return y;
}
__device__ __forceinline__ uint32_t load_shared(uint32_t at) {
  uint32_t y;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(y) : "r"(at) : "memory");
  return y;
}
// N words of a 4-bit row's scales.
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], uint32_t at) {
  if constexpr (N == 1) {
    w[0] = load_shared(at);
  } else if constexpr (N == 2) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  } else {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(at)
                 : "memory");
  }
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

// Where the scores of a segment's tiles go, for those who add the weights up by them:
// `to` is key 0's, pitch floats a key (1 or even); `keys` the tile's, -1 for none.
struct NoScores {
  static constexpr bool on = false;
};
struct Scores {
  static constexpr bool on = true;
  float* to;
  int pitch;
  const int* keys;
  __device__ __forceinline__ void put(int row, uint32_t valid, int query, float s) const {
    const int key = keys[row];  // one on a bad page weighs nothing
    if (key >= 0 && query < pitch) to[(int64_t)key * pitch + query] = valid >> row & 1 ? s : -INFINITY;
  }
  // Of an even query and the next: 8 keys and 4 such pairs of a warp fill whole sectors.
  __device__ __forceinline__ void put(int row, uint32_t valid, int query, float s0, float s1) const {
    const int key = keys[row];
    if (key < 0 || query >= pitch) return;
    if (!(valid >> row & 1)) s0 = s1 = -INFINITY;
    if (pitch == 1)
      to[key] = s0;
    else
      *reinterpret_cast<float2*>(to + (int64_t)key * pitch + query) = make_float2(s0, s1);
  }
};

// A warp's running softmax and output of one segment on the tensor cores.
// Lane (g, t) = (lane / 4, lane % 4) has the scores of keys g and g + 8 (of a tile's every 16) and
// queries 2 t, 2 t + 1 of each group of 8, and the same queries' outputs at
// components 16 i + g, + 8 (8-bit caches: 16 i + 2 g, + 1; 4-bit ones: as component() says).
// A 4-bit element enters as n s, which float16 holds exactly (5 bits times 4), its scale's byte
// turned into float16 as well.
template <int CT, int DP, int QT, bool SHORT>
struct Math {
  using S = Shape<CT, DP, QT, SHORT>;
  static constexpr int NT = QT / 8, KS = DP / 16;
  static constexpr int H = S::tk / 16;       // groups of 16 keys in a tile
  static constexpr int SW = DP < 64 ? 1 : DP / 64;  // words of a 4-bit row's scales
  uint32_t q[NT][KS][2];
  float o[NT][KS][4];
  float m[NT][2], l[NT][2];
  float sc[NT][2];  // score = sc * product, in units of log 2
  int g, t;
  uint32_t k_at, v_at;  // this lane's rows in a tile's K and V, first chunk: chunk c is ^ 16 c
  int half_word;        // the word of a 4-bit row's scales whose upper half is padding; -1: none

  // The component of o[n][k]'s row g (half 0) or g + 8 (half 1).
  __device__ __forceinline__ int component(int k, int half) const {
    if (CT == CP_BF16) return 16 * k + g + 8 * half;
    if (CT == CP_E4M3) return 16 * k + 2 * g + half;
    return 32 * (k / 2) + 4 * g + 2 * (k % 2) + half;
  }

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
    half_word = D % 64 != 0 ? D / 64 : -1;  // whose padding might be a NaN
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
          // (4 bits: pairs 4 t .. 4 t + 3 of 32 components, put in order below)
          const int d = CT == CP_I4 ? 32 * (s / 2) + 8 * t + 4 * (s % 2) + 2 * i
                                    : 16 * s + (CT == CP_E4M3 ? 4 * t + 2 * i : 2 * t + 8 * i);
          uint32_t x = 0;
          if (row_there && d < D) {
            if (pairs)
              x = *(const uint32_t*)(src + d);
            else
              x = src[d] | (uint32_t)src[d + 1] << 16;
          }
          q[n][s][i] = x;
        }
      if (CT == CP_I4) {
        // a word of a row has components 0 to 7 in its eight places; two at a time come out
        // of it, four places apart
#pragma unroll
        for (int s = 0; s < KS; s += 2) {
          const uint32_t w0 = q[n][s][0], w1 = q[n][s][1], w2 = q[n][s + 1][0], w3 = q[n][s + 1][1];
          q[n][s][0] = __byte_perm(w0, w2, 0x5410);
          q[n][s][1] = __byte_perm(w0, w2, 0x7632);
          q[n][s + 1][0] = __byte_perm(w1, w3, 0x5410);
          q[n][s + 1][1] = __byte_perm(w1, w3, 0x7632);
        }
      }
      int ex = 0;
      if (CT != CP_BF16) {
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
        if (CT != CP_BF16) sc[n][i] *= power(__shfl_sync(~0u, ex, 4 * (2 * t + i)));
        m[n][i] = kLowest;
        l[n][i] = 0.0f;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][s][i] = 0.0f;
    }
  }

  template <typename Score>
  __device__ __forceinline__ void tile(uint32_t at, uint32_t valid, char*, int, int, const Score& scores) {
    float s[H][NT][4];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int n = 0; n < NT; ++n) s[h][n][0] = s[h][n][1] = s[h][n][2] = s[h][n][3] = 0.0f;
    if (CT == CP_BF16) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t x[4];
        ldmatrix4(x, (at + k_at) ^ (32 * k));
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16_16816(s[0][n], x[0], x[1], x[2], x[3], q[n][k][0], q[n][k][1]);
      }
    } else if (CT == CP_E4M3) {
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
          for (int n = 0; n < NT; ++n) mma_f16_16816(s[0][n], a0, a1, a2, a3, q[n][k + j][0], q[n][k + j][1]);
        }
      }
    } else {
      // scales of keys g and g + 8; a lane's word of chunk c is of components 32 c + 8 t to + 7, one scale
      uint32_t lo[H][SW], hi[H][SW];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        load_words<SW>(lo[h], at + 2 * S::tk * S::row + (16 * h + g) * S::sb);
        load_words<SW>(hi[h], at + 2 * S::tk * S::row + (16 * h + g + 8) * S::sb);
        if (half_word >= 0) {
#pragma unroll
          for (int w = 0; w < SW; ++w) {
            lo[h][w] &= w == half_word ? 0xFFFFu : ~0u;
            hi[h][w] &= w == half_word ? 0xFFFFu : ~0u;
          }
        }
      }
      // (the groups of keys in turn, so that two products in a row do not wait for one another)
#pragma unroll
      for (int c = 0; c < DP / 32; c += 2) {
        uint32_t x[H][4];
#pragma unroll
        for (int h = 0; h < H; ++h) ldmatrix4(x[h], (at + 16 * h * S::row + k_at) ^ (16 * c));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t sel = (2 * j + t / 2) * 0x11;
          uint32_t s0[H], s1[H], o0[H], o1[H];
#pragma unroll
          for (int h = 0; h < H; ++h) {
            s0[h] = scales_f16x2(lo[h][c / 2], 0, sel);
            s1[h] = scales_f16x2(hi[h][c / 2], 0, sel);
            o0[h] = mul_f16x2(s0[h], kOff);
            o1[h] = mul_f16x2(s1[h], kOff);
          }
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < H; ++h) {
              const uint32_t w0 = x[h][2 * j] >> 8 * m, w1 = x[h][2 * j + 1] >> 8 * m;
              const uint32_t a0 = i4_f16x2(w0 * 16, s0[h], o0[h]), a1 = i4_f16x2(w1 * 16, s1[h], o1[h]);
              const uint32_t a2 = i4_f16x2(w0, s0[h], o0[h]), a3 = i4_f16x2(w1, s1[h], o1[h]);
#pragma unroll
              for (int n = 0; n < NT; ++n)
                mma_f16_16816(s[h][n], a0, a1, a2, a3, q[n][2 * (c + j) + m][0], q[n][2 * (c + j) + m][1]);
            }
        }
      }
    }
    if constexpr (Score::on) {
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; i += 2)
            scores.put(16 * h + g + 4 * i, valid, 8 * n + 2 * t, s[h][n][i] * sc[n][0], s[h][n][i + 1] * sc[n][1]);
    }
    const bool full = valid == S::all;
    if (!full) {
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)  // scores are multiplied by sc, of either sign, next
            if (!(valid >> (16 * h + g + 8 * (i / 2)) & 1)) s[h][n][i] = __int_as_float(0x7fffffff);
    }
    // the largest of this lane's scores of a query; fmaxf passes over the NaN of a key that is not there
    auto most = [&](int n, int i) {
      float x = fmaxf(s[0][n][i] * sc[n][i], s[0][n][i + 2] * sc[n][i]);
#pragma unroll
      for (int h = 1; h < H; ++h) x = fmaxf(x, fmaxf(s[h][n][i] * sc[n][i], s[h][n][i + 2] * sc[n][i]));
      return x;
    };
    bool above = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) above |= most(n, i) > m[n][i] + Maximum<CT>::slack;
    if (__any_sync(~0u, above)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float top = fmaxf(most(n, i) - Maximum<CT>::under, m[n][i]);
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
    uint32_t p[H][NT][2], rest[NT][2];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = exp2_fast(fmaf(s[h][n][i], sc[n][i & 1], -m[n][i & 1]));
        if (!full) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(valid >> (16 * h + g + 8 * (i / 2)) & 1)) x[i] = 0.0f;
        }
        l[n][0] += x[0] + x[2];
        l[n][1] += x[1] + x[3];
        // A weight goes on in 11 bits beside an 8- or 4-bit cache, float16's (see Maximum).  bfloat16's 8 would
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
          p[h][n][0] = movmatrix_trans(__byte_perm(below[0], below[1], 0x7632));
          p[h][n][1] = movmatrix_trans(__byte_perm(below[2], below[3], 0x7632));
          rest[n][0] = movmatrix_trans(pack_bf16(left[0], left[1]));
          rest[n][1] = movmatrix_trans(pack_bf16(left[2], left[3]));
        } else {
          p[h][n][0] = movmatrix_trans(pack_f16(x[0], x[1]));
          p[h][n][1] = movmatrix_trans(pack_f16(x[2], x[3]));
        }
      }
    const uint32_t blocks = at + (2 * S::row + S::sb) * S::tk;  // V's scales
    at += S::tk * S::row;
    if (CT == CP_BF16) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t x[4];
        ldmatrix4_trans(x, (at + v_at) ^ (32 * k));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_bf16_16816(o[n][k], x[0], x[1], x[2], x[3], p[0][n][0], p[0][n][1]);
          mma_bf16_16816(o[n][k], x[0], x[1], x[2], x[3], rest[n][0], rest[n][1]);
        }
      }
    } else if (CT == CP_E4M3) {
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
          for (int n = 0; n < NT; ++n) mma_f16_16816(o[n][k + j], a0, a1, a2, a3, p[0][n][0], p[0][n][1]);
        }
      }
    } else {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        // scales of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        uint32_t ks[4][SW];
#pragma unroll
        for (int i = 0; i < 4; ++i) load_words<SW>(ks[i], blocks + (16 * h + 2 * t + i % 2 + 8 * (i / 2)) * S::sb);
#pragma unroll
        for (int c = 0; c < DP / 32; c += 2) {
          uint32_t x[4];
          ldmatrix4_trans(x, (at + 16 * h * S::row + v_at) ^ (16 * c));
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // halves: key 2 t's components 4 g to 4 g + 3, key 2 t + 1's; one scale a key
            const uint32_t sel = 0x40 + (2 * j + g / 4) * 0x11;
            const uint32_t s0 = scales_f16x2(ks[0][c / 2], ks[1][c / 2], sel);
            const uint32_t s1 = scales_f16x2(ks[2][c / 2], ks[3][c / 2], sel);
            const uint32_t o0 = mul_f16x2(s0, kOff), o1 = mul_f16x2(s1, kOff);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              const uint32_t w0 = x[2 * j] >> 8 * m, w1 = x[2 * j + 1] >> 8 * m;
              const uint32_t a0 = i4_f16x2(w0 * 16, s0, o0), a1 = i4_f16x2(w0, s0, o0);
              const uint32_t a2 = i4_f16x2(w1 * 16, s1, o1), a3 = i4_f16x2(w1, s1, o1);
#pragma unroll
              for (int n = 0; n < NT; ++n) mma_f16_16816(o[n][2 * (c + j) + m], a0, a1, a2, a3, p[h][n][0], p[h][n][1]);
            }
          }
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
          out(query, component(k, 0), l[n][i] == 0.0f ? 0.0f : o[n][k][i] * by);
          out(query, component(k, 1), l[n][i] == 0.0f ? 0.0f : o[n][k][i + 2] * by);
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
          buf[query * S::pitch + component(k, i / 2)] = o[n][k][i] * f[query];
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

  template <typename Score>
  __device__ __forceinline__ void tile(uint32_t at, uint32_t valid, char* extra, int warp, int lane,
                                       const Score& scores) {
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
      if constexpr (Score::on)
        if (sub == n % L) scores.put(r, valid, n, s[n] * sc);
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
template <int CT, int DP, int QT, bool SHORT, bool SCORES, typename K>
__device__ __forceinline__ void math_of_keys(const DecodeArgs& a, const Rows& rows, K& keys, const int32_t* table, int lo,
                                             int hi, int hk, int b, int col, int h0, int nq, int warp, int lane, uint32_t ring,
                                             uint32_t* s_valid, int* s_keys, char* extra, Math<CT, DP, QT, SHORT>& math) {
  using S = Shape<CT, DP, QT, SHORT>;
  const Cache& ch = a.cache;
  const int chunks = (int)cache_bytes(CT, ch.D) / 16;  // of a row that is there
  const char* kp = (const char*)ch.k + cache_bytes(CT, (int64_t)hk * ch.head_stride);
  const char* vp = (const char*)ch.v + cache_bytes(CT, (int64_t)hk * ch.head_stride);
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
      if (SCORES && lane < S::tk) s_keys[slot * S::tk + lane] = key;
      if constexpr (CT == CP_I4) {  // a lane copies the scales of its own key
        const uint64_t off = ok ? (uint64_t)((uint32_t)page * rows.block_page + (uint32_t)slot_of * rows.block_slot) * 4 : 0;
        const uint8_t* kb = ch.k_block + (int64_t)hk * ch.block_head + off;
        const uint8_t* vb = ch.v_block + (int64_t)hk * ch.block_head + off;
        const uint32_t at = ring + slot * S::tile + 2 * S::tk * S::row + lane * S::sb;
        if (S::sb >= 8 && rows.piece == S::sb) {
          copy_few<(S::sb >= 8 ? S::sb : 4)>(at, kb, ok);
          copy_few<(S::sb >= 8 ? S::sb : 4)>(at + S::tk * S::sb, vb, ok);
        } else {
          const int there = block_bytes(ch.D);
#pragma unroll
          for (int i = 0; i < S::sb; i += 4) {  // what lies beyond the row's becomes 0
            const bool real = ok && i < there;
            copy_few<4>(at + i, kb + (real ? i : 0), real);
            copy_few<4>(at + S::tk * S::sb + i, vb + (real ? i : 0), real);
          }
        }
      }
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
      if (valid == S::all && chunks == S::cpr) {
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
    if constexpr (SCORES)
      math.tile(ring + slot * S::tile, s_valid[slot], extra, warp, lane,
                Scores{a.scores + ((int64_t)b * a.score_cols + col) * ch.capacity * a.score_pitch, a.score_pitch,
                       s_keys + slot * S::tk});
    else
      math.tile(ring + slot * S::tile, s_valid[slot], extra, warp, lane, NoScores{});
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

template <int CT, int DP, int QT, bool SCORES>
__global__ void __launch_bounds__(kThreads, Shape<CT, DP, QT>::bound) k_decode(DecodeArgs a, Rows rows, int unit, int tiles, float* parts,
                                                     Begin* begins, int by_column, int lines_of) {
  using S = Shape<CT, DP, QT>;
  using Row = typename Type<CT>::Row;
  extern __shared__ __align__(1024) char smem[];  // addresses of rows are put together by exclusive or
  __shared__ int s_queue[kWarps][kQueue];
  __shared__ uint32_t s_valid[kWarps][S::stages];
  __shared__ int s_keys[kWarps][SCORES ? S::stages * S::tk : 1];
  __shared__ float s_m[kWarps][QT], s_l[kWarps][QT], s_f[kWarps][QT], s_top[QT], s_sum[QT];
  wait_for_stream();
  const Cache& ch = a.cache;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  // With `lines` a column has a line of its own, and every lines-th block: the blocks that run together
  // then read the same keys of different heads, whose rows share what the memory gives at a time.
  const int lines = CT == CP_I4 ? lines_of : 1;
  const int G = a.Hq / ch.heads, every = ch.heads * tiles, cols = lines > 1 ? 1 : every;
  const int place = (int)(blockIdx.x / lines), places = (int)(gridDim.x / lines);  // of the line

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
  const int setup = total >= 8 * (int64_t)places ? S::setup : 0;
  total += (int64_t)setup * a.B * cols;
  const int64_t blocks = min((int64_t)places, total);  // each of these has a unit at least
  if (begins && !by_column && threadIdx.x == 0) begins[blockIdx.x] = Begin{0, 0, 0, 0};
  if (place >= blocks) return;
  // the first `longer` of them one more than the others
  const int64_t share = quotient(total, blocks), longer = total - share * blocks;
  int64_t u = share * place + min((int64_t)place, longer);
  const int64_t end = u + share + (place < longer);
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
      const int turn = (int)quotient(u - before, long_nu), col = lines > 1 ? (int)(blockIdx.x % lines) : turn;
      const int64_t at = before + (int64_t)turn * long_nu + setup;  // its unit 0
      const int k0 = (int)max(u - at, (int64_t)0), k1 = (int)min((int64_t)nu, end - at);
      u = min(end, at + nu);
      if (k1 <= 0) continue;  // the block ends before unit 0
      const int hk = col / tiles, h0 = hk * G + col % tiles * QT;
      const int nq = min(QT, G - col % tiles * QT);
      const int lo = first + k0 * unit, hi = (int)min((int64_t)len, first + (int64_t)k1 * unit);
      Math<CT, DP, QT, false> math;
      math_of_keys<CT, DP, QT, false, SCORES>(a, rows, keys, table, lo, hi, hk, b, col, h0, nq, warp, lane, ring, s_valid[warp],
                                              s_keys[warp], extra, math);
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
        begins[by_column ? b * every + col : (int)blockIdx.x] =
            Begin{(int)blockIdx.x, whole ? 0 : to - place + 1, b, col};
      }
      __syncthreads();  // the ring and the sums are free
    }
    before += (int64_t)long_nu * cols;
  }
}

// Few query tiles of a few units a block: a cluster of blocks shares each, and adds its
// parts from one another's shared memory, an element a thread, so that no launch has
// to follow.
template <int CT, int DP, int QT, bool SCORES>
__global__ void __launch_bounds__(kThreads, Shape<CT, DP, QT>::bound) k_decode_cluster(DecodeArgs a, Rows rows, int tiles, int size) {
  using S = Shape<CT, DP, QT>;
  using Row = typename Type<CT>::Row;
  extern __shared__ __align__(1024) char smem[];
  __shared__ int s_queue[kWarps][kQueue];
  __shared__ uint32_t s_valid[kWarps][S::stages];
  __shared__ int s_keys[kWarps][SCORES ? S::stages * S::tk : 1];
  // the warps' maxima, sums and factors, then the blocks' weights (two blocks of 4-bit heads of 256 have no 500 bytes more)
  __shared__ union {
    float warps[3][kWarps][QT];
    float blocks[QT][kMaxCluster];
  } s_by;
  auto& s_m = s_by.warps[0];
  auto& s_l = s_by.warps[1];
  auto& s_f = s_by.warps[2];
  auto& s_w = s_by.blocks;
  __shared__ float s_top[QT], s_sum[QT];  // this block's, for the others
  __shared__ float s_all[QT];             // the whole sum
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
  math_of_keys<CT, DP, QT, false, SCORES>(a, rows, keys, ch.table + (int64_t)b * ch.table_stride, lo, hi, hk, b, col, h0, nq, warp,
                                          lane, smem_addr(smem) + warp * S::stages * S::tile, s_valid[warp], s_keys[warp],
                                          smem + S::ring, math);
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
template <int CT, int DP, int QT, bool SCORES>
__global__ void __launch_bounds__(kThreads, Shape<CT, DP, QT, true>::bound) k_decode_short(DecodeArgs a, Rows rows, int tiles, int64_t columns) {
  using S = Shape<CT, DP, QT, true>;
  using Row = typename Type<CT>::Row;
  extern __shared__ __align__(1024) char smem[];
  __shared__ int s_queue[kWarps][kQueue];
  __shared__ uint32_t s_valid[kWarps][S::stages];
  __shared__ int s_keys[kWarps][SCORES ? S::stages * S::tk : 1];
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
    math_of_keys<CT, DP, QT, true, SCORES>(a, rows, keys, ch.table + (int64_t)b * ch.table_stride, first, len, hk, b, col, h0, nq,
                                           warp, lane, ring, s_valid[warp], s_keys[warp], smem + S::ring, math);
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
                                                                 const Begin* begins, int lines_of) {
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
  const int lines = CT == CP_I4 ? lines_of : 1;  // from one of a tile's blocks to the next
  auto part = [&](int i) { return parts + (2 * ((int64_t)x.block + i * lines) + (i == 0)) * S::part; };
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

template <int CT, int DP, int QT>
int launch_join(const DecodeArgs& a, dim3 joins, int tiles, int side, const float* parts, const Begin* begins, int lines, cudaStream_t s) {
  return cuda_status(launch_early(k_decode_join<CT, DP, QT>, joins, 32 * kJoinWarps, 0, s, a, tiles, side, parts, begins, lines),
                     "decode: join");
}
// The joins of a type are compiled in one of its translation units (WHERE: nothing) and used from the other, whose variants leave
// the scores behind (WHERE: extern).
#define CP_JOIN(WHERE, CT, DP, QT) \
  WHERE template int launch_join<CT, DP, QT>(const DecodeArgs&, dim3, int, int, const float*, const Begin*, int, cudaStream_t);
#define CP_JOINS(WHERE, CT, FEW, MANY)                                                                             \
  CP_JOIN(WHERE, CT, 64, FEW) CP_JOIN(WHERE, CT, 64, MANY) CP_JOIN(WHERE, CT, 128, FEW) CP_JOIN(WHERE, CT, 128, MANY) \
  CP_JOIN(WHERE, CT, 256, FEW) CP_JOIN(WHERE, CT, 256, MANY)

// The largest clusters of which `columns` run at the same time, 2 to kMaxCluster blocks
// (1: there are none): at most `all` blocks, and no more clusters than the device
// holds, which is asked once a device and size.
template <int CT, int DP, int QT, bool SCORES>
static int cluster_size(int64_t columns, int64_t all, int* size) {
  using S = Shape<CT, DP, QT>;
  static std::atomic<uint64_t> allowed{0};
  static std::atomic<int> held[64][5];  // a device's clusters of 2^i blocks, and one more (0: not asked yet)
  *size = 1;
  if (columns * 2 > all) return CP_OK;
  const void* kernel = (const void*)k_decode_cluster<CT, DP, QT, SCORES>;
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
      if (cudaOccupancyMaxActiveClusters(&n, k_decode_cluster<CT, DP, QT, SCORES>, &cfg) != cudaSuccess) {
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

template <int CT, int DP, int QT, bool SCORES>
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
  const uint64_t page = (uint64_t)cache_bytes(CT, ch.page_stride), slot = (uint64_t)cache_bytes(CT, ch.slot_stride);
  int shift = 4;
  while (shift < 31 && (page | slot) != 0 && ((page | slot) >> shift & 1) == 0) ++shift;
  const uint64_t far = (uint64_t)(ch.pages > 0 ? ch.pages - 1 : 0) * (page >> shift) +
                       (uint64_t)(ch.page_size - 1) * (slot >> shift);
  if (far > 0xFFFFFFFFu) return CP_EUNSUPPORTED;
  Rows rows{(uint32_t)(page >> shift), (uint32_t)(slot >> shift), (uint32_t)1 << shift, 0, 0, 0, 0, 4};
  if constexpr (CT == CP_I4) {
    if ((uint64_t)(ch.pages > 0 ? ch.pages - 1 : 0) * (uint64_t)(ch.block_page / 4) +
            (uint64_t)(ch.page_size - 1) * (uint64_t)(ch.block_slot / 4) > 0xFFFFFFFFu)
      return CP_EUNSUPPORTED;
    rows.block_page = (uint32_t)(ch.block_page / 4);
    rows.block_slot = (uint32_t)(ch.block_slot / 4);
    // a row's scales in one copy, where they fill the layout's and are aligned to that
    const uint64_t any = (uint64_t)ch.k_block | (uint64_t)ch.v_block | (uint64_t)ch.block_page | (uint64_t)ch.block_slot |
                         (uint64_t)ch.block_head;
    if (S::sb >= 8 && block_bytes(ch.D) == S::sb && any % S::sb == 0) rows.piece = S::sb;
  }
  while (((int64_t)1 << rows.div_shift) < ch.page_size) ++rows.div_shift;
  rows.mul = (uint32_t)((((uint64_t)1 << (31 + rows.div_shift)) + ch.page_size - 1) / ch.page_size);

  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  int64_t grid = (int64_t)di.sm_count * S::per_sm;
  if (grid > kDecodeBlocks) grid = kDecodeBlocks;
  const int64_t all = grid;
  if (grid > line) grid = line;
  const int64_t columns = (int64_t)a.B * ch.heads * tiles;
  // A 4-bit row is shorter than the 128 bytes that L2 likes, and its scales than the 32 that it fetches at least: where
  // a token's heads lie side by side, the blocks go over them together.  32 sequences of 8448 keys and 4 heads of 128
  // 47.5 us, head by head 57.7 (and 295 MB read for 156), in pages of one row 50.7, 59.5; of 20 heads of 64 126, 184.
  int lines = 1;
  // (Blocks that are no multiple of the heads are left out: 61 heads of 64 and 16 sequences 212 us on 549 of 608, head by head
  // 477; 2 sequences of 30,000 keys 99 and 98.)
  // from a token to the next: pages of one row have no second slot
  const int64_t token = ch.page_size > 1 ? ch.slot_stride : ch.page_stride;
  if (CT == CP_I4 && ch.heads > 1 && token > ch.head_stride && 4 * ch.heads * tiles <= grid) {
    lines = ch.heads * tiles;
    grid = grid / lines * lines;
  }
  const bool by_column = columns <= grid;
  Begin* begins = (Begin*)a.ws;
  float* parts = (float*)((char*)a.ws + kDecodeBlocks * sizeof(Begin));
  static std::atomic<uint64_t> allowed{0};
  CP_TRY_STATUS(allow_smem_once((const void*)k_decode<CT, DP, QT, SCORES>, S::smem, "decode: shared memory", &allowed));
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
  // 4 bits, 7 queries a head of 128: 320 tiles of 150 to 300 keys 16.5 / 15.4, of 250 to 500 18.2 / 22.9; 640 23.2 / 19.6, 26.3 /
  // 30.0; 1600 44.5 / 23.1, 53.2 / 33.6, of 500 to 1000 71.3 / 58.9; half marked 640 24.5 / 14.2, 23.6 / 18.9, of 500 to 1000
  // 32.1 / 33.9.  (The rule leaves warps out at 320 tiles where half of up to 300 keys are marked, 18.6 / 11.5, and
  // of heads of 64, 15.8 / 11.3.)
  // Few tiles too, when two tiles of keys (one of float32) are all there is: one sequence
  // of 4 tiles and 16 keys 5.5 / 3.8, of 50 5.5 / 6.2; 60 of 4, 16 keys 6.5 / 4.1, 50 keys
  // 7.2 / 6.5; float32, 8 keys 8.9 / 7.4, 16 keys 9.0 / 8.6 and, for one sequence, 7.9 /
  // 8.2.
  constexpr int kFew = CT == CP_F32 ? 8 : 32;
  const int64_t reach = CT == CP_F32 ? (a.keep ? 240 : 48) * columns : (a.keep ? 2 : 1) * kUnit * (3 * columns + all);
  if (most <= kFew || (columns > all && most <= (a.keep ? 32 : 16) * kUnit && most * all <= reach)) {
    using Short = Shape<CT, DP, QT, true>;
    static std::atomic<uint64_t> short_allowed{0};
    CP_TRY_STATUS(allow_smem_once((const void*)k_decode_short<CT, DP, QT, SCORES>, Short::smem, "decode: shared memory",
                                  &short_allowed));
    const int64_t room = (int64_t)di.sm_count * Short::per_sm, wanted = (columns + kWarps - 1) / kWarps;
    return cuda_status(launch_early(k_decode_short<CT, DP, QT, SCORES>, dim3((unsigned)(wanted < room ? wanted : room)), kThreads,
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
  // 4 bits, as one line / with clusters: 4 tiles of 500 keys 9.3 / 7.4, of 8000 15.8 / 10.5; 64 of 1500 14.0 / 12.7, of
  // 4000 20.5 / 22.2, with 15% marked 16.4 / 11.7; 128 of 1500 19.6 / 19.0.
  // float32 computes longer on a unit: half of the longest one's time and a quarter of
  // what idles; 64 tiles of 500 to 3000 keys 46 / 67 (heads of 256), 27 / 34 (128), 19 /
  // 25 (64), of 1500 41 / 40, 23.2 / 21.4, 17.4 / 15.7; 4 of 4000 16.1 / 19.5, 12.3 / 12.6,
  // 10.6 / 11.6, of 1500 12.0 / 11.0, 9.3 / 8.2, 8.1 / 7.4.
  const int64_t n64 = (most + kUnit - 1) / kUnit;
  int size = 0;
  if (cut) CP_TRY_STATUS((cluster_size<CT, DP, QT, SCORES>(columns, all, &size)));
  const bool slow = CT == CP_F32 && !a.keep;
  if (size > 1 && n64 <= (a.keep ? 48 : slow ? 8 : 16) * size &&
      n64 * (all - columns * size) <= (slow ? 2 : 8) * size * all)
    return cuda_status(launch_early_cluster(k_decode_cluster<CT, DP, QT, SCORES>, dim3((unsigned)(columns * size)), kThreads, S::smem,
                                            s, size, a, rows, tiles, size),
                       "decode: cluster");
  CP_TRY_STATUS(cuda_status(launch_early(k_decode<CT, DP, QT, SCORES>, dim3((unsigned)grid), kThreads, S::smem, s, a, rows, unit,
                                         tiles, parts, cut ? begins : nullptr, (int)by_column, lines),
                            "decode"));
  if (!cut) return CP_OK;
  // about so many parts a query tile, and the join's queries side by side for it
  const int64_t share = grid / columns + 1;
  const int queries = G < QT ? G : QT;
  int side = share <= 4 ? 8 : share <= 12 ? 2 : 1;
  while (side > 1 && side / 2 >= queries) side /= 2;
  const dim3 joins((unsigned)(by_column ? columns : grid), (unsigned)(queries + side - 1) / side);
  return launch_join<CT, DP, QT>(a, joins, tiles, side, parts, begins, lines, s);
}

template <int CT, int DP, bool SCORES>
static int launch_pass(const DecodeArgs& a, cudaStream_t s) {
  constexpr int one = CT == CP_F32 ? 4 : 8;
  return decode_pass(CT, a.Hq / a.cache.heads) == one ? launch<CT, DP, one, SCORES>(a, s) : launch<CT, DP, 2 * one, SCORES>(a, s);
}
template <int CT, bool SCORES = false>
static int launch_type(const DecodeArgs& a, cudaStream_t s) {
  switch (decode_width(a.cache.D)) {
    case 64: return launch_pass<CT, 64, SCORES>(a, s);
    case 128: return launch_pass<CT, 128, SCORES>(a, s);
    default: return launch_pass<CT, 256, SCORES>(a, s);
  }
}

}  // namespace cp
