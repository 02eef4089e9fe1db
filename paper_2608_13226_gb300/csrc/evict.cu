// Eviction from a paged cache: which keys of each sequence stay, and their rows moved up.
//
// k_evict_pick finds them: the weights become integers of the same order, the weight of the last key
// that stays is found by counting digits of 11 bits from the top (radix selection), and a
// count over the keys in their order gives each that stays its place.
//
// k_evict_rows moves the rows: HBM bounds it, every row read and written once.  A block or a cluster has
// one head's rows (of keys or values) of a sequence to itself and takes them in their
// order, a turn of some at a time: all of these are read before the first is written, and rows still
// to come lie behind every place that is written (the i-th row that stays comes from place i or
// later).  So reading goes on ahead of writing without a further wait.
#include "common.cuh"
#include "rope.cuh"

namespace cp {

// ------------------------------------------------------------------ which keys
constexpr int kPickThreads = 1024, kPickWarps = kPickThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBins = 2048;        // of a digit: sign, exponent and two bits first, so that few lanes meet at one
constexpr int kCopies = 2;         // of the counts
constexpr int kMostHeld = 32768;   // keys that a block keeps in shared memory

// Larger weights have larger numbers: a NaN 0, then -infinity to infinity, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t remote_u32(const uint32_t* p, int rank) {
  uint32_t x;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(map_rank(smem_addr(p), (uint32_t)rank)) : "memory");
  return x;
}

// A cluster of `size` blocks has a sequence.  HELD: a block's numbers fit its shared memory.
template <bool HELD>
__global__ void __launch_bounds__(kPickThreads, 1) k_evict_pick(EvictArgs a, int size) {
  extern __shared__ uint32_t s_held[];
  __shared__ uint32_t s_count[kCopies][kBins];
  __shared__ uint32_t s_all[kBins], s_warp[kPickWarps];  // this block's counts, for the others: of a bin, of a warp's 64
  __shared__ uint32_t s_total[kPickWarps];    // the cluster's of a warp's
  __shared__ uint32_t s_above[kPickWarps], s_equal[kPickWarps];
  __shared__ uint32_t s_pair[2];              // this block's numbers above and equal
  __shared__ uint32_t s_digit, s_left, s_size;
  wait_for_stream();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int b = blockIdx.x / size, rank = size > 1 ? (int)cluster_ctarank() : 0;
  const int given = a.lens[b], len = min(max(given, 0), a.cache.capacity);
  const float* weight = a.weight + b * a.weight_stride;
  int32_t* kept = a.kept + (int64_t)b * a.left;
  float* to = a.new_weight ? a.new_weight + b * a.new_weight_stride : nullptr;
  const int n = min(len, a.left);
  const bool all = len <= a.left;
  const int front = all ? len : a.first, back = all ? 0 : a.recent;
  // what stays in any case, and what follows the last key (in the end: barriers of a cluster wait for what was written)
  auto rest = [&] {
    const int threads = kPickThreads * size, tid = rank * kPickThreads + threadIdx.x;
    if (tid == 0 && a.new_lens) a.new_lens[b] = given < 0 ? given : n;
    for (int i = tid; i < front; i += threads) {
      kept[i] = i;
      if (to && i < a.new_weight_width) to[i] = weight[i];
    }
    for (int i = tid; i < back; i += threads) {
      const int j = len - back + i, at = n - back + i;
      kept[at] = j;
      if (to && at < a.new_weight_width) to[at] = weight[j];
    }
    for (int i = n + tid; i < a.left; i += threads) kept[i] = -1;
    if (to)
      for (int64_t i = n + tid; i < a.new_weight_width; i += threads) to[i] = 0.0f;
  };
  const int want = n - front - back;  // of the keys [lo, hi) between
  if (all || want <= 0) {             // the same in every block of the cluster
    rest();
    return;
  }
  const int lo = a.first, hi = len - a.recent;
  // a warp's keys: [w0, w1), in the order of ranks and warps
  const int warps = kPickWarps * size, each = ((hi - lo + warps - 1) / warps + 31) / 32 * 32;
  const int w0 = (int)min((int64_t)hi, lo + (int64_t)(rank * kPickWarps + warp) * each), w1 = min(hi, w0 + each);
  uint32_t* held = s_held + warp * each - w0;
  auto number = [&](int j) { return HELD ? held[j] : order_of(weight[j]); };

  uint32_t prefix = 0, left = (uint32_t)want;  // the digits so far; how many of the keys with them stay
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass < 2 ? 2048 : 1024;
    const uint32_t mask = pass == 0 ? 0 : pass == 1 ? ~0u << 21 : ~0u << 10;
    for (int i = threadIdx.x; i < kCopies * kBins; i += kPickThreads) (&s_count[0][0])[i] = 0;
    __syncthreads();
#pragma unroll 8
    for (int j = w0 + lane; j < w1; j += 32) {
      const uint32_t u = pass == 0 ? order_of(weight[j]) : number(j);
      if (HELD && pass == 0) held[j] = u;
      if ((u & mask) == prefix) atomicAdd(&s_count[warp % kCopies][u >> shift & (bins - 1)], 1u);
    }
    __syncthreads();
    // The digit in which the last key that stays falls.  A thread has bins kBins - 1 - 2 i and the one below, so that
    // they go from the top; first by what the 64 bins of a warp hold, then within the one warp's.
    const int top = kBins - 1 - 2 * threadIdx.x;
    uint32_t x = 0, y = 0;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      x += s_count[i][top];
      y += s_count[i][top - 1];
    }
    uint32_t total = __reduce_add_sync(~0u, x + y);
    if (size > 1) {
      s_all[top] = x;
      s_all[top - 1] = y;
      if (lane == 0) s_warp[warp] = total;
      __syncwarp();
      hw_cluster_sync();
      total = __reduce_add_sync(~0u, lane < size ? remote_u32(&s_warp[warp], lane) : 0);
    }
    if (lane == 0) s_total[warp] = total;
    __syncthreads();
    const uint32_t above = __reduce_add_sync(~0u, lane < warp ? s_total[lane] : 0);
    if (above < left && above + total >= left) {  // one warp
      if (size > 1) {
        uint32_t xs[kMaxCluster], ys[kMaxCluster];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
          xs[r] = r < size ? remote_u32(&s_all[top], r) : 0;
          ys[r] = r < size ? remote_u32(&s_all[top - 1], r) : 0;
        }
        x = y = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
          x += xs[r];
          y += ys[r];
        }
      }
      uint32_t upto = x + y;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint32_t z = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += z;
      }
      const uint32_t before = above + upto - x - y;
      if (before < left && before + x + y >= left) {  // one lane
        const bool first = before + x >= left;
        s_digit = (uint32_t)(first ? top : top - 1);
        s_left = left - before - (first ? 0 : x);
        s_size = first ? x : y;
      }
    }
    __syncthreads();
    prefix |= s_digit << shift;
    left = s_left;
    const bool whole = s_left == s_size;
    if (size > 1) hw_cluster_sync();  // the others have read this block's counts
    // All keys with these digits stay, as where there is one: those above what lies below them do, and no digit
    // more is wanted.  (They are not all keys that there are, so there is something below.)
    if (whole) {
      prefix -= 1;
      left = 0;
      break;
    }
  }

  // all above `prefix` stay, and the first `left` that equal it: each warp's numbers of both
  uint32_t above = 0, equal = 0;
#pragma unroll 8
  for (int j = w0 + lane; j < w1; j += 32) {
    const uint32_t u = number(j);
    above += u > prefix;
    equal += u == prefix;
  }
  above = __reduce_add_sync(~0u, above);
  equal = __reduce_add_sync(~0u, equal);
  if (lane == 0) {
    s_above[warp] = above;
    s_equal[warp] = equal;
  }
  __syncthreads();
  uint32_t before_above, before_equal;
  {
    const uint32_t x = s_above[lane], y = s_equal[lane];
    before_above = __reduce_add_sync(~0u, lane < warp ? x : 0);
    before_equal = __reduce_add_sync(~0u, lane < warp ? y : 0);
    if (warp == 0) {
      const uint32_t sx = __reduce_add_sync(~0u, x), sy = __reduce_add_sync(~0u, y);
      if (lane == 0) {
        s_pair[0] = sx;
        s_pair[1] = sy;
      }
    }
  }
  if (size > 1) {
    __syncwarp();
    hw_cluster_sync();
    const uint32_t x = lane < rank ? remote_u32(&s_pair[0], lane) : 0, y = lane < rank ? remote_u32(&s_pair[1], lane) : 0;
    before_above += __reduce_add_sync(~0u, x);
    before_equal += __reduce_add_sync(~0u, y);
    hw_cluster_sync();  // no block ends while its numbers are read
  }
  // the place of each key that stays, some groups of 32 at a time, whose loads are under way together
  constexpr int kGroups = 4;
  const uint32_t below = (1u << lane) - 1;
  for (int j0 = w0; j0 < w1; j0 += 32 * kGroups) {
    uint32_t u[kGroups];
    float x[kGroups];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int j = j0 + 32 * i + lane;
      u[i] = j < w1 ? number(j) : 0;
      x[i] = j < w1 && to ? weight[j] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int j = j0 + 32 * i + lane;
      const uint32_t is_above = __ballot_sync(~0u, j < w1 && u[i] > prefix), is_equal = __ballot_sync(~0u, j < w1 && u[i] == prefix);
      const uint32_t equals = before_equal + __popc(is_equal & below);  // before this key
      const bool stays = (is_above >> lane & 1) || ((is_equal >> lane & 1) && equals < left);
      if (stays) {
        const int at = front + (int)(before_above + __popc(is_above & below) + min(equals, left));
        kept[at] = j;
        if (to && at < a.new_weight_width) to[at] = x[i];
      }
      before_above += __popc(is_above);
      before_equal += __popc(is_equal);
    }
  }
  rest();
}

// ------------------------------------------------------------------ their rows
constexpr int kMoveThreads = 256;
constexpr int kPer = 4;        // pieces of a thread in a turn
constexpr int kStages = 4;     // turns under way
constexpr int kAhead = 3;      // turns that a trip to L2 takes, about (one sequence of 200,001 keys: 2 180 us, 3 174, 4 171; 64 of 1240: 34, 35, 36)
constexpr int64_t kTogether = 256;  // bytes that heads side by side go together up to
constexpr int kMostLooked = 256;    // sequences that a block looks through
constexpr int kNotes = kStages + 1;  // turns of notes: one is written while others may still go by the oldest

// Rows of one kind: codes or elements, or a 4-bit row's scales.  Of a row, heads that lie side by side make a part of
// `bytes` bytes, and parts are `part` bytes apart.
struct Kind {
  char *k, *v;
  int64_t page, slot, part;  // bytes
  int parts, bytes;
};
// Where a row comes from and where it goes, bytes; -1: it stays.
struct Move {
  int64_t from, to;
};

// Which rows move, found out by a thread a row: its key, then kAhead turns later the pages, and again that
// later where it goes, so that no turn waits for a trip to L2.
struct Moves {
  const EvictArgs& a;
  const int64_t page, slot;  // bytes
  const Divisor by_page;
  const int32_t *kept, *table;
  int n, stride;  // rows that stay, rows of a cluster's turn
  int row;        // this thread's of turn 0; stride: none
  int keys[2 * kAhead];
  int2 pages[kAhead];

  __device__ int row_of(int turn) const { return row + turn * stride; }  // n < 2^30, and a few turns more
  __device__ int key_of(int turn) const { return row < stride && row_of(turn) < n ? kept[row_of(turn)] : -1; }
  __device__ int2 pages_of(int turn, int key) const {
    if (key < 0 || key == row_of(turn)) return make_int2(-1, -1);
    return make_int2(table[by_page.of(key)], table[by_page.of(row_of(turn))]);
  }
  __device__ Move move_of(int turn, int key, int2 p) const {
    Move m{-1, -1};
    const int to = row_of(turn);
    if (key < 0 || key == to) return m;
    if (p.x >= 0 && p.x < a.cache.pages && p.y >= 0 && p.y < a.cache.pages) {
      m.from = p.x * page + (key - by_page.of(key) * (int)by_page.d) * slot;
      m.to = p.y * page + (to - by_page.of(to) * (int)by_page.d) * slot;
    } else if (a.status) {
      set_status(a.status, CP_EINVAL);
    }
    return m;
  }
  __device__ Move at_once(int turn) const {
    const int key = key_of(turn);
    return move_of(turn, key, pages_of(turn, key));
  }
  __device__ void start(int turn) {
#pragma unroll
    for (int i = 0; i < 2 * kAhead; ++i) keys[i] = key_of(turn + i);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) pages[i] = pages_of(turn + i, keys[i]);
  }
  // u: how many calls there have been, modulo 2 kAhead, a constant where it counts: a register that is still being loaded
  // must not be moved to another.
  __device__ __forceinline__ Move next(int turn, int u) {
    const Move m = move_of(turn, keys[u], pages[u % kAhead]);
    pages[u % kAhead] = pages_of(turn + kAhead, keys[(u + kAhead) % (2 * kAhead)]);
    keys[u] = key_of(turn + 2 * kAhead);
    return m;
  }
};

// What a cluster has to move: `bytes` bytes of `n` rows of a sequence, from `base` on.
struct Job {
  char* base;
  int b, n, bytes;
  bool of_scales;
};
// Into how many pieces a row's part may be divided: of 64 bytes (a turn has no more rows of smaller ones), or of 32 where
// those do not make it up.
template <int BYTES>
__host__ __device__ __forceinline__ int units_of(const Kind& rows) {
  const int bytes = rows.bytes % 64 == 0 ? 64 : 32;
  return BYTES == 16 && rows.bytes % bytes == 0 ? rows.bytes / bytes : 1;
}
// Into how many they are, so that `cut` sequences' jobs are at most `clusters` (if they are undivided).
__host__ __device__ __forceinline__ int divided_by(int clusters, int cut, const Kind& rows, const Kind& scales, int units) {
  const int most = (clusters / (2 * cut) - scales.parts) / rows.parts;
  int f = most < units ? most : units;
  while (f > 1 && units % f != 0) --f;
  return f < 1 ? 1 : f;
}
// The cluster's job (n 0: none).  Sequences that keep all their keys have none; where that leaves clusters without, they take pieces
// of the others' rows (32 sequences of 1300 to 8704 keys, a few of them above 8000, 44 us, undivided 96; one of
// 200,001 keys 174, 254).  Where all are cut, rows go whole as far as that fills the device (32 sequences by 128 bytes
// 54.6 us, by 256 50.1, in an earlier version).
template <int BYTES>
__device__ __forceinline__ Job job_of(const EvictArgs& a, const Kind& rows, const Kind& scales, int id, int clusters) {
  __shared__ uint32_t s_cut[kMostLooked / 32];  // which sequences are cut
  const int lane = threadIdx.x % 32;
  uint32_t word = 0;
  int cut = a.B;
  if (a.B <= kMostLooked) {
    const int seq = threadIdx.x;
    const uint32_t all = __ballot_sync(~0u, seq < a.B && min(a.lens[min(seq, a.B - 1)], a.cache.capacity) > a.left);
    if (lane == 0) s_cut[seq / 32] = all;
    __syncthreads();
    word = lane < kMostLooked / 32 ? s_cut[lane] : 0;
    cut = __reduce_add_sync(~0u, __popc(word));
  }
  Job x{nullptr, 0, 0, 0, false};
  if (cut == 0) return x;
  int f = divided_by(clusters, cut, rows, scales, units_of<BYTES>(rows));
  const int of_rows = cut * 2 * rows.parts * f;
  if (id >= of_rows + cut * 2 * scales.parts) return x;
  x.of_scales = id >= of_rows;
  const Kind& kind = x.of_scales ? scales : rows;
  if (x.of_scales) {
    id -= of_rows;
    f = 1;
  }
  x.bytes = kind.bytes / f;
  const int part = id % (kind.parts * f);
  id /= kind.parts * f;
  x.base = (id % 2 ? kind.v : kind.k) + part / f * kind.part + part % f * x.bytes;
  int b = id / 2;  // of those that are cut
  if (cut < a.B) {
    int upto = __popc(word);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int y = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += y;
    }
    const int at = __ffs(__ballot_sync(~0u, upto > b)) - 1;
    b -= __shfl_sync(~0u, upto - __popc(word), at);
    word = __shfl_sync(~0u, word, at);
    for (; b > 0; --b) word &= word - 1;
    b = 32 * at + __ffs(word) - 1;
  }
  x.b = b;
  x.n = a.B <= kMostLooked || min(a.lens[b], a.cache.capacity) > a.left ? a.left : 0;
  return x;
}
__device__ __forceinline__ void turn_barrier(int size) {
  // The notes go from thread to thread of a block, which __syncthreads orders.  Between blocks nothing is handed on but that
  // rows have been read, and a read that has come back cannot see what is written later: the cluster's barrier
  // need not order memory.  Doing so it would wait for every row written so far, each turn (one sequence of
  // 200,001 keys 174 us, else 279).
  __syncthreads();
  if (size > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
template <int BYTES> struct Piece;
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<4> { using type = uint32_t; };
template <int BYTES>
__device__ __forceinline__ void copy_piece(uint32_t to, const void* from) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}

// Rows that a block's threads have side by side: as many as have a thread each to find out about kPer of them.
__host__ __device__ __forceinline__ int side_of(int pieces) {
  return pieces < kPer ? kMoveThreads / kPer : kMoveThreads / pieces;
}

// A thread has a piece of kPer rows of every turn, which it copies to a slot of its own and takes from there.
template <int BYTES>
__global__ void __launch_bounds__(kMoveThreads) k_evict_rows(EvictArgs a, Kind rows_of, Kind scales_of, Divisor by_page, int size) {
  using P = typename Piece<BYTES>::type;
  extern __shared__ __align__(16) char smem[];  // kStages turns of pieces, and notes of kNotes
  wait_for_stream();
  const Job job = job_of<BYTES>(a, rows_of, scales_of, blockIdx.x / size, gridDim.x / size);
  const int b = job.b, n = job.n;
  if (n == 0) return;  // in every block of the cluster
  const Kind& kind = job.of_scales ? scales_of : rows_of;
  char* base = job.base;
  const int pieces = job.bytes / BYTES, side = side_of(pieces), rows = side * kPer;  // rows side by side, and of a turn
  const int piece = threadIdx.x % pieces, r0 = threadIdx.x / pieces;
  const bool works = r0 < side;
  const int rank = size > 1 ? (int)cluster_ctarank() : 0;
  Moves moves{a, kind.page, kind.slot, by_page, a.kept + (int64_t)b * a.left, a.cache.table + b * a.cache.table_stride, n, rows * size,
              (int)threadIdx.x < rows ? rank * rows + (int)threadIdx.x : rows * size};
  const int turns = (n + rows * size - 1) / (rows * size);
  P* ring = reinterpret_cast<P*>(smem) + threadIdx.x;
  Move* notes = reinterpret_cast<Move*>(smem + kStages * kPer * kMoveThreads * sizeof(P));
  base += piece * BYTES;
  auto note = [&](int turn, const Move& m) {
    notes[turn % kNotes * kMoveThreads + threadIdx.x] = m;
  };
  auto load = [&](int turn) {
    if (turn < turns && works) {
      const Move* of = notes + turn % kNotes * kMoveThreads + r0;
      P* to = ring + turn % kStages * (kPer * kMoveThreads);
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int64_t from = of[k * side].from;
        if (from >= 0) copy_piece<BYTES>(smem_addr(to + k * kMoveThreads), base + from);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int t = 0; t < kStages - 1; ++t) note(t, moves.at_once(t));
  moves.start(kStages - 1);
  __syncthreads();
  for (int t = 0; t < kStages - 1; ++t) load(t);
  for (int t0 = 0; t0 < turns; t0 += 2 * kAhead)
#pragma unroll
    for (int u = 0; u < 2 * kAhead; ++u) {
      const int t = t0 + u;
      if (t >= turns) break;  // in every block of the cluster
      note(t + kStages - 1, moves.next(t + kStages - 1, u));
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      turn_barrier(size);  // turn t has been read by every thread of the cluster; its rows may be written over
      if (works) {
        const Move* of = notes + t % kNotes * kMoveThreads + r0;
        const P* from = ring + t % kStages * (kPer * kMoveThreads);
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          const int64_t to = of[k * side].to;
          if (to >= 0) *reinterpret_cast<P*>(base + to) = from[k * kMoveThreads];
        }
      }
      load(t + kStages - 1);
    }
}

template <int BYTES>
constexpr size_t smem_of() {
  return kMoveThreads * (kStages * kPer * (size_t)BYTES + kNotes * sizeof(Move));
}

// How many clusters of `size` blocks (1 to kMaxCluster) run at the same time; asked once a device and size.
template <int BYTES>
static int clusters_at_once(int size, int* n) {
  static std::atomic<uint64_t> allowed{0};
  static std::atomic<int> held[64][4];  // and one more (0: not asked yet)
  CP_TRY_STATUS(allow_smem_once((const void*)k_evict_rows<BYTES>, smem_of<BYTES>(), "evict: shared memory", &allowed));
  int dev = 0;
  CP_TRY_STATUS(cuda_status(cudaGetDevice(&dev), "evict: device"));
  std::atomic<int>& known = held[dev & 63][size >= 8 ? 3 : size / 2];
  *n = known.load(std::memory_order_relaxed) - 1;
  if (*n >= 0) return CP_OK;
  cudaLaunchAttribute with{};
  with.id = cudaLaunchAttributeClusterDimension;
  with.val.clusterDim = {(unsigned)size, 1, 1};
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)size);
  cfg.blockDim = dim3(kMoveThreads);
  cfg.dynamicSmemBytes = smem_of<BYTES>();
  cfg.attrs = &with;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(n, k_evict_rows<BYTES>, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();  // a size that the device does not take
    *n = 0;
  }
  known.store(*n + 1, std::memory_order_relaxed);
  return CP_OK;
}

// Rows of two kinds (of the second there may be none) moved up.
template <int BYTES>
static int move_rows(const EvictArgs& a, const Kind& first, const Kind& second, cudaStream_t s) {
  const int rows = side_of(first.bytes / BYTES) * kPer, units = units_of<BYTES>(first);
  const int64_t jobs = (int64_t)a.B * 2 * (first.parts + second.parts);
  // Clusters where there are few heads and sequences, if they get some turns: of the sizes of which all jobs run at the same
  // time (a cluster waits for its own blocks only, so more would be right as well, one after another) the one that
  // keeps most blocks busy should every sequence be cut.
  int size = 1;
  int64_t clusters = jobs, busy = 0;
  for (int z = kMaxCluster; z >= 1; z /= 2) {
    if (z > 1 && (int64_t)rows * z * 4 > a.left) continue;
    int n = 0;
    CP_TRY_STATUS(clusters_at_once<BYTES>(z, &n));
    if (jobs > n && z > 1) continue;
    const int64_t with = jobs > n ? jobs : ((int64_t)divided_by(n, a.B, first, second, units) * first.parts + second.parts) * 2 * a.B;
    if (with * z <= busy) continue;
    busy = with * z;
    size = z;
    clusters = std::max(jobs, std::min((int64_t)n, (int64_t)a.B * 2 * ((int64_t)first.parts * units + second.parts)));
  }
  if (clusters * size > 0x7FFFFFFF) return CP_EUNSUPPORTED;
  return cuda_status(launch_early_cluster(k_evict_rows<BYTES>, dim3((unsigned)(clusters * size)), kMoveThreads, smem_of<BYTES>(), s,
                                          size, a, first, second, divisor(a.cache.page_size), size),
                     "evict: rows");
}
// How rows of `bytes` bytes a head move, heads `head` bytes apart: by 16 bytes (`whole`) or by 4.
static int divide(const EvictArgs& a, Kind* kind, int64_t head, int bytes, bool* whole) {
  int group = 1;  // heads that lie side by side go together
  const int heads = a.cache.heads;
  if (head == bytes)
    for (int g = 2; g <= heads && (int64_t)g * bytes <= kTogether; ++g)
      if (heads % g == 0) group = g;
  kind->parts = heads / group;
  kind->part = head * group;
  kind->bytes = bytes * group;
  const uint64_t any = (uint64_t)kind->k | (uint64_t)kind->v | (uint64_t)kind->page | (uint64_t)kind->slot | (uint64_t)kind->part |
                       (uint64_t)kind->bytes;
  *whole = any % 16 == 0;
  if ((int64_t)a.B * 2 * kind->parts > 0x3FFFFFFF) return CP_EUNSUPPORTED;
  return CP_OK;
}

int launch_cache_evict(const EvictArgs& a, int cache_dtype, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const Cache& ch = a.cache;
  // As many blocks of a sequence as the device has room for, of 8192 keys at least (one of 8192 keys 14.2 us a call, by
  // two blocks 15.0).
  int size = 1;
  while (size < kMaxCluster && (int64_t)a.B * size * 2 <= di.sm_count && (int64_t)size * 16384 <= ch.capacity) size *= 2;
  if ((int64_t)a.B * size > 0x7FFFFFFF) return CP_EUNSUPPORTED;
  const int64_t most = (((int64_t)ch.capacity + kPickWarps * size - 1) / (kPickWarps * size) + 31) / 32 * 32 * kPickWarps;
  static std::atomic<uint64_t> allowed{0};
  CP_TRY_STATUS(allow_smem_once((const void*)k_evict_pick<true>, kMostHeld * 4, "evict: shared memory", &allowed));
  const dim3 grid((unsigned)(a.B * size));
  CP_TRY_STATUS(cuda_status(most <= kMostHeld
                                ? launch_early_cluster(k_evict_pick<true>, grid, kPickThreads, (size_t)most * 4, s, size, a, size)
                                : launch_early_cluster(k_evict_pick<false>, grid, kPickThreads, 0, s, size, a, size),
                            "evict: pick"));
  if (a.left == 0 || ch.capacity <= a.left) return CP_OK;  // no row moves
  Kind rows{(char*)ch.k, (char*)ch.v, cache_bytes(cache_dtype, ch.page_stride), cache_bytes(cache_dtype, ch.slot_stride)};
  Kind scales{(char*)ch.k_block, (char*)ch.v_block, ch.block_page, ch.block_slot}, none{};
  bool whole = true, together = false;  // (rows of the cache are multiples of 16 bytes)
  CP_TRY_STATUS(divide(a, &rows, cache_bytes(cache_dtype, ch.head_stride), (int)cache_bytes(cache_dtype, ch.D), &whole));
  if (cache_dtype == CP_I4) CP_TRY_STATUS(divide(a, &scales, ch.block_head, block_bytes(ch.D), &together));
  CP_TRY_STATUS(move_rows<16>(a, rows, together ? scales : none, s));
  return cache_dtype == CP_I4 && !together ? move_rows<4>(a, scales, none, s) : CP_OK;
}

}  // namespace cp
