// Eviction from a paged cache: which keys of each sequence stay, and their rows moved up.
//
// k_evict_pick finds them: the weights become integers of the same order, the weight of the last key
// that stays is found by counting digits of 8 bits from the top (radix selection), and a
// count over the keys in their order gives each that stays its place.  Weights are read five
// times, from L2 after the first: its latency bounds it.
//
// k_evict_move moves the rows: HBM bounds it, every row read and written once.  A block has a slice
// of one head's rows (of keys or values) of a sequence to itself and takes them in their
// order, some at a time: all of these are read before the first is written, and rows still
// to come lie behind every place that is written (the i-th row that stays comes from place i or
// later).  So reading goes on ahead of writing without a further wait.
#include "common.cuh"
#include "rope.cuh"

namespace cp {

// ------------------------------------------------------------------ which keys
constexpr int kPickThreads = 1024, kPickWarps = kPickThreads / 32;
constexpr int kMaxPick = 8;     // blocks of a cluster
constexpr int kBins = 256;
constexpr int kCopies = 8;      // of the counts, so that fewer lanes meet at one

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

__global__ void __launch_bounds__(kPickThreads) k_evict_pick(EvictArgs a, int size) {
  __shared__ uint32_t s_count[kCopies][kBins];
  __shared__ uint32_t s_sum[kBins];           // this block's counts, for the others
  __shared__ uint32_t s_all[kBins];           // the cluster's
  __shared__ uint32_t s_above[kPickWarps], s_equal[kPickWarps];
  __shared__ uint32_t s_pair[2];              // this block's numbers above and equal
  __shared__ uint32_t s_digit, s_left;
  wait_for_stream();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int b = blockIdx.x / size, rank = size > 1 ? (int)cluster_ctarank() : 0;
  const int given = a.lens[b], len = min(max(given, 0), a.cache.capacity);
  const float* weight = a.weight + b * a.weight_stride;
  int32_t* kept = a.kept + (int64_t)b * a.left;
  float* to = a.new_weight ? a.new_weight + b * a.new_weight_stride : nullptr;
  const int n = min(len, a.left);
  if (rank == 0 && threadIdx.x == 0 && a.new_lens) a.new_lens[b] = given < 0 ? given : n;
  // what stays in any case, and what follows the last key
  const int threads = kPickThreads * size, tid = rank * kPickThreads + threadIdx.x;
  const bool all = len <= a.left;
  const int front = all ? len : a.first, back = all ? 0 : a.recent;
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
  const int want = n - front - back;  // of the keys [lo, hi) between
  if (all || want <= 0) return;       // the same in every block of the cluster
  const int lo = a.first, hi = len - a.recent;
  // a warp's keys: [w0, w1), in the order of ranks and warps
  const int warps = kPickWarps * size, each = ((hi - lo + warps - 1) / warps + 31) / 32 * 32;
  const int w0 = (int)min((int64_t)hi, lo + (int64_t)(rank * kPickWarps + warp) * each), w1 = min(hi, w0 + each);

  uint32_t prefix = 0, left = (uint32_t)want;  // the digits so far; how many of the keys with them stay
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < kCopies * kBins; i += kPickThreads) (&s_count[0][0])[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0 : ~0u << (shift + 8);
    for (int j = w0 + lane; j < w1; j += 32) {
      const uint32_t u = order_of(weight[j]);
      if ((u & mask) == prefix) atomicAdd(&s_count[warp % kCopies][u >> shift & 255], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kBins) {
      uint32_t x = 0;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) x += s_count[i][threadIdx.x];
      s_sum[threadIdx.x] = s_all[threadIdx.x] = x;
    }
    if (size > 1) {
      hw_cluster_sync();
      if (threadIdx.x < kBins) {
        uint32_t x = 0;
        for (int r = 0; r < size; ++r) x += remote_u32(&s_sum[threadIdx.x], r);
        s_all[threadIdx.x] = x;
      }
    }
    __syncthreads();
    if (warp == 0) {  // the digit in which the last key that stays falls: lane's 8 bins, from the top
      uint32_t own = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) own += s_all[kBins - 1 - 8 * lane - i];
      uint32_t upto = own;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint32_t x = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += x;
      }
      const uint32_t before = upto - own;
      if (before < left && upto >= left) {
        uint32_t over = before;
        int digit = kBins - 1 - 8 * lane;
        while (over + s_all[digit] < left) over += s_all[digit--];
        s_digit = (uint32_t)digit;
        s_left = left - over;
      }
    }
    __syncthreads();
    prefix |= s_digit << shift;
    left = s_left;
    if (size > 1) hw_cluster_sync();  // the others have read this block's counts
  }

  // all above `prefix` stay, and the first `left` that equal it: each warp's numbers of both
  uint32_t above = 0, equal = 0;
  for (int j = w0 + lane; j < w1; j += 32) {
    const uint32_t u = order_of(weight[j]);
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
    hw_cluster_sync();
    for (int r = 0; r < rank; ++r) {
      before_above += remote_u32(&s_pair[0], r);
      before_equal += remote_u32(&s_pair[1], r);
    }
    hw_cluster_sync();  // no block ends while its numbers are read
  }
  // the place of each key that stays
  for (int j0 = w0; j0 < w1; j0 += 32) {
    const int j = j0 + lane;
    const float x = j < w1 ? weight[j] : 0.0f;
    const uint32_t u = j < w1 ? order_of(x) : 0;
    const uint32_t is_above = __ballot_sync(~0u, j < w1 && u > prefix), is_equal = __ballot_sync(~0u, j < w1 && u == prefix);
    const uint32_t below = (1u << lane) - 1;
    const uint32_t equals = before_equal + __popc(is_equal & below);  // before this key
    const bool stays = (is_above >> lane & 1) || ((is_equal >> lane & 1) && equals < left);
    if (stays) {
      const int at = front + (int)(before_above + __popc(is_above & below) + min(equals, left));
      kept[at] = j;
      if (to && at < a.new_weight_width) to[at] = x;
    }
    before_above += __popc(is_above);
    before_equal += __popc(is_equal);
  }
}

// ------------------------------------------------------------------ their rows
constexpr int kMoveThreads = 256;
constexpr int kPer = 4;     // pieces of a thread in a turn
constexpr int kStages = 4;  // turns under way

// Rows of one kind: codes or elements (16-byte pieces), a 4-bit row's scales (4-byte ones).
struct Kind {
  char *k, *v;
  int64_t page, slot, head;  // bytes
  int pieces;                // of a slice's row
  int slices;
};
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

// Row i of the sequence's, as a thread notes it: where it comes from and where it goes, -1: it stays.
struct Move {
  int64_t from, to;
};

template <int BYTES>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(EvictArgs a, Kind kind) {
  using P = typename Piece<BYTES>::type;
  extern __shared__ __align__(16) char smem[];  // kStages turns of pieces, a thread's its own, and notes
  wait_for_stream();
  const Cache& ch = a.cache;
  int job = blockIdx.x;
  const int slice = job % kind.slices;
  job /= kind.slices;
  const int head = job % ch.heads;
  job /= ch.heads;
  char* base = job % 2 ? kind.v : kind.k;
  const int b = job / 2;
  const int n = min(min(max(a.lens[b], 0), ch.capacity), a.left);
  const int32_t* kept = a.kept + (int64_t)b * a.left;
  if (n == 0 || kept[n - 1] == n - 1) return;  // nothing moves
  base += head * kind.head + slice * kind.pieces * BYTES;
  const int32_t* table = ch.table + b * ch.table_stride;

  P* ring = reinterpret_cast<P*>(smem);
  const int rows = kMoveThreads * kPer / kind.pieces;  // of a turn
  Move* notes = reinterpret_cast<Move*>(smem + kStages * kPer * kMoveThreads * sizeof(P));
  const int turns = (n + rows - 1) / rows;
  auto page_of = [&](int key) { return table[(uint32_t)key / (uint32_t)ch.page_size]; };
  auto issue = [&](int turn) {
    if (turn < turns) {
      Move* to = notes + turn % kStages * rows;
      for (int r = threadIdx.x; r < rows; r += kMoveThreads) {
        const int i = turn * rows + r;
        Move m{-1, -1};
        if (i < n) {
          const int j = kept[i];
          if (j != i) {
            const int p = page_of(j), q = page_of(i);
            if (p >= 0 && p < ch.pages && q >= 0 && q < ch.pages) {
              m.from = p * kind.page + (int64_t)((uint32_t)j % (uint32_t)ch.page_size) * kind.slot;
              m.to = q * kind.page + (int64_t)((uint32_t)i % (uint32_t)ch.page_size) * kind.slot;
            } else if (a.status) {
              set_status(a.status, CP_EINVAL);
            }
          }
        }
        to[r] = m;
      }
    }
    __syncthreads();
    if (turn < turns) {
      const Move* of = notes + turn % kStages * rows;
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int x = k * kMoveThreads + threadIdx.x, r = x / kind.pieces;
        if (r < rows && of[r].from >= 0)
          copy_piece<BYTES>(smem_addr(ring + (turn % kStages * kPer + k) * kMoveThreads + threadIdx.x),
                            base + of[r].from + (x - r * kind.pieces) * BYTES);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int t = 0; t < kStages - 1; ++t) issue(t);
  for (int t = 0; t < turns; ++t) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncthreads();  // turn t has been read by every thread; its rows may be written over
    const Move* of = notes + t % kStages * rows;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int x = k * kMoveThreads + threadIdx.x, r = x / kind.pieces;
      if (r < rows && of[r].to >= 0)
        *reinterpret_cast<P*>(base + of[r].to + (x - r * kind.pieces) * BYTES) =
            ring[(t % kStages * kPer + k) * kMoveThreads + threadIdx.x];
    }
    issue(t + kStages - 1);
  }
}

template <int BYTES>
static int move(const EvictArgs& a, Kind kind, int row_pieces, int sms, cudaStream_t s) {
  // whole rows of a head, or where that gives few blocks a part of 4 pieces at least
  kind.slices = 1;
  const int64_t jobs = (int64_t)a.B * 2 * a.cache.heads;
  while (BYTES == 16 && jobs * kind.slices < 2 * sms && row_pieces % (2 * kind.slices) == 0 &&
         row_pieces / (2 * kind.slices) >= 4)
    kind.slices *= 2;
  kind.pieces = row_pieces / kind.slices;
  const int rows = kMoveThreads * kPer / kind.pieces;
  const size_t smem = kStages * (kPer * kMoveThreads * BYTES + rows * sizeof(Move));
  static std::atomic<uint64_t> allowed{0};
  CP_TRY_STATUS(allow_smem_once((const void*)k_evict_move<BYTES>, 200 * 1024, "evict: shared memory", &allowed));
  if (jobs * kind.slices > 0x7FFFFFFF) return CP_EUNSUPPORTED;
  return cuda_status(launch_early(k_evict_move<BYTES>, dim3((unsigned)(jobs * kind.slices)), kMoveThreads, smem, s, a, kind),
                     "evict: move");
}

int launch_cache_evict(const EvictArgs& a, int cache_dtype, cudaStream_t s) {
  DeviceInfo di;
  CP_TRY_STATUS(device_info(&di));
  const Cache& ch = a.cache;
  int size = 1;
  while (size < kMaxPick && (int64_t)size * 16384 < ch.capacity) size *= 2;
  if ((int64_t)a.B * size > 0x7FFFFFFF) return CP_EUNSUPPORTED;
  CP_TRY_STATUS(cuda_status(launch_early_cluster(k_evict_pick, dim3((unsigned)(a.B * size)), kPickThreads, 0, s, size, a, size),
                            "evict: pick"));
  if (a.left == 0 || ch.capacity <= a.left) return CP_OK;  // no row moves
  Kind kind{(char*)ch.k, (char*)ch.v, cache_bytes(cache_dtype, ch.page_stride), cache_bytes(cache_dtype, ch.slot_stride),
            cache_bytes(cache_dtype, ch.head_stride), 0, 1};
  CP_TRY_STATUS(move<16>(a, kind, (int)cache_bytes(cache_dtype, ch.D) / 16, di.sm_count, s));
  if (cache_dtype != CP_I4) return CP_OK;
  kind = Kind{(char*)ch.k_block, (char*)ch.v_block, ch.block_page, ch.block_slot, ch.block_head, 0, 1};
  return move<4>(a, kind, block_bytes(ch.D) / 4, di.sm_count, s);
}

}  // namespace cp
