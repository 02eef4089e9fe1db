// Declarations shared by the operators of the decoding model (rotary.cu,
// decode.cu) and their host side (api_serve.cu).  Not part of the public ABI.
#pragma once

#include "internal.h"

namespace cp {

constexpr int kMaxRows = 4;  // tensors of one rotary call

struct Rope {
  const double* inv_freq;
  int half;  // rotated pairs
  int interleaved;
  float scale;
  int back;  // 1: the transpose
};

struct RowSet {
  const void* in;
  void* out;
  int64_t in_b, in_t, in_h, out_b, out_t, out_h;  // strides, elements
  int heads;
};

struct RotaryArgs {
  RowSet set[kMaxRows];
  int n;
  int64_t B, T;
  int D;
  const int64_t* pos;
  int64_t pos_stride;
  Rope rope;
};
int launch_rotary(const RotaryArgs& a, int dtype, cudaStream_t s);

struct Cache {
  void *k, *v;
  int64_t pages;
  int64_t page_stride, slot_stride, head_stride;  // elements
  const float *k_scale, *v_scale;
  const int32_t* table;
  int64_t table_stride;
  int32_t page_size;
  int32_t capacity;  // keys a table row holds
  int heads, D;
  uint8_t *k_block, *v_block;  // CP_I4: the rows' scales
  int64_t block_page, block_slot, block_head;  // bytes
};

// n elements of a cache in bytes (4 bits: n is even wherever it is asked for).
__host__ __device__ constexpr int64_t cache_bytes(int dtype, int64_t n) {
  return dtype == CP_F32 ? 4 * n : dtype == CP_BF16 ? 2 * n : dtype == CP_E4M3 ? n : n / 2;
}
// Bytes of a 4-bit row's scales.
__host__ __device__ constexpr int block_bytes(int D) { return (D / 16 + 3) / 4 * 4; }

struct AppendArgs {
  Cache cache;
  const void *k, *v;
  int64_t k_t, k_h, v_t, v_h;
  RowSet q;  // heads = 0: none
  int64_t T;
  const int32_t *starts, *lens;
  int B;
  const int64_t* pos;
  Rope rope;
  int32_t *new_lens, *status;
};
int launch_cache_append(const AppendArgs& a, int dtype, int cache_dtype, cudaStream_t s);

// The append to a 4-bit cache.
int launch_append_fours(const AppendArgs& a, int dtype, cudaStream_t s);

struct ReadArgs {
  Cache cache;
  void *k, *v;
  int64_t k_t, k_h, v_t, v_h;
  int64_t T;
  const int32_t *starts, *lens;
  int B;
  int32_t* status;
};
int launch_cache_read(const ReadArgs& a, int dtype, int cache_dtype, cudaStream_t s);

struct EvictArgs {
  Cache cache;
  const int32_t* lens;
  int B;
  const float* weight;
  int64_t weight_stride;
  int left, first, recent;
  int32_t* new_lens;
  float* new_weight;
  int64_t new_weight_stride, new_weight_width;
  int32_t *kept, *status;
};
int launch_cache_evict(const EvictArgs& a, int cache_dtype, cudaStream_t s);

struct DecodeArgs {
  Cache cache;
  const void* q;
  int64_t q_b, q_h;
  void* out;
  int64_t o_b, o_h;
  int B, Hq;
  const int32_t* lens;
  const uint8_t* keep;
  int64_t keep_stride;
  float scale;
  int64_t window;
  float* lse;
  void* ws;
  int32_t* status;
  // Only where weights are added up: scores in units of log 2, [B, score_cols, capacity, score_pitch],
  // a column for every query tile of a sequence (see score_shape).
  float* scores;
  int score_cols, score_pitch;
};
// A launch that may begin before what precedes it on the stream has ended: its
// blocks come to the SMs and wait there (wait_for_stream, first of all), so that its
// latency is spent beside the other's last blocks.
template <typename... Params, typename... Args>
cudaError_t launch_early_cluster(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t s,
                                 int cluster, Args... args) {
  cudaLaunchAttribute with[2] = {};
  with[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  with[0].val.programmaticStreamSerializationAllowed = 1;
  with[1].id = cudaLaunchAttributeClusterDimension;
  with[1].val.clusterDim = {(unsigned)cluster, 1, 1};
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = with;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  note_launch();
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t s,
                         Args... args) {
  return launch_early_cluster(kernel, grid, threads, smem, s, 1, args...);
}

size_t decode_ws_bytes(int64_t Hq, int64_t heads, int64_t D, int cache_dtype);
int launch_decode(const DecodeArgs& a, int cache_dtype, cudaStream_t s);
int launch_decode_bf16(const DecodeArgs& a, cudaStream_t s);
int launch_decode_e4m3(const DecodeArgs& a, cudaStream_t s);
int launch_decode_f32(const DecodeArgs& a, cudaStream_t s);
int launch_decode_i4(const DecodeArgs& a, cudaStream_t s);
// With the scores left in `scores`; launch_weigh then adds the weights up by them.
int launch_decode_scores(const DecodeArgs& a, int cache_dtype, cudaStream_t s);
int launch_decode_bf16_scores(const DecodeArgs& a, cudaStream_t s);
int launch_decode_e4m3_scores(const DecodeArgs& a, cudaStream_t s);
int launch_decode_f32_scores(const DecodeArgs& a, cudaStream_t s);
int launch_decode_i4_scores(const DecodeArgs& a, cudaStream_t s);
int launch_weigh(const DecodeArgs& a, int cache_dtype, float* weight, int64_t weight_stride, cudaStream_t s);

// Query heads that one pass of the attention takes for groups of G, the width that a
// head is laid out for, and the most blocks of a launch: what the workspace goes by.
inline int decode_pass(int cache_dtype, int64_t G) {
  if (cache_dtype == CP_F32) return G <= 4 ? 4 : 8;
  return G <= 8 ? 8 : 16;
}
// Columns of a sequence's scores (query tiles) and floats of a key in one: a tile's queries, to a power of two.
inline void score_shape(int cache_dtype, int64_t Hq, int64_t heads, int64_t* cols, int64_t* pitch) {
  const int64_t G = Hq / heads, pass = decode_pass(cache_dtype, G);
  *pitch = 1;
  while (*pitch < G && *pitch < pass) *pitch *= 2;
  *cols = heads * ((G + pass - 1) / pass);
}
inline int decode_width(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
constexpr int kDecodeBlocks = 1024;
// What the blocks leave for the join: the block that a query tile of sequence b
// begins in and over how many it goes on (0: it is whole, or there is none).
struct Begin {
  int block, blocks, b, col;
};

}  // namespace cp
