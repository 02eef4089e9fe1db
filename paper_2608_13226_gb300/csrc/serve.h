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
};

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

// Query heads that one pass of the attention takes for groups of G, the width that a
// head is laid out for, and the most blocks of a launch: what the workspace goes by.
inline int decode_pass(int cache_dtype, int64_t G) {
  if (cache_dtype == CP_F32) return G <= 4 ? 4 : 8;
  return G <= 8 ? 8 : 16;
}
inline int decode_width(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
constexpr int kDecodeBlocks = 1024;
// What the blocks leave for the join: the block that a query tile of sequence b
// begins in and over how many it goes on (0: it is whole, or there is none).
struct Begin {
  int block, blocks, b, col;
};

}  // namespace cp
