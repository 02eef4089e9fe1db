// Host side of the operators that the decoding model runs on the kept tokens
// (rotary positions, cache append, attention over the cache): argument
// validation and launches.
#include <math.h>
#include <stddef.h>

#include "serve.h"

using namespace cp;

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
static size_t size_of(int dtype) { return dtype == CP_F32 ? 4 : dtype == CP_BF16 ? 2 : 1; }

// `rows` rows of `bytes` bytes, `apart` bytes from one to the next (a stride of the caller's may be any number: 128 bits
// hold what its products come to).
struct Area {
  __int128 at;
  int64_t rows;
  __int128 bytes, apart;
};
static Area area(const void* p, int64_t rows, __int128 bytes, __int128 apart) {
  if (!p || rows < 1 || bytes < 1) return Area{0, 0, 0, 0};
  Area x{(__int128)(uintptr_t)p, rows, bytes, apart};
  if (x.apart < 0) {  // from the lowest row on
    x.at += (x.rows - 1) * x.apart;
    x.apart = -x.apart;
  }
  if (x.apart == 0) x.rows = 1;
  return x;
}
static Area area(const void* p, __int128 bytes) { return area(p, 1, bytes, 0); }
// Rows of heads, as one stretch a token or sequence.
static Area area_of_heads(const void* p, int64_t n, const int64_t* stride, int64_t heads, int64_t D, int dtype) {
  const __int128 e = (__int128)size_of(dtype), far = e * (heads - 1) * stride[1];
  Area x = area(p, n, (far < 0 ? -far : far) + e * D, e * stride[0]);
  if (x.rows > 0 && far < 0) x.at += far;
  return x;
}
// Whether two share a byte.  Rows that take turns at one distance do not; of rows at two distances whose
// ranges overlap it is taken for granted.
static bool meet(const Area& a, const Area& b) {
  if (a.rows == 0 || b.rows == 0) return false;
  const auto end = [](const Area& x) { return x.at + (x.rows - 1) * x.apart + x.bytes; };
  if (a.at >= end(b) || b.at >= end(a)) return false;
  if (a.rows > 1 && b.rows > 1 && a.apart != b.apart) return true;
  const __int128 apart = a.rows > 1 ? a.apart : b.rows > 1 ? b.apart : 0;
  if (apart == 0) return true;
  const __int128 from = ((a.at - b.at) % apart + apart) % apart;  // of a's rows, behind b's
  return from < b.bytes || apart - from < a.bytes;
}

// Room for a call's element offsets (a stride times a size) in 64 bits.
constexpr int64_t kMaxSize = 0x7FFFFFFF;
// Keys of a sequence: an index a little past the last is still an int.
constexpr int64_t kMaxKeys = (int64_t)1 << 30;

static int rope_of(const cp_rope* r, int64_t D, int back, Rope* out) {
  *out = Rope{nullptr, 0, 0, 1.0f, back};
  if (!r) return CP_OK;
  if (r->rot < 0 || r->rot > D || r->rot % 2 != 0) return CP_EINVAL;
  if (r->layout != CP_ROPE_HALF && r->layout != CP_ROPE_INTERLEAVED) return CP_EINVAL;
  if (!isfinite(r->scale)) return CP_EINVAL;
  if (r->rot > 0 && (!r->inv_freq || !aligned(r->inv_freq, 8))) return CP_EINVAL;
  *out = Rope{r->inv_freq, r->rot / 2, r->layout == CP_ROPE_INTERLEAVED, r->scale, back};
  return CP_OK;
}

// Rows' description; where `tokens` is false there need not be memory.
static int rows_of(const cp_rows& r, int dtype, bool tokens, RowSet* out) {
  if (r.heads < 0 || r.heads > 65536) return CP_EINVAL;
  *out = RowSet{r.in, r.out, r.in_stride[0], r.in_stride[1], r.in_stride[2],
                r.out_stride[0], r.out_stride[1], r.out_stride[2], (int)r.heads};
  if (r.heads == 0 || !tokens) return CP_OK;
  if (!r.in || !r.out || !aligned(r.in, size_of(dtype)) || !aligned(r.out, size_of(dtype)))
    return CP_EINVAL;
  return CP_OK;
}

// A cache's description; the table is wanted by the calls that go through it.
static int cache_of(const cp_cache* c, bool with_memory, Cache* out) {
  // (what was compiled before there were 4-bit caches has no fields for them)
  if (!c || (c->struct_size != sizeof(cp_cache) &&
             (c->struct_size != offsetof(cp_cache, k_block) || c->dtype == CP_I4)))
    return CP_EINVAL;
  if (c->dtype != CP_F32 && c->dtype != CP_BF16 && c->dtype != CP_E4M3 && c->dtype != CP_I4) return CP_EINVAL;
  if (c->heads < 1 || c->heads > 65536 || c->D < 1 || c->page_size < 1 || c->pages < 0 ||
      c->table_width < 0 || c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0)
    return CP_EINVAL;
  const auto unaligned = [&](int64_t n) { return (c->dtype == CP_I4 ? n : n * (int64_t)size_of(c->dtype) * 2) % 32 != 0; };
  if (c->page_size > kMaxSize || c->table_width > kMaxSize || c->pages > kMaxSize)
    return CP_EINVAL;
  if (c->table_width * c->page_size > kMaxKeys) return CP_EUNSUPPORTED;
  if (c->D > 256 || unaligned(c->D)) return CP_EUNSUPPORTED;
  if (unaligned(c->page_stride) || unaligned(c->slot_stride) || unaligned(c->head_stride)) return CP_EINVAL;
  const bool fours = c->dtype == CP_I4;
  if (fours && (c->block_page_stride < 0 || c->block_slot_stride < 0 || c->block_head_stride < 0 ||
                c->block_page_stride % 4 != 0 || c->block_slot_stride % 4 != 0 || c->block_head_stride % 4 != 0))
    return CP_EINVAL;
  *out = Cache{};
  out->k = c->k;
  out->v = c->v;
  out->pages = c->pages;
  out->page_stride = c->page_stride;
  out->slot_stride = c->slot_stride;
  out->head_stride = c->head_stride;
  out->k_scale = c->k_scale;
  out->v_scale = c->v_scale;
  out->table = c->table;
  out->table_stride = c->table_stride;
  out->page_size = (int32_t)c->page_size;
  out->capacity = (int32_t)(c->table_width * c->page_size);
  out->heads = (int)c->heads;
  out->D = (int)c->D;
  if (fours) {
    out->k_block = (uint8_t*)c->k_block;
    out->v_block = (uint8_t*)c->v_block;
    out->block_page = c->block_page_stride;
    out->block_slot = c->block_slot_stride;
    out->block_head = c->block_head_stride;
  }
  if (!with_memory) return CP_OK;
  if (fours && (!aligned(c->k_block, 4) || !aligned(c->v_block, 4) || (c->pages > 0 && (!c->k_block || !c->v_block))))
    return CP_EINVAL;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4) || !aligned(c->table, 4))
    return CP_EINVAL;
  if (c->pages > 0 && (!c->k || !c->v)) return CP_EINVAL;
  if (c->table_width > 0 && !c->table) return CP_EINVAL;
  return CP_OK;
}

extern "C" {

int coverprune_rotary_frequencies(int64_t rot, double base, int stretch, double factor,
                                  double original, double low, double high, double* inv_freq) {
  if (rot < 2 || rot > 65536 || rot % 2 != 0 || !inv_freq || !(isfinite(base) && base > 1.0))
    return CP_EINVAL;
  if (stretch < CP_STRETCH_NONE || stretch > CP_STRETCH_INDEX) return CP_EINVAL;
  if (stretch != CP_STRETCH_NONE && !(isfinite(factor) && factor >= 1.0)) return CP_EINVAL;
  const bool ends = stretch == CP_STRETCH_TURNS || stretch == CP_STRETCH_INDEX;
  if (ends && !(isfinite(original) && original > 0.0 && isfinite(high) && low > 0.0 && low < high))
    return CP_EINVAL;
  if (stretch == CP_STRETCH_BASE) {
    if (rot == 2) return CP_EINVAL;  // a single pair has no slowest one to stretch to
    base *= pow(factor, (double)rot / (double)(rot - 2));
  }
  const double turn = 6.283185307179586477;
  double lo = 0.0, hi = 0.0;
  if (stretch == CP_STRETCH_INDEX) {
    const double last = (double)(rot - 1);
    lo = floor((double)rot * log(original / (turn * high)) / (2.0 * log(base)));
    hi = ceil((double)rot * log(original / (turn * low)) / (2.0 * log(base)));
    lo = fmin(fmax(lo, 0.0), last);
    hi = fmin(fmax(hi, 0.0), last);
    if (hi <= lo) hi = lo + 0.001;  // a step
  }
  for (int64_t i = 0; i < rot / 2; ++i) {
    const double f = pow(base, -2.0 * (double)i / (double)rot);
    double keep = 1.0;  // share of the unstretched speed
    if (stretch == CP_STRETCH_LINEAR)
      keep = 0.0;
    else if (stretch == CP_STRETCH_TURNS)
      keep = (original * f / turn - low) / (high - low);
    else if (stretch == CP_STRETCH_INDEX)
      keep = 1.0 - ((double)i - lo) / (hi - lo);
    keep = fmin(fmax(keep, 0.0), 1.0);
    const double slow = stretch == CP_STRETCH_NONE || stretch == CP_STRETCH_BASE ? f : f / factor;
    inv_freq[i] = keep * f + (1.0 - keep) * slow;
  }
  return CP_OK;
}

int coverprune_rotary(const cp_rows* rows, int n, int dtype, int64_t B, int64_t T, int64_t D,
                      const int64_t* pos, int64_t pos_stride, const cp_rope* rope, int inverse,
                      cp_stream_t stream) {
  if (dtype != CP_F32 && dtype != CP_BF16) return CP_EINVAL;
  if (!rows || n < 1 || n > kMaxRows || !rope || (inverse != 0 && inverse != 1)) return CP_EINVAL;
  if (B < 0 || T < 0 || B > kMaxSize || T > kMaxSize || D < 1 || D > 4096) return CP_EINVAL;
  RotaryArgs a{};
  CP_TRY_STATUS(rope_of(rope, D, inverse, &a.rope));
  int64_t heads = 0;
  for (int i = 0; i < n; ++i) {
    CP_TRY_STATUS(rows_of(rows[i], dtype, true, &a.set[i]));
    heads += rows[i].heads;
  }
  if (B == 0 || T == 0 || heads == 0) return CP_OK;
  if (!pos || !aligned(pos, 8)) return CP_EINVAL;
  a.n = n;
  a.B = B;
  a.T = T;
  a.D = (int)D;
  a.pos = pos;
  a.pos_stride = pos_stride;
  Stage st(CP_STAGE_ROTARY, (cudaStream_t)stream);
  return launch_rotary(a, dtype, (cudaStream_t)stream);
}

// Keys and values in one place: fine where they are read, but a call that writes both would mix them up.
static bool one_place(const Cache& c, bool fours) {
  return (c.k && c.k == c.v) || (fours && c.k_block && c.k_block == c.v_block);
}

int coverprune_cache_append(const cp_cache* cache, const void* k, const int64_t* k_stride,
                            const void* v, const int64_t* v_stride, int dtype, int64_t T,
                            const int32_t* starts, const int32_t* lens, int64_t B,
                            const int64_t* pos, const cp_rope* rope, const cp_rows* q,
                            int32_t* new_lens, int32_t* status, cp_stream_t stream) {
  if (dtype != CP_F32 && dtype != CP_BF16) return CP_EINVAL;
  if (T < 0 || B < 0 || T > kMaxSize || B > (1 << 24)) return CP_EINVAL;
  AppendArgs a{};
  CP_TRY_STATUS(cache_of(cache, true, &a.cache));
  if (cache->dtype != CP_E4M3 && cache->dtype != CP_I4 && cache->dtype != dtype) return CP_EUNSUPPORTED;
  CP_TRY_STATUS(rope_of(rope, cache->D, 0, &a.rope));
  if (q) CP_TRY_STATUS(rows_of(*q, dtype, T > 0, &a.q));
  if (!starts && T != B) return CP_EINVAL;
  if (B == 0) return CP_OK;  // whatever rows there are, are padding
  if (!lens || !aligned(lens, 4) || !aligned(starts, 4) || !aligned(new_lens, 4) ||
      !aligned(status, 4) || !aligned(pos, 8))
    return CP_EINVAL;
  // blocks read the lengths and starts while others write
  const Area lens_out = area(new_lens, 4 * B);
  if (meet(lens_out, area(lens, 4 * B)) || meet(lens_out, area(starts, 4 * (B + 1)))) return CP_EINVAL;
  if (T > 0 && (!k || !v || !k_stride || !v_stride || !aligned(k, size_of(dtype)) ||
                !aligned(v, size_of(dtype))))
    return CP_EINVAL;
  if (T == 0 && !new_lens) return CP_OK;
  if (T > 0 && cache->dtype == CP_I4 && one_place(a.cache, true)) return CP_EINVAL;
  a.k = k;
  a.v = v;
  if (T > 0) {
    a.k_t = k_stride[0];
    a.k_h = k_stride[1];
    a.v_t = v_stride[0];
    a.v_h = v_stride[1];
  }
  a.T = T;
  a.starts = starts;
  a.lens = lens;
  a.B = (int)B;
  a.pos = pos;
  a.new_lens = new_lens;
  a.status = status;
  Stage st(CP_STAGE_CACHE, (cudaStream_t)stream);
  return launch_cache_append(a, dtype, cache->dtype, (cudaStream_t)stream);
}

// Where the parts of the attention's workspace begin: its own, and with weights the lse and the scores.
struct Room {
  size_t decode, lse, scores, all;
};
static int room_of(int64_t B, int64_t Hq, const Cache& c, int cache_dtype, Room* room) {
  const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Room& r = *room;
  r.decode = decode_ws_bytes(Hq, c.heads, c.D, cache_dtype);
  r.lse = up(r.decode);
  r.scores = r.lse + up(4 * (size_t)B * (size_t)Hq);
  int64_t cols = 0, pitch = 0;
  score_shape(cache_dtype, Hq, c.heads, &cols, &pitch);
  // (B heads <= 2^24 and tiles times pitch < 2^18 leave what is below 2^42)
  if (c.capacity > 0 && B * cols * pitch > ((int64_t)1 << 60) / c.capacity) return CP_EUNSUPPORTED;
  r.all = r.scores + 4 * (size_t)(B * cols * pitch) * (size_t)c.capacity;
  return CP_OK;
}

static int check_decode(int64_t B, int64_t Hq, const cp_cache* cache, bool with_memory, Cache* c) {
  CP_TRY_STATUS(cache_of(cache, with_memory, c));
  if (B < 0 || Hq < 0 || Hq > 65536 || Hq % cache->heads != 0) return CP_EINVAL;
  if (B > (1 << 24) / cache->heads) return CP_EUNSUPPORTED;
  return CP_OK;
}

int coverprune_decode_workspace_size(int64_t B, int64_t Hq, const cp_cache* cache,
                                     size_t* bytes) {
  if (!bytes) return CP_EINVAL;
  Cache c;
  CP_TRY_STATUS(check_decode(B, Hq, cache, false, &c));
  *bytes = decode_ws_bytes(Hq, c.heads, c.D, cache->dtype);
  return CP_OK;
}

// The attention's arguments; `weights`: its scores are left behind for them, in the workspace's rest.
static int attend(const void* q, const int64_t* q_stride, int dtype, int64_t B, int64_t Hq,
                  const cp_cache* cache, const int32_t* lens, const uint8_t* keep,
                  int64_t keep_stride, float scale, int64_t window, void* out,
                  const int64_t* out_stride, float* lse, bool weights, float* weight,
                  int64_t weight_stride, void* ws, size_t ws_bytes, int32_t* status,
                  cp_stream_t stream) {
  if (dtype != CP_F32 && dtype != CP_BF16) return CP_EINVAL;
  DecodeArgs a{};
  CP_TRY_STATUS(check_decode(B, Hq, cache, true, &a.cache));
  if ((dtype == CP_F32) != (cache->dtype == CP_F32)) return CP_EUNSUPPORTED;
  if (!isfinite(scale) || window < 0 || weight_stride < 0) return CP_EINVAL;
  if (B == 0 || Hq == 0) return CP_OK;
  if (!q || !q_stride || !out || !out_stride || !lens || !aligned(q, size_of(dtype)) ||
      !aligned(out, size_of(dtype)) || !aligned(lens, 4) || !aligned(lse, 4) ||
      !aligned(status, 4))
    return CP_EINVAL;
  if (weights && ((!weight && a.cache.capacity > 0) || !aligned(weight, 4) || (B > 1 && weight_stride < a.cache.capacity)))
    return CP_EINVAL;
  Room room;
  const int st_room = room_of(B, Hq, a.cache, cache->dtype, &room);
  if (weights) CP_TRY_STATUS(st_room);
  if (!ws || !aligned(ws, 256) || ws_bytes < (weights ? room.all : room.decode)) return CP_EWORKSPACE;
  if (weights) {  // written while others are read or written
    const Area w = area(weight, B, 4 * (__int128)a.cache.capacity, 4 * (__int128)weight_stride);
    const Area others[] = {area_of_heads(q, B, q_stride, Hq, a.cache.D, dtype), area_of_heads(out, B, out_stride, Hq, a.cache.D, dtype),
                           area(lse, 4 * (__int128)B * Hq), area(lens, 4 * B), area(keep, B, a.cache.capacity, keep_stride),
                           area(ws, room.all)};
    for (const Area& x : others)
      if (meet(w, x)) return CP_EINVAL;
  }
  a.q = q;
  a.q_b = q_stride[0];
  a.q_h = q_stride[1];
  a.out = out;
  a.o_b = out_stride[0];
  a.o_h = out_stride[1];
  a.B = (int)B;
  a.Hq = (int)Hq;
  a.lens = lens;
  a.keep = keep;
  a.keep_stride = keep_stride;
  a.scale = scale;
  a.window = window;
  a.lse = lse;
  a.ws = ws;
  a.status = status;
  Stage st(CP_STAGE_ATTEND, (cudaStream_t)stream);
  if (!weights) return launch_decode(a, cache->dtype, (cudaStream_t)stream);
  if (!lse) a.lse = (float*)((char*)ws + room.lse);
  a.scores = (float*)((char*)ws + room.scores);
  int64_t cols = 0, pitch = 0;
  score_shape(cache->dtype, Hq, a.cache.heads, &cols, &pitch);
  a.score_cols = (int)cols;
  a.score_pitch = (int)pitch;
  CP_TRY_STATUS(launch_decode_scores(a, cache->dtype, (cudaStream_t)stream));
  return launch_weigh(a, cache->dtype, weight, weight_stride, (cudaStream_t)stream);
}

int coverprune_decode_attention(const void* q, const int64_t* q_stride, int dtype, int64_t B,
                                int64_t Hq, const cp_cache* cache, const int32_t* lens,
                                const uint8_t* keep, int64_t keep_stride, float scale,
                                int64_t window, void* out, const int64_t* out_stride, float* lse,
                                void* ws, size_t ws_bytes, int32_t* status, cp_stream_t stream) {
  return attend(q, q_stride, dtype, B, Hq, cache, lens, keep, keep_stride, scale, window, out, out_stride, lse,
                false, nullptr, 0, ws, ws_bytes, status, stream);
}

int coverprune_decode_weigh_workspace_size(int64_t B, int64_t Hq, const cp_cache* cache,
                                           size_t* bytes) {
  if (!bytes) return CP_EINVAL;
  Cache c;
  CP_TRY_STATUS(check_decode(B, Hq, cache, false, &c));
  Room room;
  CP_TRY_STATUS(room_of(B, Hq, c, cache->dtype, &room));
  *bytes = room.all;
  return CP_OK;
}

int coverprune_decode_attention_weigh(const void* q, const int64_t* q_stride, int dtype, int64_t B,
                                      int64_t Hq, const cp_cache* cache, const int32_t* lens,
                                      const uint8_t* keep, int64_t keep_stride, float scale,
                                      int64_t window, void* out, const int64_t* out_stride,
                                      float* lse, float* weight, int64_t weight_stride, void* ws,
                                      size_t ws_bytes, int32_t* status, cp_stream_t stream) {
  return attend(q, q_stride, dtype, B, Hq, cache, lens, keep, keep_stride, scale, window, out, out_stride, lse,
                true, weight, weight_stride, ws, ws_bytes, status, stream);
}

int coverprune_cache_read(const cp_cache* cache, int64_t T, const int32_t* starts,
                          const int32_t* lens, int64_t B, void* k, const int64_t* k_stride,
                          void* v, const int64_t* v_stride, int dtype, int32_t* status,
                          cp_stream_t stream) {
  if (dtype != CP_F32 && dtype != CP_BF16) return CP_EINVAL;
  if (T < 0 || B < 0 || T > kMaxSize || B > (1 << 24)) return CP_EINVAL;
  ReadArgs a{};
  CP_TRY_STATUS(cache_of(cache, true, &a.cache));
  if (cache->dtype != CP_E4M3 && cache->dtype != CP_I4 && cache->dtype != dtype) return CP_EUNSUPPORTED;
  if (!starts && T != B) return CP_EINVAL;
  if (B == 0 || T == 0) return CP_OK;
  if (!lens || !aligned(lens, 4) || !aligned(starts, 4) || !aligned(status, 4) || !k || !v || !k_stride ||
      !v_stride || !aligned(k, size_of(dtype)) || !aligned(v, size_of(dtype)) || k == v)
    return CP_EINVAL;
  a.k = k;
  a.v = v;
  a.k_t = k_stride[0];
  a.k_h = k_stride[1];
  a.v_t = v_stride[0];
  a.v_h = v_stride[1];
  a.T = T;
  a.starts = starts;
  a.lens = lens;
  a.B = (int)B;
  a.status = status;
  Stage st(CP_STAGE_CACHE, (cudaStream_t)stream);
  return launch_cache_read(a, dtype, cache->dtype, (cudaStream_t)stream);
}

int coverprune_cache_evict(const cp_cache* cache, const int32_t* lens, int64_t B,
                           const float* weight, int64_t weight_stride, int64_t left,
                           int64_t first, int64_t recent, int32_t* new_lens, float* new_weight,
                           int64_t new_weight_stride, int64_t new_weight_width, int32_t* kept,
                           int32_t* status, cp_stream_t stream) {
  EvictArgs a{};
  CP_TRY_STATUS(cache_of(cache, true, &a.cache));
  constexpr int64_t far = (int64_t)1 << 36;  // between rows of weights: their offsets stay within 64 bits
  if (B < 0 || B > (1 << 24) || left < 0 || first < 0 || recent < 0 || first > left || recent > left - first ||
      weight_stride > far || new_weight_stride > far || weight_stride < 0 || new_weight_stride < 0 || new_weight_width < 0 || new_weight_width > kMaxSize)
    return CP_EINVAL;
  if (left > kMaxKeys || left * B >= (int64_t)1 << 35) return CP_EUNSUPPORTED;
  if (B == 0) return CP_OK;
  if (!lens || !aligned(lens, 4) || !aligned(weight, 4) || !aligned(new_lens, 4) || !aligned(new_weight, 4) ||
      !aligned(kept, 4) || !aligned(status, 4) || (left > 0 && !kept) || (a.cache.capacity > 0 && !weight))
    return CP_EINVAL;
  if (new_weight && B > 1 && new_weight_stride < new_weight_width) return CP_EINVAL;
  if (one_place(a.cache, cache->dtype == CP_I4)) return CP_EINVAL;
  // what a block writes others still read
  const Area in[2] = {area(lens, 4 * B), area(weight, B, 4 * (__int128)a.cache.capacity, 4 * (__int128)weight_stride)};
  const Area out[3] = {area(new_lens, 4 * B), area(new_weight, B, 4 * (__int128)new_weight_width, 4 * (__int128)new_weight_stride),
                       area(kept, 4 * left * B)};
  for (int i = 0; i < 3; ++i) {
    for (const Area& x : in)
      if (meet(out[i], x)) return CP_EINVAL;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return CP_EINVAL;
  }
  a.lens = lens;
  a.B = (int)B;
  a.weight = weight;
  a.weight_stride = weight_stride;
  a.left = (int)left;
  a.first = (int)first;
  a.recent = (int)recent;
  a.new_lens = new_lens;
  a.new_weight = new_weight;
  a.new_weight_stride = new_weight_stride;
  a.new_weight_width = new_weight_width;
  a.kept = kept;
  a.status = status;
  Stage st(CP_STAGE_CACHE, (cudaStream_t)stream);
  return launch_cache_evict(a, cache->dtype, (cudaStream_t)stream);
}

}  // extern "C"
