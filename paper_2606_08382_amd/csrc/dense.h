// Internal interface between the host side (dense_host.cpp) and the kernels (rope.hip,
// dense_cache.hip, dense_attn.hip) of uncompressed layers.  Not part of the public ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "starkv.h"

namespace starkv {

// Records the detail string of starkv_last_error (starkv_host.cpp) and returns st.
starkv_status fail_with(starkv_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

struct Pair { float x, y; };

constexpr int kMaxRotaryPairs = 256;

struct RopeParams {
  const void* x;
  void* out;
  const int32_t* positions;
  int64_t xs_b, xs_t, xs_h, os_b, os_t, os_h;   // element strides
  int64_t tokens;                               // B * n
  int32_t n, heads, d, rotary, dtype, interleaved;
  int32_t units;                                // work units of a head: rotated, then copied
  int32_t rot_units;
  int32_t heads_per_thread, head_groups;
  int32_t streaming;                            // more bytes than the caches hold
  float gain, sine;                             // factor on cos; on sin (its sign: inverse)
  double turns[kMaxRotaryPairs];                // f_j / 2 pi
};

// The cache of a plan, as every kernel sees it.
struct DenseCache {
  uint8_t* codes;
  Pair* scales;
  uint16_t* tails;
  const int32_t* table;
  int32_t batch, n_kv, d, shift;                // T = 1 << shift
  int32_t blocks_per_head, n_blocks, capacity;
  int32_t e4m3, bf16;
};

struct DenseAppendParams {
  DenseCache c;
  const uint16_t* x[2];                         // keys, values
  int64_t xs_b[2], xs_t[2], xs_h[2];
  const int32_t* pos;
  const int32_t* n_new_dev;
  int32_t n_new;
  int32_t wide[2];                              // rows 16-byte aligned
};

struct DenseReadParams {
  DenseCache c;
  void* out[2];
  int64_t os_b[2], os_t[2], os_h[2];
  const int32_t* ctx_len;
  const int32_t* start;
  int32_t n, out_dtype;
  int32_t wide[2];                              // rows aligned to four elements
};

struct DenseEvictParams {
  const int32_t* table;
  int32_t* table_out;
  const float* weights;
  float* weights_out;
  const int32_t* ctx_len;
  int32_t* ctx_out;
  int32_t batch, n_kv, shift, blocks_per_head, capacity;
  int32_t keep, sink, recent;
};

// A sequence's parts in the partials of an attention pass.
struct Slots {
  int32_t first, count, ctx, pad;
};

struct DenseAttnParams {
  DenseCache c;
  const uint16_t* q;
  uint16_t* out;
  int64_t qs_b, qs_t, qs_h, os_b, os_t, os_h;
  const int32_t* q_len;
  const int32_t* ctx_len;
  float* weights;
  Slots* slots;                                 // [B]
  float* part_o;                                // [slot][H_kv][rows][d], normalized
  Pair* part_ml;                            // [slot][H_kv][rows]: (reference, sum)
  Pair* sub;                                // [B*H_kv][subtile][rows]: (sum, reference)
  int32_t n_q, group, rows;                     // rows = n_q * group
  int32_t max_ctx, ranges, min_units, sub_per_head;   // min_units: of a range
  int32_t q_wide, out_wide;                     // query rows 16-, output rows 8-byte aligned
  float scale_log2;                             // softmax scale * log2(e)
};

// Query rows of a KV head that the split kernel takes; above them the chunk kernel, in row tiles.
constexpr int kSplitRows = 64;
constexpr int kChunkRows = 128;

int launch_rope(const RopeParams& p, bool wide, void* stream);
int launch_dense_append(const DenseAppendParams& p, void* stream);
int launch_dense_read(const DenseReadParams& p, void* stream);
int launch_dense_evict(const DenseEvictParams& p, void* stream);
int launch_dense_attn(const DenseAttnParams& p, void* stream);

}  // namespace starkv
