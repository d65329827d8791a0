// Host side of the entry points for uncompressed layers: plans, validation, cache layout,
// workspace sizes and launches.  No device allocation, no synchronization.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "dense.h"

using namespace starkv;

struct starkv_rope_plan {
  starkv_rope_config cfg;
  double gain;
  double turns[kMaxRotaryPairs];          // f_j / 2 pi
};

struct starkv_dense_plan {
  starkv_dense_config cfg;
  starkv_dense_layout layout;
  int32_t shift;                          // log2(block_tokens)
  double scale;
};

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr int kMaxDenseCtx = 524288;
int64_t align256(int64_t x) { return (x + 255) / 256 * 256; }
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

starkv_status hip_status(int e, const char* what) {
  if (e != hipSuccess)
    return fail_with(STARKV_ERR_HIP, "%s: %s", what, hipGetErrorString((hipError_t)e));
  return STARKV_OK;
}

// The strides of a [B][n][H][d] array, packed if s is NULL.
starkv_strides strides_of(const starkv_strides* s, int64_t n, int64_t heads, int64_t d) {
  if (s) return *s;
  return {n * heads * d, heads * d, d};
}

// Rows of an output must not overlap.
bool rows_apart(const starkv_strides& s, int64_t B, int64_t n, int64_t heads, int64_t d) {
  return (B <= 1 || std::llabs(s.batch) >= d) && (n <= 1 || std::llabs(s.token) >= d) &&
         (heads <= 1 || std::llabs(s.head) >= d);
}

// Whether every row of the array starts on a multiple of `bytes`.
bool rows_wide(const void* p, const starkv_strides& s, int64_t elem, int bytes = 16) {
  return !misaligned(p, bytes) && s.batch * elem % bytes == 0 && s.token * elem % bytes == 0 &&
         s.head * elem % bytes == 0;
}

bool is_dtype16(int dt) { return dt == STARKV_DT_F16 || dt == STARKV_DT_BF16; }

}  // namespace

extern "C" {

// ------------------------------------------------------------------------- rotary positions

starkv_status starkv_rope_plan_create(const starkv_rope_config* c, starkv_rope_plan** out) {
  if (!out) return fail_with(STARKV_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!c) return fail_with(STARKV_ERR_INVALID_ARG, "config is NULL");
  if (c->head_dim < 2 || c->head_dim % 2)
    return fail_with(STARKV_ERR_INVALID_ARG, "head_dim %d: need a positive even number", c->head_dim);
  if (c->head_dim > 2 * kMaxRotaryPairs)
    return fail_with(STARKV_ERR_UNSUPPORTED, "head_dim %d > %d", c->head_dim, 2 * kMaxRotaryPairs);
  const int R = c->rotary_dim;
  if (R < 2 || R % 2 || R > c->head_dim)
    return fail_with(STARKV_ERR_INVALID_ARG, "rotary_dim %d: need an even number in [2, %d]", R, c->head_dim);
  if (c->layout != STARKV_ROPE_HALF && c->layout != STARKV_ROPE_INTERLEAVED)
    return fail_with(STARKV_ERR_INVALID_ARG, "layout %d", c->layout);
  if (c->scaling < STARKV_ROPE_PLAIN || c->scaling > STARKV_ROPE_YARN)
    return fail_with(STARKV_ERR_INVALID_ARG, "scaling %d", c->scaling);
  if (!is_dtype16(c->dtype) && c->dtype != STARKV_DT_F32)
    return fail_with(STARKV_ERR_INVALID_ARG, "dtype %d", c->dtype);
  if (!(c->theta > 1.0) || !std::isfinite(c->theta))
    return fail_with(STARKV_ERR_INVALID_ARG, "theta must be finite and > 1");
  const bool scaled = c->scaling != STARKV_ROPE_PLAIN;
  if (scaled && (!(c->factor >= 1.0) || !std::isfinite(c->factor)))
    return fail_with(STARKV_ERR_INVALID_ARG, "factor must be finite and >= 1");
  if (c->scaling == STARKV_ROPE_NTK && R <= 2)
    return fail_with(STARKV_ERR_INVALID_ARG, "rotary_dim 2 has no scaled base");
  if (!(c->gain >= 0.0) || !std::isfinite(c->gain))
    return fail_with(STARKV_ERR_INVALID_ARG, "gain must be finite and positive, or 0");
  const bool banded = c->scaling == STARKV_ROPE_BANDS || c->scaling == STARKV_ROPE_YARN;
  double lo = c->turns_low, hi = c->turns_high;
  if (banded) {
    if (c->original_ctx < 1) return fail_with(STARKV_ERR_INVALID_ARG, "original_ctx %d < 1", c->original_ctx);
    if (lo == 0.0 && hi == 0.0) {
      lo = 1.0;
      hi = c->scaling == STARKV_ROPE_BANDS ? 4.0 : 32.0;
    }
    if (!(lo > 0.0) || !(hi > lo) || !std::isfinite(hi))
      return fail_with(STARKV_ERR_INVALID_ARG, "need 0 < turns_low < turns_high");
  }
  starkv_rope_plan* P = new (std::nothrow) starkv_rope_plan();
  if (!P) return fail_with(STARKV_ERR_INVALID_ARG, "out of host memory");
  P->cfg = *c;
  const double s = c->factor, L0 = c->original_ctx;
  const double theta = c->scaling == STARKV_ROPE_NTK ? c->theta * std::pow(s, R / (R - 2.0)) : c->theta;
  double j0 = 0.0, j1 = 0.0;
  if (c->scaling == STARKV_ROPE_YARN) {
    auto at = [&](double n) { return R * std::log(L0 / (kTwoPi * n)) / (2.0 * std::log(theta)); };
    j0 = std::max(std::floor(at(hi)), 0.0);
    j1 = std::min(std::ceil(at(lo)), R - 1.0);
  }
  for (int j = 0; j < R / 2; ++j) {
    double f = std::pow(theta, -2.0 * j / R);
    if (c->scaling == STARKV_ROPE_LINEAR) f /= s;
    if (c->scaling == STARKV_ROPE_BANDS) {
      const double w = std::min(std::max((L0 * f / kTwoPi - lo) / (hi - lo), 0.0), 1.0);
      f *= w + (1.0 - w) / s;
    }
    if (c->scaling == STARKV_ROPE_YARN) {
      const double r = std::min(std::max((j - j0) / std::max(j1 - j0, 1e-3), 0.0), 1.0);
      f = f * (1.0 - r) + f / s * r;
    }
    P->turns[j] = f / kTwoPi;
  }
  P->gain = c->gain > 0.0 ? c->gain : c->scaling == STARKV_ROPE_YARN ? 0.1 * std::log(s) + 1.0 : 1.0;
  *out = P;
  return STARKV_OK;
}

void starkv_rope_plan_destroy(starkv_rope_plan* plan) { delete plan; }

starkv_status starkv_rope(const starkv_rope_plan* P, const void* x, const starkv_strides* xs,
                          void* out, const starkv_strides* os, const int32_t* positions,
                          int32_t batch, int32_t n_tokens, int32_t n_heads, int32_t inverse,
                          starkv_stream_t stream) {
  if (!P) return fail_with(STARKV_ERR_INVALID_ARG, "plan is NULL");
  if (batch < 1 || n_tokens < 1 || n_heads < 1)
    return fail_with(STARKV_ERR_INVALID_ARG, "batch, n_tokens and n_heads must be positive");
  if (!x || !out || !positions) return fail_with(STARKV_ERR_INVALID_ARG, "NULL device pointer");
  const int elem = P->cfg.dtype == STARKV_DT_F32 ? 4 : 2;
  if (misaligned(x, elem) || misaligned(out, elem) || misaligned(positions, 4))
    return fail_with(STARKV_ERR_ALIGNMENT, "x, out or positions not aligned to their elements");
  const int D = P->cfg.head_dim, R = P->cfg.rotary_dim;
  const starkv_strides a = strides_of(xs, n_tokens, n_heads, D), o = strides_of(os, n_tokens, n_heads, D);
  if (!rows_apart(o, batch, n_tokens, n_heads, D))
    return fail_with(STARKV_ERR_INVALID_ARG, "rows of out overlap");
  if (x == out && ((batch > 1 && a.batch != o.batch) || (n_tokens > 1 && a.token != o.token) ||
                   (n_heads > 1 && a.head != o.head)))
    return fail_with(STARKV_ERR_INVALID_ARG, "in place with other strides");
  RopeParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x;
  p.out = out;
  p.positions = positions;
  p.xs_b = a.batch;
  p.xs_t = a.token;
  p.xs_h = a.head;
  p.os_b = o.batch;
  p.os_t = o.token;
  p.os_h = o.head;
  p.tokens = (int64_t)batch * n_tokens;
  p.n = n_tokens;
  p.heads = n_heads;
  p.d = D;
  p.rotary = R;
  p.dtype = P->cfg.dtype;
  p.interleaved = P->cfg.layout == STARKV_ROPE_INTERLEAVED;
  p.gain = (float)P->gain;
  p.sine = inverse ? -p.gain : p.gain;
  std::memcpy(p.turns, P->turns, sizeof(p.turns));
  const int E = 16 / elem;
  const bool wide = rows_wide(x, a, elem) && rows_wide(out, o, elem) && D % E == 0 &&
                    (p.interleaved ? R : R / 2) % E == 0;
  p.rot_units = wide ? (p.interleaved ? R : R / 2) / E : R / 2;
  p.units = p.rot_units + (wide ? (D - R) / E : D - R);
  // Heads share a token's angles: a thread takes two, where that leaves 2^17 threads (two waves per
  // SIMD).  More heads a thread leave too few rows in flight (16384 tokens of 40 heads: 60 us with
  // two, 62 with three, 65 with four, 68 with eight, 82 with one).
  const int64_t per = p.tokens * p.units * n_heads >= (int64_t)1 << 18 ? 2 : 1;
  p.heads_per_thread = (int32_t)per;
  p.head_groups = (n_heads + p.heads_per_thread - 1) / p.heads_per_thread;
  // (half of the 256 MB of last-level cache)
  p.streaming = p.tokens * n_heads * D * elem * 2 > (int64_t)128 << 20;
  const double threads = (double)p.tokens * p.head_groups * p.units;
  if (threads > 256.0 * 0x7fffffff)
    return fail_with(STARKV_ERR_UNSUPPORTED, "%lld tokens of %d heads in one call", (long long)p.tokens, n_heads);
  return hip_status(launch_rope(p, wide, static_cast<void*>(stream)), "rope launch");
}

// --------------------------------------------------------------------------- 8-bit cache

starkv_status starkv_dense_plan_create(const starkv_dense_config* c, starkv_dense_plan** out) {
  if (!out) return fail_with(STARKV_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (!c) return fail_with(STARKV_ERR_INVALID_ARG, "config is NULL");
  if (c->batch < 1) return fail_with(STARKV_ERR_INVALID_ARG, "batch %d < 1", c->batch);
  if (c->n_kv_heads < 1 || c->n_q_heads < 1)
    return fail_with(STARKV_ERR_INVALID_ARG, "head counts must be positive");
  if (c->n_q_heads % c->n_kv_heads)
    return fail_with(STARKV_ERR_INVALID_ARG, "n_q_heads %d not a multiple of n_kv_heads %d",
                     c->n_q_heads, c->n_kv_heads);
  if (c->capacity < 1) return fail_with(STARKV_ERR_INVALID_ARG, "capacity %d < 1", c->capacity);
  if (c->code != STARKV_CODE_INT8 && c->code != STARKV_CODE_E4M3)
    return fail_with(STARKV_ERR_INVALID_ARG, "code %d", c->code);
  if (!is_dtype16(c->dtype)) return fail_with(STARKV_ERR_INVALID_ARG, "dtype %d", c->dtype);
  const int T = c->block_tokens;
  if (T != 16 && T != 32 && T != 64 && T != 128)
    return fail_with(STARKV_ERR_INVALID_ARG, "block_tokens %d not 16, 32, 64 or 128", T);
  if (c->n_blocks < 1) return fail_with(STARKV_ERR_INVALID_ARG, "n_blocks %d < 1", c->n_blocks);
  if (!(c->softmax_scale >= 0.0) || c->softmax_scale > 1e38)
    return fail_with(STARKV_ERR_INVALID_ARG, "softmax_scale must be positive and at most 1e38, or 0");
  if (!c->block_table) return fail_with(STARKV_ERR_INVALID_ARG, "block_table is NULL");
  if (misaligned(c->block_table, 4))
    return fail_with(STARKV_ERR_ALIGNMENT, "block_table not 4-byte aligned");
  if (c->batch > 32767) return fail_with(STARKV_ERR_UNSUPPORTED, "batch %d > 32767", c->batch);
  if (c->n_kv_heads > STARKV_MAX_KV_HEADS)
    return fail_with(STARKV_ERR_UNSUPPORTED, "n_kv_heads %d > %d", c->n_kv_heads, STARKV_MAX_KV_HEADS);
  if (c->n_q_heads > STARKV_MAX_Q_HEADS)
    return fail_with(STARKV_ERR_UNSUPPORTED, "n_q_heads %d > %d", c->n_q_heads, STARKV_MAX_Q_HEADS);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail_with(STARKV_ERR_UNSUPPORTED, "head_dim %d not 64 or 128", c->head_dim);
  if (c->capacity > kMaxDenseCtx)
    return fail_with(STARKV_ERR_UNSUPPORTED, "capacity %d > %d", c->capacity, kMaxDenseCtx);
  if ((int64_t)c->n_blocks * T > ((int64_t)1 << 31) - 1)
    return fail_with(STARKV_ERR_UNSUPPORTED, "pool of %d x %d tokens too large", c->n_blocks, T);
  starkv_dense_plan* P = new (std::nothrow) starkv_dense_plan();
  if (!P) return fail_with(STARKV_ERR_INVALID_ARG, "out of host memory");
  P->cfg = *c;
  P->shift = T == 16 ? 4 : T == 32 ? 5 : T == 64 ? 6 : 7;
  P->scale = c->softmax_scale > 0.0 ? c->softmax_scale : 1.0 / std::sqrt((double)c->head_dim);
  starkv_dense_layout& L = P->layout;
  std::memset(&L, 0, sizeof(L));
  L.block_bytes = (int64_t)2 * T * c->head_dim;
  L.tail_bytes = (int64_t)2 * 2 * T * c->head_dim * 2;
  L.blocks_per_head = (c->capacity + T - 1) / T;
  L.code_offset = 0;
  L.scale_offset = align256(c->n_blocks * L.block_bytes);
  L.tail_offset = L.scale_offset + align256((int64_t)c->n_blocks * 8);
  L.total_bytes = L.tail_offset + align256((int64_t)c->batch * c->n_kv_heads * L.tail_bytes);
  *out = P;
  return STARKV_OK;
}

void starkv_dense_plan_destroy(starkv_dense_plan* plan) { delete plan; }

size_t starkv_dense_cache_bytes(const starkv_dense_plan* P) {
  return P ? (size_t)P->layout.total_bytes : 0;
}

starkv_status starkv_dense_cache_layout(const starkv_dense_plan* P, starkv_dense_layout* out) {
  if (!P || !out) return fail_with(STARKV_ERR_INVALID_ARG, "plan or out is NULL");
  *out = P->layout;
  return STARKV_OK;
}

static DenseCache cache_of(const starkv_dense_plan* P, const void* cache) {
  const starkv_dense_config& c = P->cfg;
  DenseCache d;
  std::memset(&d, 0, sizeof(d));
  uint8_t* base = static_cast<uint8_t*>(const_cast<void*>(cache));
  d.codes = base + P->layout.code_offset;
  d.scales = reinterpret_cast<Pair*>(base + P->layout.scale_offset);
  d.tails = reinterpret_cast<uint16_t*>(base + P->layout.tail_offset);
  d.table = c.block_table;
  d.batch = c.batch;
  d.n_kv = c.n_kv_heads;
  d.d = c.head_dim;
  d.shift = P->shift;
  d.blocks_per_head = P->layout.blocks_per_head;
  d.n_blocks = c.n_blocks;
  d.capacity = c.capacity;
  d.e4m3 = c.code == STARKV_CODE_E4M3;
  d.bf16 = c.dtype == STARKV_DT_BF16;
  return d;
}

static starkv_status check_cache(const starkv_dense_plan* P, const void* cache) {
  if (!P) return fail_with(STARKV_ERR_INVALID_ARG, "plan is NULL");
  if (!cache) return fail_with(STARKV_ERR_INVALID_ARG, "cache is NULL");
  if (misaligned(cache, 256)) return fail_with(STARKV_ERR_ALIGNMENT, "cache not 256-byte aligned");
  return STARKV_OK;
}

starkv_status starkv_dense_append(const starkv_dense_plan* P, void* cache, const void* k,
                                  const starkv_strides* ks, const void* v,
                                  const starkv_strides* vs, const int32_t* pos_dev,
                                  int32_t n_new, const int32_t* n_new_dev,
                                  starkv_stream_t stream) {
  starkv_status st = check_cache(P, cache);
  if (st != STARKV_OK) return st;
  if (n_new < 1) return fail_with(STARKV_ERR_INVALID_ARG, "n_new %d < 1", n_new);
  if (!k || !v || !pos_dev) return fail_with(STARKV_ERR_INVALID_ARG, "NULL device pointer");
  if (misaligned(k, 2) || misaligned(v, 2)) return fail_with(STARKV_ERR_ALIGNMENT, "k or v not 2-byte aligned");
  if (misaligned(pos_dev, 4) || misaligned(n_new_dev, 4))
    return fail_with(STARKV_ERR_ALIGNMENT, "pos or n_new not 4-byte aligned");
  DenseAppendParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = cache_of(P, cache);
  const void* x[2] = {k, v};
  const starkv_strides* s[2] = {ks, vs};
  for (int i = 0; i < 2; ++i) {
    const starkv_strides a = strides_of(s[i], n_new, P->cfg.n_kv_heads, P->cfg.head_dim);
    p.x[i] = static_cast<const uint16_t*>(x[i]);
    p.xs_b[i] = a.batch;
    p.xs_t[i] = a.token;
    p.xs_h[i] = a.head;
    p.wide[i] = rows_wide(x[i], a, 2);
  }
  p.pos = pos_dev;
  p.n_new_dev = n_new_dev;
  p.n_new = n_new;
  return hip_status(launch_dense_append(p, static_cast<void*>(stream)), "dense append launch");
}

starkv_status starkv_dense_read(const starkv_dense_plan* P, const void* cache,
                                const int32_t* ctx_len_dev, const int32_t* start_dev, int32_t n,
                                void* k_out, const starkv_strides* ks, void* v_out,
                                const starkv_strides* vs, int32_t out_dtype,
                                starkv_stream_t stream) {
  starkv_status st = check_cache(P, cache);
  if (st != STARKV_OK) return st;
  if (n < 1) return fail_with(STARKV_ERR_INVALID_ARG, "n %d < 1", n);
  if (!is_dtype16(out_dtype) && out_dtype != STARKV_DT_F32)
    return fail_with(STARKV_ERR_INVALID_ARG, "out_dtype %d", out_dtype);
  if (!ctx_len_dev || !start_dev || (!k_out && !v_out))
    return fail_with(STARKV_ERR_INVALID_ARG, "NULL device pointer");
  const int elem = out_dtype == STARKV_DT_F32 ? 4 : 2;
  if (misaligned(ctx_len_dev, 4) || misaligned(start_dev, 4) || misaligned(k_out, elem) ||
      misaligned(v_out, elem))
    return fail_with(STARKV_ERR_ALIGNMENT, "pointer not aligned to its elements");
  DenseReadParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = cache_of(P, cache);
  void* o[2] = {k_out, v_out};
  const starkv_strides* s[2] = {ks, vs};
  for (int i = 0; i < 2; ++i) {
    const starkv_strides a = strides_of(s[i], n, P->cfg.n_kv_heads, P->cfg.head_dim);
    if (o[i] && !rows_apart(a, P->cfg.batch, n, P->cfg.n_kv_heads, P->cfg.head_dim))
      return fail_with(STARKV_ERR_INVALID_ARG, "rows of the output overlap");
    p.out[i] = o[i];
    p.wide[i] = rows_wide(o[i], a, elem, 4 * elem);
    p.os_b[i] = a.batch;
    p.os_t[i] = a.token;
    p.os_h[i] = a.head;
  }
  p.ctx_len = ctx_len_dev;
  p.start = start_dev;
  p.n = n;
  p.out_dtype = out_dtype;
  return hip_status(launch_dense_read(p, static_cast<void*>(stream)), "dense read launch");
}

// ----------------------------------------------------------------------------- attention

// Workgroups that an attention pass runs at a time.  The split kernel: one per compute unit, since a
// workgroup's start and end (queries, merge of its waves, partials) cost more than a second one in
// flight gains (with two: 32 ragged sequences of 8 KV heads 128 us against 121, 32 query rows 67
// against 61, 4 x 128K the same 164); two where a range holds more than a sequence, so that one's
// starts and ends run beside the other's stream (300 sequences of 200 to 600 tokens 124 us against
// 165, 64 of 1000 to 3000 67 against 69), up to the two row tiles that fit twice.  The chunk
// kernel: two.
static int64_t target_of(const starkv_dense_plan* P, int64_t rows) {
  if (rows > kSplitRows) return 512;
  return rows <= 32 && (int64_t)P->cfg.batch * P->cfg.n_kv_heads > 256 ? 512 : 256;
}

// Ranges of a pass over `rows` query rows per KV head.  Its workgroups (ranges x KV heads x row
// tiles) run target_of() at a time.  The ranges are as many as one round takes, or, where a few
// more make the last round fuller, up to four more (two, where one range fills a round: the
// partials are large there); each costs 2 % for its start and partials.  From two rounds on the
// row tiles are enough, and one range needs no partials.
static int64_t split_ranges(const starkv_dense_plan* P, int64_t rows) {
  const int64_t tiles = rows <= kSplitRows ? 1 : (rows + kChunkRows - 1) / kChunkRows;
  const int64_t per_range = P->cfg.n_kv_heads * tiles, target = target_of(P, rows);
  if (per_range >= 2 * target) return 1;
  const int64_t one = std::max<int64_t>(target / per_range, 1);
  const int64_t most = per_range >= target ? 3 : one + 4;
  int64_t best = one;
  double least = 1e30;
  for (int64_t r = one; r <= most; ++r) {
    const double rounds = (double)((r * per_range + target - 1) / target);
    const double cost = rounds / r * (1.0 + 0.02 * (r - one));
    if (cost < least) {
      least = cost;
      best = r;
    }
  }
  return best;
}

struct DenseWorkspace {
  int64_t ranges;
  int64_t part, ml, sub, total;       // offsets in bytes; the sequences' slots come first
  int32_t sub_per_head;
};
static DenseWorkspace workspace_of(const starkv_dense_plan* P, int32_t n_q, int32_t max_ctx,
                                   bool weights) {
  DenseWorkspace w;
  const starkv_dense_config& c = P->cfg;
  const int64_t rows = (int64_t)n_q * (c.n_q_heads / c.n_kv_heads);
  w.ranges = split_ranges(P, rows);
  // (the chunk kernel writes the output itself where one range holds all sequences)
  const bool whole = rows > kSplitRows && w.ranges == 1;
  const int64_t slots = whole ? 1 : (w.ranges + c.batch) * c.n_kv_heads * rows;
  w.part = align256((int64_t)c.batch * sizeof(Slots));
  w.ml = w.part + align256(slots * c.head_dim * 4);
  w.sub = w.ml + align256(slots * 8);
  w.sub_per_head = (max_ctx + 15) / 16;
  w.total = w.sub + (weights ? align256((int64_t)c.batch * c.n_kv_heads * w.sub_per_head * rows * 8) : 0);
  return w;
}

size_t starkv_dense_workspace_bytes(const starkv_dense_plan* P, int32_t n_q, int32_t max_ctx,
                                    int32_t with_weights) {
  if (!P || n_q < 1 || max_ctx < 1) return 0;
  // Fewer query tokens may take more ranges: the largest need lies at n_q or just before a step
  // of the rows that the rule goes by.
  const int G = P->cfg.n_q_heads / P->cfg.n_kv_heads;
  const int gather = with_weights ? std::min(n_q, std::max(kSplitRows / G, 1)) : 0;
  int64_t need = workspace_of(P, n_q, max_ctx, false).total;
  for (int64_t rows = 32; rows <= 2 * 512 * (int64_t)kChunkRows;
       rows += rows < kChunkRows ? rows : kChunkRows) {
    const int64_t n = rows / G;
    if (n >= n_q) break;
    if (n >= 1) {
      need = std::max(need, workspace_of(P, (int32_t)n, max_ctx, false).total);
      if (n < gather) need = std::max(need, workspace_of(P, (int32_t)n, max_ctx, true).total);
    }
  }
  if (gather) need = std::max(need, workspace_of(P, gather, max_ctx, true).total);
  return (size_t)need;
}

starkv_status starkv_dense_attn(const starkv_dense_plan* P, const void* cache, const void* q,
                                const starkv_strides* qs, int32_t n_q, const int32_t* q_len_dev,
                                const int32_t* ctx_len_dev, int32_t max_ctx, void* out,
                                const starkv_strides* os, float* weights, void* ws,
                                size_t ws_bytes, starkv_stream_t stream) {
  starkv_status st = check_cache(P, cache);
  if (st != STARKV_OK) return st;
  const starkv_dense_config& c = P->cfg;
  if (n_q < 1) return fail_with(STARKV_ERR_INVALID_ARG, "n_q %d < 1", n_q);
  if (max_ctx < 1) return fail_with(STARKV_ERR_INVALID_ARG, "max_ctx %d < 1", max_ctx);
  if (max_ctx > c.capacity)
    return fail_with(STARKV_ERR_CAPACITY, "max_ctx %d > capacity %d", max_ctx, c.capacity);
  if (!q || !ctx_len_dev || !out) return fail_with(STARKV_ERR_INVALID_ARG, "NULL device pointer");
  const int G = c.n_q_heads / c.n_kv_heads;
  if (n_q > kMaxDenseCtx) return fail_with(STARKV_ERR_UNSUPPORTED, "n_q %d > %d", n_q, kMaxDenseCtx);
  if (weights && (int64_t)n_q * G > kSplitRows)
    return fail_with(STARKV_ERR_UNSUPPORTED, "weights with %d query rows per KV head > %d", n_q * G, kSplitRows);
  if (misaligned(q, 2) || misaligned(out, 2)) return fail_with(STARKV_ERR_ALIGNMENT, "q or out not 2-byte aligned");
  if (misaligned(ctx_len_dev, 4) || misaligned(q_len_dev, 4) || misaligned(weights, 4))
    return fail_with(STARKV_ERR_ALIGNMENT, "lengths or weights not 4-byte aligned");
  const starkv_strides a = strides_of(qs, n_q, c.n_q_heads, c.head_dim);
  const starkv_strides o = strides_of(os, n_q, c.n_q_heads, c.head_dim);
  if (!rows_apart(o, c.batch, n_q, c.n_q_heads, c.head_dim))
    return fail_with(STARKV_ERR_INVALID_ARG, "rows of out overlap");
  const DenseWorkspace w = workspace_of(P, n_q, max_ctx, weights != nullptr);
  if (!ws || ws_bytes < (size_t)w.total)
    return fail_with(STARKV_ERR_WORKSPACE, "attention workspace %zu bytes < %lld", ws_bytes, (long long)w.total);
  if (misaligned(ws, 256)) return fail_with(STARKV_ERR_ALIGNMENT, "ws not 256-byte aligned");
  DenseAttnParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = cache_of(P, cache);
  p.q = static_cast<const uint16_t*>(q);
  p.out = static_cast<uint16_t*>(out);
  p.qs_b = a.batch;
  p.qs_t = a.token;
  p.qs_h = a.head;
  p.os_b = o.batch;
  p.os_t = o.token;
  p.os_h = o.head;
  p.q_len = q_len_dev;
  p.ctx_len = ctx_len_dev;
  p.weights = weights;
  uint8_t* base = static_cast<uint8_t*>(ws);
  p.slots = reinterpret_cast<Slots*>(base);
  p.part_o = reinterpret_cast<float*>(base + w.part);
  p.part_ml = reinterpret_cast<Pair*>(base + w.ml);
  p.sub = reinterpret_cast<Pair*>(base + w.sub);
  p.n_q = n_q;
  p.group = G;
  p.rows = n_q * G;
  p.max_ctx = max_ctx;
  p.ranges = (int32_t)w.ranges;
  // (a chunk workgroup's start and end cost more than a tile: 100 queries over 2000 tokens 32 us
  // against 38 with one unit; not where there are fewer units than ranges)
  p.min_units = p.rows > kSplitRows ? 2 : 1;
  p.sub_per_head = w.sub_per_head;
  p.q_wide = rows_wide(q, a, 2);
  p.out_wide = rows_wide(out, o, 2, 8);
  p.scale_log2 = (float)(P->scale * 1.4426950408889634);
  return hip_status(launch_dense_attn(p, static_cast<void*>(stream)), "dense attention launch");
}

// ------------------------------------------------------------------------------- eviction

starkv_status starkv_dense_evict(const starkv_dense_plan* P, float* weights,
                                 int32_t* ctx_len_dev, int32_t keep, int32_t sink,
                                 int32_t recent, int32_t* table_out, float* weights_out,
                                 int32_t* ctx_out, starkv_stream_t stream) {
  if (!P) return fail_with(STARKV_ERR_INVALID_ARG, "plan is NULL");
  if (!weights || !ctx_len_dev) return fail_with(STARKV_ERR_INVALID_ARG, "NULL device pointer");
  if (keep < 1 || sink < 0 || recent < 0 || (int64_t)sink + recent > keep)
    return fail_with(STARKV_ERR_INVALID_ARG, "keep %d, sink %d, recent %d: need sink + recent <= keep, keep >= 1",
                     keep, sink, recent);
  if (misaligned(weights, 4) || misaligned(ctx_len_dev, 4) || misaligned(table_out, 4) ||
      misaligned(weights_out, 4) || misaligned(ctx_out, 4))
    return fail_with(STARKV_ERR_ALIGNMENT, "pointer not 4-byte aligned");
  DenseEvictParams p;
  std::memset(&p, 0, sizeof(p));
  p.table = P->cfg.block_table;
  p.table_out = table_out ? table_out : P->cfg.block_table;
  p.weights = weights;
  p.weights_out = weights_out ? weights_out : weights;
  p.ctx_len = ctx_len_dev;
  p.ctx_out = ctx_out ? ctx_out : ctx_len_dev;
  p.batch = P->cfg.batch;
  p.n_kv = P->cfg.n_kv_heads;
  p.shift = P->shift;
  p.blocks_per_head = P->layout.blocks_per_head;
  p.capacity = P->cfg.capacity;
  p.keep = keep;
  p.sink = sink;
  p.recent = recent;
  return hip_status(launch_dense_evict(p, static_cast<void*>(stream)), "dense evict launch");
}

}  // extern "C"
