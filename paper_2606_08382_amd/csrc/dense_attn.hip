// Attention over the 8-bit cache of an uncompressed layer (starkv_dense_attn).
//
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - reference)
// in one pass over the cache with a running reference and sum.  A decode step reads 2 d bytes of
// codes per token and KV head and does 4 d flops per query row on them: HBM bounds it.  So the
// split kernel is built as a read stream: a wave owns 32-token steps, keeps the next steps' codes in
// flight in registers, and shares nothing with other waves until its range is done.
//
// Matrix products, per wave and step (v_mfma_f32_16x16x32):
//   S^T = K q^T   rows: 16 tokens, columns: 16 query rows; operand K from the key codes
//   O^T += V^T p^T  rows: 16 channels, columns: 16 query rows, depth: 32 tokens
// A lane's four scores of a 16-token subtile are exactly the depth positions that it must supply
// of p^T for the second product (the order along the depth is free as long as V follows it), so
// probabilities never leave the lane.  The cache's byte order (see the header) makes every
// operand a contiguous 16-byte load per lane and 1 KiB per wave.
//
// Codes become fp16 exactly (|code| <= 448); the block's key scale multiplies the fp32 score and
// its value scale the probability.  Queries are fp16 after a power-of-two scale per row.
// Probabilities are rounded to fp16: 2^-12 relative, below an fp16 output's own rounding.  They
// stand relative to a reference 6 (log2) below the largest score so far, which is raised once a
// score passes it by 14: between 2^-24 and 2^14, so what fp16 drops is below 2^-30 of the largest.
// Value scales are relative to the largest of the wave, which keeps products in fp16's range.
#include <hip/hip_runtime.h>

#include "dense.h"

namespace starkv {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

constexpr int kWavesA = 4;
constexpr int kUnit = 32 * kWavesA;         // tokens of a workgroup's round: granule of ranges
constexpr float kBelow = 6.0f;              // reference: largest score - kBelow (log2)
constexpr float kAbove = 14.0f;             // scores may pass the reference by this much
constexpr float kTinyScale = 0x1p-100f;     // smallest reference of the value scales

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Reductions over the four lanes of a column (lanes 16 and 32 apart), in all of them: a register
// swapped with a copy of itself holds the even and the odd rows, or halves, of the wave.
__device__ __forceinline__ void swap16(float v, float* a, float* b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  *a = __uint_as_float(r[0]);
  *b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap32(float v, float* a, float* b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  *a = __uint_as_float(r[0]);
  *b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float quad_max(float v) {
  float a, b;
  swap16(v, &a, &b);
  swap32(fmaxf(a, b), &a, &b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float quad_sum(float v) {
  float a, b;
  swap16(v, &a, &b);
  swap32(a + b, &a, &b);
  return a + b;
}

// Four codes of a dword as fp16.
template <bool E4M3>
__device__ __forceinline__ void code4(uint32_t w, h2* out) {
  if constexpr (E4M3) {
    out[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    out[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  } else {
    // 0x64xx is 1024 + xx in fp16
    const h2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    out[0] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x05010400u)) - bias;
    out[1] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x05030402u)) - bias;
  }
}

template <bool E4M3>
__device__ __forceinline__ h8 code8(uint32_t lo, uint32_t hi) {
  union { h2 p[4]; h8 v; } u;
  code4<E4M3>(lo, u.p);
  code4<E4M3>(hi, u.p + 2);
  return u.v;
}

__device__ __forceinline__ f4 mfma_f16(h8 a, h8 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 mfma_bf16(b8 a, b8 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float from16(uint32_t u, int bf16) {
  return bf16 ? __uint_as_float(u << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)u);
}

// ---- work plan ----------------------------------------------------------------------
// The sequences' tokens, in units of kUnit, lie end to end; range w of p.ranges takes the units
// [w R, (w + 1) R), R = ceil(all units / ranges), and with them the end of one sequence and the
// start of the next: ranges are equal however ragged the lengths are.  The part of sequence b in
// range w is slot w + b of the partials (one of the two grows from part to part), at most
// ranges + B of them.  Every wave derives this from the lengths, so nothing is planned on the
// host and a captured call serves any lengths.
__device__ __forceinline__ int clamp_ctx(const DenseAttnParams& p, int b) {
  return min(max(p.ctx_len[b], 0), p.max_ctx);
}
__device__ __forceinline__ int units_of(int ctx) { return (ctx + kUnit - 1) / kUnit; }

// Inclusive sum over the wave's lanes (row shifts, then the rows' ends broadcast).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);    // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return v;
}

// Lane l: length of sequence l of the first 64 and the units up to its end.
struct Lens {
  int ctx, incl;
};
__device__ __forceinline__ Lens first_lens(const DenseAttnParams& p, int lane) {
  const int ctx = lane < p.c.batch ? clamp_ctx(p, lane) : 0;
  return {ctx, wave_scan(units_of(ctx))};
}

// Units of a range (all of them: < 2^31, with B <= 32767 and 4096 units each at most).
__device__ __forceinline__ int range_units(const DenseAttnParams& p, const Lens& ls, int lane) {
  int sum = __builtin_amdgcn_readlane(ls.incl, 63);
  for (int b0 = 64; b0 < p.c.batch; b0 += 64) {
    const int b = b0 + lane;
    sum += __builtin_amdgcn_readlane(wave_scan(b < p.c.batch ? units_of(clamp_ctx(p, b)) : 0), 63);
  }
  return max((int)(((uint32_t)sum + (uint32_t)p.ranges - 1) / (uint32_t)p.ranges), 1);
}

// The sequence that holds unit `at`, its length and its first unit; false past the last.
struct Place {
  int b, ctx, start;
};
__device__ __forceinline__ bool find_unit(const DenseAttnParams& p, const Lens& ls, int at, int lane,
                                          Place* pl) {
  Lens x = ls;
  for (int b0 = 0;;) {
    const uint64_t hit = __ballot(x.incl > at);
    if (hit) {
      const int l = (int)__builtin_ctzll(hit);
      pl->b = b0 + l;
      pl->ctx = __builtin_amdgcn_readlane(x.ctx, l);
      pl->start = __builtin_amdgcn_readlane(x.incl, l) - units_of(pl->ctx);
      return true;
    }
    b0 += 64;
    if (b0 >= p.c.batch) return false;
    const int b = b0 + lane, before = __builtin_amdgcn_readlane(x.incl, 63);
    x.ctx = b < p.c.batch ? clamp_ctx(p, b) : 0;
    x.incl = before + wave_scan(units_of(x.ctx));
  }
}
// First slot and number of slots of sequence b, and its length.
__device__ __forceinline__ void slots_of(const DenseAttnParams& p, int b, int lane, int* first,
                                         int* count, int* ctx) {
  const Lens ls = first_lens(p, lane);
  const uint32_t R = range_units(p, ls, lane);
  Lens x = ls;
  int before = 0;
  for (int b0 = 64; b0 <= b; b0 += 64) {
    before += __builtin_amdgcn_readlane(x.incl, 63);
    x.ctx = b0 + lane < p.c.batch ? clamp_ctx(p, b0 + lane) : 0;
    x.incl = wave_scan(units_of(x.ctx));
  }
  *ctx = __builtin_amdgcn_readlane(x.ctx, b & 63);
  const uint32_t u = units_of(*ctx);
  const uint32_t start = before + __builtin_amdgcn_readlane(x.incl, b & 63) - u;
  *first = start / R + b;
  *count = u > 0 ? (start + u - 1) / R - start / R + 1 : 0;
}

// Tokens that query row r (query token r / group) of sequence b sees: at most ctx; 0: none;
// -1: a row past the sequence's query tokens.
__device__ __forceinline__ int row_limit(const DenseAttnParams& p, int b, int ctx, int r) {
  const int q_len = p.q_len ? min(max(p.q_len[b], 0), p.n_q) : p.n_q;
  const int j = r / p.group;
  if (r >= p.rows || j >= q_len) return -1;
  return max(ctx - q_len + j + 1, 0);
}

__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// ---- split --------------------------------------------------------------------------

template <int D>
struct Tile {                       // codes of a 32-token step: two subtiles
  static constexpr int N = D / 64;
  u4 k[2][N], v[2][N];
  float sk[2], sv[2];
};

// State of RT tiles of 16 query rows.
template <int D, int RT>
struct State {
  f4 o[RT][D / 16];
  float m[RT], l[RT];               // reference (log2) of a lane's column; its lane's sum
  float vref, vinv;                 // reference of the value scales and its inverse
};

// Raises references so that scores up to `top` and value scales up to sv fit.
template <int D, int RT>
__device__ __forceinline__ void raise(State<D, RT>& s, const float* top, float sv) {
  float vr = 1.0f;
  if (sv > s.vref) {
    vr = s.vref / sv;
    s.vref = sv;
    s.vinv = 1.0f / sv;
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float t = quad_max(top[r]);
    const float m = t > s.m[r] + kAbove ? t - kBelow : s.m[r];
    const float a = m == s.m[r] ? 1.0f : exp2_fast(s.m[r] - m);
    s.m[r] = m;
    s.l[r] *= a;
    const float f = a * vr;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) s.o[r][c] *= f;
  }
}

template <int D, bool E4M3, int RT, bool SUMS>
__global__ __launch_bounds__(256, RT == 1 ? 2 : 1) void dense_split_kernel(const DenseAttnParams p) {
  constexpr int N = D / 64, CT = D / 16, NB = RT == 1 ? 3 : 2;
  const int tid_lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.y, row0 = blockIdx.z * (16 * RT);
  const Lens lens = first_lens(p, tid_lane);
  const int R = range_units(p, lens, tid_lane);
  __shared__ float so[kWavesA][16][D + 4];
  __shared__ float sm[kWavesA][RT * 16], sl[kWavesA][RT * 16];
  const int sh = p.c.shift, T = 1 << sh;
  Place pl;
  int at = blockIdx.x * R;
  const int at_end = at + R;
  if (!find_unit(p, lens, at, tid_lane, &pl)) return;
  for (;;) {                                       // the range's part of one sequence after another
  // (a lane index that the compiler takes for new: addresses and masks are formed where they are
  // used instead of being kept in registers over the whole range)
  int lane = fresh(tid_lane);
  int col = lane & 15, quad = lane >> 4;
  struct { int b, ctx, t0, t1; } it;
  it.b = pl.b;
  it.ctx = pl.ctx;
  it.t0 = (at - pl.start) * kUnit;
  it.t1 = min(min(at_end - pl.start, units_of(pl.ctx)) * kUnit, pl.ctx);
  const int full = it.ctx & ~(T - 1);
  const int64_t head = (int64_t)it.b * p.c.n_kv + g;
  const int e8 = min(it.t1, full), tw = it.t0 + 32 * wave;   // the wave's finished blocks

  // The chains of loads that a part begins with overlap: the table entries of the first 64 steps
  // (a subtile per lane and 32 steps), the queries, then the entries' scales and codes.
  const int32_t* table = p.c.table + head * p.c.blocks_per_head;
  auto entry_token = [&](int i0) {
    return max(min(tw + (i0 + (lane >> 1)) * kUnit + (lane & 1) * 16, e8 - 16), 0);
  };
  const int entry0 = table[entry_token(0) >> sh], entry1 = table[entry_token(32) >> sh];

  // queries: row r of the tile in column `col`, channels i*64 + quad*16 + h*8 + e
  h8 q[RT][2 * N];
  float qs[RT];
  int lim[RT];
  int lim_lo = 0x7fffffff, lim_hi = 0;
  union Raw { u4 v; uint16_t h[8]; };
  Raw raw[RT][2 * N];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row0 + r * 16 + col;
    const int lm = row_limit(p, it.b, it.ctx, row);
    lim[r] = lm < 0 ? 0x7fffffff : lm;             // rows without a query see everything
    lim_lo = min(lim_lo, lim[r]);
    lim_hi = max(lim_hi, lm);
    const int jq = row / p.group, iq = row % p.group;
    const uint16_t* src = p.q + it.b * p.qs_b + jq * p.qs_t + (g * p.group + iq) * p.qs_h;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) {
      const int ch = (i >> 1) * 64 + quad * 16 + (i & 1) * 8;
      raw[r][i].v = (u4){0, 0, 0, 0};
      if (lm >= 0) {
        if (p.q_wide) {
          raw[r][i].v = *reinterpret_cast<const u4*>(src + ch);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) raw[r][i].h[e] = src[ch + e];
        }
      }
    }
  }
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) {
    lim_lo = min(lim_lo, __shfl_xor(lim_lo, o));
    lim_hi = max(lim_hi, __shfl_xor(lim_hi, o));
  }
  lim_lo = __builtin_amdgcn_readfirstlane(lim_lo);
  lim_hi = __builtin_amdgcn_readfirstlane(lim_hi);

  // row tiles of early query tokens end before the sequence does; a part's sums are written for
  // all of its subtiles
  const int stop = SUMS ? e8 : min(e8, (lim_hi + 15) & ~15);
  const int steps = stop > tw ? (stop - tw + kUnit - 1) / kUnit : 0;
  struct Entry { uint32_t sub; float sk, sv; };
  auto entry_of = [&](int e, int i0) {
    const int t = entry_token(i0);
    e = min(max(e, 0), p.c.n_blocks - 1);
    const Pair sc = p.c.scales[e];
    return Entry{((uint32_t)e << (sh - 3)) + ((uint32_t)(t & (T - 1)) >> 4), sc.x, sc.y};
  };
  const uint32_t v_sub = (uint32_t)T >> 4;          // from a key subtile to its value subtile
  auto load = [&](Tile<D>& x, const Entry& en, int i) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const int l = 2 * (i & 31) + a;
      const uint32_t sub = __builtin_amdgcn_readlane(en.sub, l);
      x.sk[a] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(en.sk), l));
      x.sv[a] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(en.sv), l));
      const uint8_t* kb = p.c.codes + (uint64_t)sub * (16 * D) + lane * 16;
      const uint8_t* vb = p.c.codes + (uint64_t)(sub + v_sub) * (16 * D) + lane * 16;
      // (streaming: a code is read once a step; 5.8 TB/s with plain loads, 6.7 with these)
#pragma unroll
      for (int n = 0; n < N; ++n)
        x.k[a][n] = __builtin_nontemporal_load(reinterpret_cast<const u4*>(kb + n * 1024));
#pragma unroll
      for (int n = 0; n < N; ++n)
        x.v[a][n] = __builtin_nontemporal_load(reinterpret_cast<const u4*>(vb + n * 1024));
    }
  };
  // A step's codes are loaded NB - 1 steps ahead, past the last one the last again; the entries of
  // the next 32 steps while these 32 run.
  Entry now, next;
  Tile<D> x[NB];
  auto fetch = [&](Tile<D>& y, int i) {
    if (i > 0 && (i & 31) == 0) {
      now = next;
      next = entry_of(table[entry_token(i + 32) >> sh], i + 32);
    }
    load(y, now, min(i, steps - 1));
  };
  if (steps > 0) {
    now = entry_of(entry0, 0);
    next = entry_of(entry1, 32);
#pragma unroll
    for (int u = 0; u < NB - 1; ++u) fetch(x[u], u);
  }

  // queries as fp16, scaled by a power of two per row
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(from16(raw[r][i].h[e], p.c.bf16)));
    top = quad_max(top);
    const int ex = top > 0.0f && top < __builtin_inff() ? 8 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
    for (int i = 0; i < 2 * N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        q[r][i][e] = (_Float16)__builtin_amdgcn_ldexpf(from16(raw[r][i].h[e], p.c.bf16), ex);
    qs[r] = __builtin_amdgcn_ldexpf(p.scale_log2, -ex);
  }

  State<D, RT> s;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    s.m[r] = -__builtin_inff();
    s.l[r] = 0.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c) s.o[r][c] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  s.vref = kTinyScale;
  s.vinv = 1.0f / kTinyScale;

  // Softmax of a step's scores and its product with the values.  x: log2 scores; t: first token;
  // sv: value scales of the two subtiles; pv(r, pr): the product.  Scores of tokens from lim
  // on, and from `end` on, count as absent.
  auto softmax = [&](f4 (&x)[RT][2], int t, int end, const float* sv, float (&pr)[RT][8], bool odd) {
    if (t + 32 > lim_lo || t + 32 > end) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = t + a * 16 + quad * 4 + e;
            x[r][a][e] = tok < lim[r] && tok < end ? x[r][a][e] : -__builtin_inff();
          }
    }
    float top[RT];
    bool over = fmaxf(sv[0], sv[1]) > s.vref;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      top[r] = fmaxf(fmaxf(fmaxf(x[r][0][0], x[r][0][1]), fmaxf(x[r][0][2], x[r][0][3])),
                     fmaxf(fmaxf(x[r][1][0], x[r][1][1]), fmaxf(x[r][1][2], x[r][1][3])));
      over |= top[r] > s.m[r] + kAbove;
    }
    if (__any(over)) raise(s, top, fmaxf(sv[0], sv[1]));
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      // a column that has seen nothing keeps reference -inf: x - 0 is -inf, its exponential 0
      const float m = s.m[r] == -__builtin_inff() ? 0.0f : s.m[r];
      float part[2];
#pragma unroll
      for (int a = 0; a < 2; ++a) {
#pragma unroll
        for (int e = 0; e < 4; ++e) pr[r][a * 4 + e] = exp2_fast(x[r][a][e] - m);
        part[a] = (pr[r][a * 4] + pr[r][a * 4 + 1]) + (pr[r][a * 4 + 2] + pr[r][a * 4 + 3]);
        s.l[r] += part[a];
        if constexpr (SUMS) {
          const float y = quad_sum(part[a]);
          const int row = r * 16 + col;
          if (quad == 0 && row < p.rows && (a == 0 || odd))
            p.sub[(head * p.sub_per_head + (t >> 4) + a) * p.rows + row] = {y, s.m[r]};
        }
      }
    }
  };

  // ---- finished blocks
  auto compute = [&](const Tile<D>& y, int i) {
    const int t = tw + i * kUnit;
    f4 sc[RT][2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r][a] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const h8 k = code8<E4M3>(y.k[a][n][2 * h], y.k[a][n][2 * h + 1]);
#pragma unroll
          for (int r = 0; r < RT; ++r) sc[r][a] = mfma_f16(k, q[r][2 * n + h], sc[r][a]);
        }
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r][a] *= y.sk[a] * qs[r];
    }
    float pr[RT][8];
    softmax(sc, t, e8, y.sv, pr, t + 16 < e8);
    h8 ph[RT];
    const float f0 = y.sv[0] * s.vinv, f1 = y.sv[1] * s.vinv;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) ph[r][e] = (_Float16)(pr[r][e] * (e < 4 ? f0 : f1));
    if (t + 32 > lim_lo || t + 32 > e8) {
      // an absent token's probability is zero whatever its block's scale
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) ph[r][e] = pr[r][e] == 0.0f ? (_Float16)0.0f : ph[r][e];
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const h8 v = code8<E4M3>(y.v[0][n][j], y.v[1][n][j]);
#pragma unroll
        for (int r = 0; r < RT; ++r) s.o[r][n * 4 + j] = mfma_f16(v, ph[r], s.o[r][n * 4 + j]);
      }
  };
  if (steps > 0) {
    for (int i = 0; i < steps; i += NB) {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        fetch(x[(u + NB - 1) % NB], i + u + NB - 1);
        if (i + u < steps) compute(x[u], i + u);
      }
    }
  }

  // ---- the unfinished block, from its 16-bit rows
  if (full < it.t1 && (SUMS || lim_hi > full)) {
    lane = fresh(tid_lane);
    col = lane & 15;
    quad = lane >> 4;
    const uint16_t* kt = p.c.tails + head * 2 * (2 * T * D);
    const uint16_t* vt = kt + 2 * T * D;
    for (int t = full + 32 * wave; t < it.ctx; t += kUnit) {
      f4 sc[RT][2];
      const int bf16 = p.c.bf16;
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r][0] = sc[r][1] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < 2 * N; ++n) {
        const int ch = n * 32 + quad * 8;
        u4 k[2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int tok = t + a * 16 + col;
          k[a] = tok < it.ctx ? *reinterpret_cast<const u4*>(kt + (tok & (2 * T - 1)) * D + ch)
                              : (u4){0, 0, 0, 0};
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          // the query row as it was given
          const int row = row0 + r * 16 + col, jq = row / p.group, iq = row % p.group;
          const uint16_t* src = p.q + it.b * p.qs_b + jq * p.qs_t + (g * p.group + iq) * p.qs_h + ch;
          union { u4 v; uint16_t h[8]; } w;
          w.v = (u4){0, 0, 0, 0};
          if (lim[r] != 0x7fffffff) {
            if (p.q_wide) {
              w.v = *reinterpret_cast<const u4*>(src);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) w.h[e] = src[e];
            }
          }
#pragma unroll
          for (int a = 0; a < 2; ++a)
            sc[r][a] = bf16 ? mfma_bf16(__builtin_bit_cast(b8, k[a]), __builtin_bit_cast(b8, w.v), sc[r][a])
                            : mfma_f16(__builtin_bit_cast(h8, k[a]), __builtin_bit_cast(h8, w.v), sc[r][a]);
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        sc[r][0] *= p.scale_log2;
        sc[r][1] *= p.scale_log2;
      }
      const float one[2] = {1.0f, 1.0f};
      float pr[RT][8];
      softmax(sc, t, it.ctx, one, pr, t + 16 < it.ctx);
      h8 ph[RT];
      b8 pb[RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = pr[r][e] * s.vinv;
          ph[r][e] = (_Float16)v;
          pb[r][0][e] = (__bf16)v;
          pb[r][1][e] = (__bf16)(v - (float)pb[r][0][e]);
        }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        u2 w[2];
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          // tokens t + 16a + 4 quad .. + 3 of channel 16c + col; absent ones cleared
          const int tok = t + a * 16 + quad * 4, rr = tok & (2 * T - 1);
          w[a] = (u2){0, 0};
          if (tok < it.ctx) {
            w[a] = *reinterpret_cast<const u2*>(vt + ((rr >> 4) * D + c * 16 + col) * 16 + quad * 4);
            const int left = it.ctx - tok;
            if (left < 2) w[a].x &= 0xffffu;
            if (left < 3) w[a].y = 0;
            else if (left < 4) w[a].y &= 0xffffu;
          }
        }
        const u4 v = {w[0].x, w[0].y, w[1].x, w[1].y};
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if (bf16) {
            s.o[r][c] = mfma_bf16(__builtin_bit_cast(b8, v), pb[r][0], s.o[r][c]);
            s.o[r][c] = mfma_bf16(__builtin_bit_cast(b8, v), pb[r][1], s.o[r][c]);
          } else {
            s.o[r][c] = mfma_f16(__builtin_bit_cast(h8, v), ph[r], s.o[r][c]);
          }
        }
      }
    }
  }

  lane = fresh(tid_lane);
  col = lane & 15;
  quad = lane >> 4;
  // ---- the waves' states merged, normalized and written as the part's partial
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = quad_sum(s.l[r]);
    if (quad == 0) {
      sm[wave][r * 16 + col] = s.m[r];
      sl[wave][r * 16 + col] = l;
    }
  }
  __syncthreads();
  const int64_t slot0 = ((int64_t)(blockIdx.x + it.b) * p.c.n_kv + g) * p.rows + row0;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    float M = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < kWavesA; ++w) M = fmaxf(M, sm[w][r * 16 + col]);
    float L = 0.0f, own = 0.0f;
#pragma unroll
    for (int w = 0; w < kWavesA; ++w) {
      const float mw = sm[w][r * 16 + col], lw = sl[w][r * 16 + col];
      const float a = mw == M ? 1.0f : exp2_fast(mw - M);
      // a wave without tokens: sum 0 (NaN stays)
      L += lw * a;
      if (w == wave) own = a;
    }
    const float f = L == 0.0f ? 0.0f : own / L;
    if (wave == 0 && quad == 0 && row0 + r * 16 + col < p.rows)
      p.part_ml[slot0 + r * 16 + col] = {M, L};
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      f4 v = s.o[r][c] * f;                         // at most fp16's largest code, then the scale
      v *= s.vref;
      *reinterpret_cast<f4*>(&so[wave][col][c * 16 + quad * 4]) = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * D / 4; i += 256) {
      const int row = i / (D / 4), ch = i % (D / 4) * 4;
      if (row0 + r * 16 + row < p.rows) {
        f4 v = *reinterpret_cast<const f4*>(&so[0][row][ch]);
#pragma unroll
        for (int w = 1; w < kWavesA; ++w) v += *reinterpret_cast<const f4*>(&so[w][row][ch]);
        *reinterpret_cast<f4*>(p.part_o + (slot0 + r * 16 + row) * D + ch) = v;
      }
    }
    __syncthreads();
  }
  at = pl.start + units_of(pl.ctx);
  if (at >= at_end || !find_unit(p, lens, at, tid_lane, &pl)) return;
  }
}

// ---- combine ------------------------------------------------------------------------
// The row's parts weighted by their softmax sums: lane i holds part i's reference and sum (64 parts
// at a time), merged over the wave; every wave of a workgroup does this for itself.
struct Merged {
  float m, l;                       // largest reference, sum relative to it
};
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
  return quad_max(v);
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o);
  return quad_sum(v);
}
__device__ __forceinline__ Merged merge_row(const DenseAttnParams& p, int first, int count, int g,
                                            int row, int lane) {
  float m = -__builtin_inff(), l = 0.0f;
  for (int i = lane; i < count; i += 64) {
    const Pair ml = p.part_ml[((int64_t)(first + i) * p.c.n_kv + g) * p.rows + row];
    const float mn = fmaxf(m, ml.x);
    l = (m == mn ? l : l * exp2_fast(m - mn)) + (ml.x == mn ? ml.y : ml.y * exp2_fast(ml.x - mn));
    m = mn;
  }
  const float M = wave_max(m);
  return {M, wave_sum(m == M ? l : l * exp2_fast(m - M))};
}

// w_j += sum over rows and over block j's subtiles of sum * 2^(reference - M_row) / L_row, for
// 256 blocks of a KV head.
__device__ __forceinline__ void gather_weights(const DenseAttnParams& p, int tile, int g, int b,
                                               float* sM, float* sI) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int first, count, ctx;
  slots_of(p, b, lane, &first, &count, &ctx);
  const int64_t head = (int64_t)b * p.c.n_kv + g;
  const int sub_shift = p.c.shift - 4, subs = (ctx + 15) >> 4;
  if (tile * (256 << sub_shift) >= subs) return;
  for (int row = wave; row < p.rows; row += 4) {
    Merged t = {0.0f, 0.0f};
    if (row_limit(p, b, ctx, row) > 0) t = merge_row(p, first, count, g, row, lane);
    if (lane == 0) {
      sM[row] = t.m;
      sI[row] = t.l == 0.0f ? 0.0f : 1.0f / t.l;
    }
  }
  __syncthreads();
  const int j = tile * 256 + threadIdx.x, s0 = j << sub_shift;
  if (s0 >= subs) return;
  const int n = (min(s0 + (1 << sub_shift), subs) - s0) * p.rows;
  const Pair* y = p.sub + (head * p.sub_per_head + s0) * p.rows;
  float w = 0.0f;
  int row = 0;
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    const Pair v = y[i];
    // (a row without tokens or without a query has weight 0 whatever its reference)
    w += v.x == 0.0f || sI[row] == 0.0f ? 0.0f : v.x * exp2_fast(v.y - sM[row]) * sI[row];
    row = row + 1 == p.rows ? 0 : row + 1;
  }
  p.weights[head * p.c.blocks_per_head + j] += w;
}

// A workgroup per (row, KV head, sequence); its four waves take every fourth part.  Workgroups
// past the rows gather the weights.
template <int D>
__global__ __launch_bounds__(256) void dense_combine_kernel(const DenseAttnParams p) {
  constexpr int C = D / 64;
  __shared__ float so[4][D], sM[64], sI[64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  if (row >= p.rows) {
    gather_weights(p, row - p.rows, g, b, sM, sI);
    return;
  }
  int first, count, ctx;
  slots_of(p, b, lane, &first, &count, &ctx);
  if (row_limit(p, b, ctx, row) < 0) return;
  const Merged t = merge_row(p, first, count, g, row, lane);
  float o[C] = {};
#pragma unroll 4
  for (int i = wave; i < count; i += 4) {
    const int64_t slot = ((int64_t)(first + i) * p.c.n_kv + g) * p.rows + row;
    const Pair ml = p.part_ml[slot];
    const float f = ml.x == t.m ? ml.y : ml.y * exp2_fast(ml.x - t.m);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float v = p.part_o[slot * D + c * 64 + lane];
      o[c] += f == 0.0f ? 0.0f : f * v;
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) so[wave][c * 64 + lane] = o[c];
  __syncthreads();
  if (threadIdx.x < D) {
    const int i = threadIdx.x;
    float v = (so[0][i] + so[1][i]) + (so[2][i] + so[3][i]);
    v = t.l == 0.0f ? 0.0f : v / t.l;
    const int jq = row / p.group, iq = row % p.group;
    uint16_t* out = p.out + b * p.os_b + jq * p.os_t + (g * p.group + iq) * p.os_h;
    out[i] = p.c.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v)
                      : __builtin_bit_cast(uint16_t, (_Float16)v);
  }
}

template <int D, bool E4M3, int RT>
void launch_split(const DenseAttnParams& p, hipStream_t st) {
  const dim3 grid(p.ranges, p.c.n_kv, (p.rows + 16 * RT - 1) / (16 * RT));
  if (p.weights) hipLaunchKernelGGL((dense_split_kernel<D, E4M3, RT, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((dense_split_kernel<D, E4M3, RT, false>), grid, dim3(256), 0, st, p);
}

template <int D, bool E4M3>
void launch_rows(const DenseAttnParams& p, hipStream_t st) {
  if (p.rows <= 16) launch_split<D, E4M3, 1>(p, st);
  else if (p.rows <= 32) launch_split<D, E4M3, 2>(p, st);
  else launch_split<D, E4M3, 4>(p, st);
}

}  // namespace

int launch_dense_attn(const DenseAttnParams& p, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p.c.d == 128) {
    if (p.c.e4m3) launch_rows<128, true>(p, st);
    else launch_rows<128, false>(p, st);
  } else {
    if (p.c.e4m3) launch_rows<64, true>(p, st);
    else launch_rows<64, false>(p, st);
  }
  int e = (int)hipGetLastError();
  if (e) return e;
  const int J = (p.max_ctx + (1 << p.c.shift) - 1) >> p.c.shift;
  const dim3 grid(p.rows + (p.weights ? (J + 255) / 256 : 0), p.c.n_kv, p.c.batch);
  if (p.c.d == 128) hipLaunchKernelGGL(dense_combine_kernel<128>, grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(dense_combine_kernel<64>, grid, dim3(256), 0, st, p);
  return (int)hipGetLastError();
}

}  // namespace starkv
