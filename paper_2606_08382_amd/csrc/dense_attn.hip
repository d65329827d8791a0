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
constexpr float kTinyScale = -100.0f;       // smallest reference of the value scales (log2)

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

__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
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
// [w R, (w + 1) R), R = ceil(all units / ranges) (at least p.min_units where that leaves none idle),
// and with them the end of one sequence and the
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
  const int R = max((int)(((uint32_t)sum + (uint32_t)p.ranges - 1) / (uint32_t)p.ranges), 1);
  return sum >= p.ranges ? max(R, p.min_units) : R;
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
// Leaves every sequence's first slot, number of slots and length for the combine pass, which would
// otherwise walk over the batch once per row.  By one wave of the first workgroup.
__device__ __forceinline__ void write_slots(const DenseAttnParams& p, const Lens& ls, int R, int lane) {
  Lens x = ls;
  uint32_t before = 0;
  for (int b0 = 0; b0 < p.c.batch; b0 += 64) {
    const int b = b0 + lane;
    if (b0) {
      x.ctx = b < p.c.batch ? clamp_ctx(p, b) : 0;
      x.incl = wave_scan(units_of(x.ctx));
    }
    const uint32_t u = units_of(x.ctx), start = before + x.incl - u, r = R;
    if (b < p.c.batch)
      p.slots[b] = {(int)(start / r) + b, u ? (int)((start + u - 1) / r - start / r) + 1 : 0, x.ctx, 0};
    before += __builtin_amdgcn_readlane(x.incl, 63);
  }
}

// Tokens that query row r (query token r / group) of sequence b sees: at most ctx; 0: none;
// -1: a row past the sequence's query tokens.
__device__ __forceinline__ int row_limit(const DenseAttnParams& p, int b, int ctx, int r) {
  const int q_len = p.q_len ? min(max(p.q_len[b], 0), p.n_q) : p.n_q;
  const int j = r / p.group;
  if (r >= p.rows || j >= q_len) return -1;
  return max(ctx - q_len + j + 1, 0);
}

// ---- split --------------------------------------------------------------------------

template <int D>
struct Tile {                       // codes of a 32-token step: two subtiles
  static constexpr int N = D / 64;
  u4 k[2][N], v[2][N];
  float sk[2], lsv[2];
};

// State of RT tiles of 16 query rows.
template <int D, int RT>
struct State {
  f4 o[RT][D / 16];
  float m[RT], l[RT];               // reference (log2) of a lane's column; its lane's sum
  float lv;                         // reference of the value scales (log2)
};

// Raises references so that scores up to `top` and (log2) value scales up to lsv fit.
template <int D, int RT>
__device__ __forceinline__ void raise(State<D, RT>& s, const float* top, float lsv) {
  const float lv = fmaxf(s.lv, lsv), vr = exp2_fast(s.lv - lv);
  s.lv = lv;
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

template <int D, int RT>
__device__ __forceinline__ void reset(State<D, RT>& s) {
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    s.m[r] = -__builtin_inff();
    s.l[r] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) s.o[r][c] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  s.lv = kTinyScale;
}

// Where a split pass with weights leaves the sums of 16-token subtiles.
struct SubSums {
  Pair* at;                         // of the KV head's first subtile, row 0
  int row0, rows;                   // the wave's first row; rows of the KV head
};

// Softmax of ST 32-token steps of tokens t.., in two parts.  sc: products q.k; fk: what makes them
// log2 scores; lsv: log2 of the value scales of the subtiles.  Tokens from lim[] on, and from
// `end` on, are absent.  A lane's tokens are t + 32 st + 16 a + 4 quad + e, a = 0, 1, e = 0..3, for
// column col of each row tile.
//
// begin_steps masks, raises the references where needed, and leaves d, the log2 of each subtile's
// value scale over the wave's reference.  finish_step gives a step's probabilities times that
// factor, as the product with the values takes them, and adds them to the running sums without
// it.  The factor enters the exponent, 2^(x - m + d), instead of a product per probability; d is
// held above -40, where fp16 has dropped the values anyway, so that the sums keep every token.
template <int D, int RT, int ST>
__device__ __forceinline__ void begin_steps(State<D, RT>& s, f4 (&sc)[ST][RT][2], float (&fk)[ST][RT][2],
                                            const int (&lim)[RT], int lim_lo, int t, int end,
                                            const float* lsv, int quad, float (&d)[2 * ST]) {
  const bool masked = t + 32 * ST > lim_lo || t + 32 * ST > end;
  if (masked) {
    // (through fresh(), so that the selects stay in the branch)
    const int first = fresh(t + quad * 4);
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int a = 0; a < 2; ++a) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int tok = first + st * 32 + a * 16 + e;
            sc[st][r][a][e] = tok < lim[r] && tok < end ? sc[st][r][a][e] * fk[st][r][a]
                                                         : -__builtin_inff();
          }
          fk[st][r][a] = 1.0f;
        }
  }
  float top[RT], most = lsv[0];
#pragma unroll
  for (int i = 1; i < 2 * ST; ++i) most = fmaxf(most, lsv[i]);
  bool over = most > s.lv;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    top[r] = -__builtin_inff();
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const f4 x = sc[st][r][a];
        top[r] = fmaxf(top[r], fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), x[3]) * fk[st][r][a]);
      }
    over |= top[r] > s.m[r] + kAbove;
  }
  if (__any(over)) raise(s, top, most);
#pragma unroll
  for (int i = 0; i < 2 * ST; ++i) d[i] = fmaxf(lsv[i] - s.lv, -40.0f);
}

enum { kPlain, kSubSums, kNoSums };   // sums of finish_step: for l; also of subtiles; none (the caller's)
template <int D, int RT, int SUMS>
__device__ __forceinline__ void finish_step(State<D, RT>& s, const f4 (&sc)[RT][2],
                                            const float (&fk)[RT][2], const float* d, int t, int end,
                                            int col, int quad, const SubSums& sums,
                                            float (&pr)[RT][8]) {
  const float back[2] = {exp2_fast(-d[0]), exp2_fast(-d[1])};
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    // a column that has seen nothing keeps reference -inf: x - 0 is -inf, its exponential 0
    const float m = s.m[r] == -__builtin_inff() ? 0.0f : s.m[r];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const float c = d[a] - m;
#pragma unroll
      for (int e = 0; e < 4; ++e) pr[r][a * 4 + e] = exp2_fast(__builtin_fmaf(sc[r][a][e], fk[r][a], c));
      if constexpr (SUMS == kNoSums) continue;
      const float part = (pr[r][a * 4] + pr[r][a * 4 + 1]) + (pr[r][a * 4 + 2] + pr[r][a * 4 + 3]);
      s.l[r] = __builtin_fmaf(part, back[a], s.l[r]);
      if constexpr (SUMS == kSubSums) {
        const float y = quad_sum(part) * back[a];
        const int row = sums.row0 + r * 16 + col;
        if (quad == 0 && row < sums.rows && t + a * 16 < end)
          sums.at[(int64_t)((t >> 4) + a) * sums.rows + row] = {y, s.m[r]};
      }
    }
  }
}

template <int RT>
__device__ __forceinline__ void to_operand(const float (&pr)[RT][8], h8 (&ph)[RT]) {
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int e = 0; e < 8; ++e) ph[r][e] = (_Float16)pr[r][e];
}

// log2 of a block's value scale (of a block of zeros: the smallest reference).  A NaN value scale is
// carried by the key scale: it makes NaN of the scores, and is masked with them.
__device__ __forceinline__ float log_scale(float sv) {
  return sv >= 0x1p-100f ? __builtin_amdgcn_logf(sv) : kTinyScale;
}
__device__ __forceinline__ float key_scale(float sk, float sv) { return sv == sv ? sk : sv; }

// Query rows row0 + 16 r + col, channels i*64 + quad*16 + h*8 + e (operand n = 2 i + h), as given.
union Raw {
  u4 v;
  uint16_t h[8];
};
__device__ __forceinline__ u4 load_query(const DenseAttnParams& p, int b, int g, int row, int ch) {
  const int jq = row / p.group, iq = row % p.group;
  const uint16_t* src = p.q + b * p.qs_b + jq * p.qs_t + (g * p.group + iq) * p.qs_h + ch;
  Raw w;
  if (p.q_wide) {
    w.v = *reinterpret_cast<const u4*>(src);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) w.h[e] = src[e];
  }
  return w.v;
}
template <int D, int RT>
__device__ __forceinline__ void load_queries(const DenseAttnParams& p, int b, int g, int row0, int col,
                                             int quad, const int (&lm)[RT], Raw (&raw)[RT][D / 32]) {
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      raw[r][i].v = lm[r] < 0 ? (u4){0, 0, 0, 0}
                              : load_query(p, b, g, row0 + r * 16 + col,
                                           (i >> 1) * 64 + quad * 16 + (i & 1) * 8);
}
// The same as fp16, scaled by a power of two per row; qs: what then makes a score a log2 score.
template <int D, int RT>
__device__ __forceinline__ void scale_queries(const DenseAttnParams& p, const Raw (&raw)[RT][D / 32],
                                              h8 (&q)[RT][D / 32], float (&qs)[RT]) {
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(from16(raw[r][i].h[e], p.c.bf16)));
    top = quad_max(top);
    const int ex = top > 0.0f && top < __builtin_inff() ? 8 - __builtin_amdgcn_frexp_expf(top) : 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        q[r][i][e] = (_Float16)__builtin_amdgcn_ldexpf(from16(raw[r][i].h[e], p.c.bf16), ex);
    qs[r] = __builtin_amdgcn_ldexpf(p.scale_log2, -ex);
  }
}

__device__ __forceinline__ f4 mfma_raw(u4 a, u4 b, f4 c, int bf16) {
  return bf16 ? mfma_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c)
              : mfma_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c);
}

// The unfinished block, from its 16-bit rows: 32-token steps at t0, t0 + stride, .. below `end`
// (of ctx tokens).  Operands are the stored type; a bf16 probability is split in two parts.
// A value that is not finite is left out of the product, where it would reach rows that do not
// see its token; the rows that do get NaN in its channel.
template <int D, int RT, bool SUMS>
__device__ __forceinline__ void unfinished_block(const DenseAttnParams& p, State<D, RT>& s, int b, int g,
                                                 int ctx, int end, int t0, int stride, int row0,
                                                 const int (&lim)[RT], int lim_lo,
                                                 const SubSums& sums, int lane) {
  constexpr int CT = D / 16;
  const int col = lane & 15, quad = lane >> 4, T = 1 << p.c.shift, bf16 = p.c.bf16;
  const uint16_t* kt = p.c.tails + ((int64_t)b * p.c.n_kv + g) * 2 * (2 * T * D);
  const uint16_t* vt = kt + 2 * T * D;
  for (int t = t0; t < end; t += stride) {
    f4 sc[1][RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) sc[0][r][0] = sc[0][r][1] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const int ch = (i >> 1) * 64 + quad * 16 + (i & 1) * 8;
      u4 k[2];
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const int tok = t + a * 16 + col;
        k[a] = tok < ctx ? *reinterpret_cast<const u4*>(kt + (tok & (2 * T - 1)) * D + ch)
                         : (u4){0, 0, 0, 0};
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        u4 q = {0, 0, 0, 0};
        if (lim[r] != 0x7fffffff) q = load_query(p, b, g, row0 + r * 16 + col, ch);
#pragma unroll
        for (int a = 0; a < 2; ++a) sc[0][r][a] = mfma_raw(k[a], q, sc[0][r][a], bf16);
      }
    }
    float fk[1][RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) fk[0][r][0] = fk[0][r][1] = p.scale_log2;
    const float lsv[2] = {0.0f, 0.0f};
    float d[2], pr[RT][8];
    begin_steps<D, RT, 1>(s, sc, fk, lim, lim_lo, t, ctx, lsv, quad, d);
    finish_step<D, RT, SUMS ? kSubSums : kPlain>(s, sc[0], fk[0], d, t, ctx, col, quad, sums, pr);
    u4 pa[RT], pb[RT];                              // fp16; or two bf16 parts
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      union { _Float16 h[8]; __bf16 b[8]; u4 v; } hi, lo;
      lo.v = (u4){0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = pr[r][e];
        if (bf16) {
          hi.b[e] = (__bf16)x;
          lo.b[e] = (__bf16)(x - (float)hi.b[e]);
        } else {
          hi.h[e] = (_Float16)x;
        }
      }
      pa[r] = hi.v;
      pb[r] = lo.v;
    }
    const uint32_t inf16 = bf16 ? 0x7f80u : 0x7c00u, one = bf16 ? 0x3f80u : 0x3c00u;
#pragma unroll
    for (int c0 = 0; c0 < CT; c0 += 4) {
      // values: tokens t + 16 a + 4 quad .. + 3 of channel 16 c + col; absent ones cleared
      u4 v[4];
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int tok = t + a * 16 + quad * 4, rr = tok & (2 * T - 1);
          u2 w = {0, 0};
          if (tok < ctx) {
            w = *reinterpret_cast<const u2*>(vt + ((rr >> 4) * D + (c0 + c) * 16 + col) * 16 + quad * 4);
            const int left = ctx - tok;
            if (left < 2) w.x &= 0xffffu;
            if (left < 3) w.y = 0;
            else if (left < 4) w.y &= 0xffffu;
          }
          v[c][2 * a] = w.x;
          v[c][2 * a + 1] = w.y;
        }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          top = max(top, max((v[c][i] & 0x7fffu) << 16, v[c][i] & 0x7fff0000u));
      if (__any(top >= inf16 << 16)) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u4 bad;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool lo = (v[c][i] & 0x7fffu) >= inf16, hi = (v[c][i] >> 16 & 0x7fffu) >= inf16;
            bad[i] = (lo ? one : 0) | (hi ? one << 16 : 0);
            v[c][i] &= (lo ? 0 : 0xffffu) | (hi ? 0 : 0xffff0000u);
          }
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            u4 sees;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tok = t + (i >> 1) * 16 + quad * 4 + (i & 1) * 2;
              sees[i] = (tok < lim[r] ? one : 0) | (tok + 1 < lim[r] ? one << 16 : 0);
            }
            const f4 n = mfma_raw(bad, sees, (f4){0.0f, 0.0f, 0.0f, 0.0f}, bf16);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s.o[r][c0 + c][e] = n[e] > 0.0f ? __builtin_nanf("") : s.o[r][c0 + c][e];
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          s.o[r][c0 + c] = mfma_raw(v[c], pa[r], s.o[r][c0 + c], bf16);
          if (bf16) s.o[r][c0 + c] = mfma_raw(v[c], pb[r], s.o[r][c0 + c], 1);
        }
    }
  }
}

// Sixteen bytes of codes; past the caches where one wave alone reads them (5.8 TB/s with plain loads,
// 6.7 with these).
template <int READERS>
__device__ __forceinline__ u4 load_codes(const uint8_t* a) {
  const u4* v = reinterpret_cast<const u4*>(a);
  if constexpr (READERS == 1) return __builtin_nontemporal_load(v);
  else return *v;
}

// Up to 64 query rows of a KV head.  A workgroup's waves take 32-token steps in turn.  A wave holds
// RT row tiles: one or two in 256 registers, so that two workgroups fit a compute unit; three in
// the registers of a whole SIMD (40 rows: 75 us against 92 with two groups of two tiles, 2 x 64K
// tokens of 8 heads).  Four tiles spill; there (RG = 2) two groups of two tiles share the steps,
// and the codes' second reader finds them in cache (64 rows: 96 us against 132).
template <int D, bool E4M3, int RT, int RG, bool SUMS>
__global__ __launch_bounds__(256, RT >= 3 ? 1 : 2) void dense_split_kernel(const DenseAttnParams p) {
  constexpr int N = D / 64, CT = D / 16, NB = RT == 1 ? 3 : 2, TW = kWavesA / RG, kRound = 32 * TW;
  const int tid_lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int token_wave = wave / RG, row0 = wave % RG * (16 * RT), g = blockIdx.y;
  const Lens lens = first_lens(p, tid_lane);
  const int R = range_units(p, lens, tid_lane);
  __shared__ float so[kWavesA][16][D + 4];
  __shared__ float sm[kWavesA][RT * 16], sl[kWavesA][RT * 16];
  const int sh = p.c.shift, T = 1 << sh;
  if (blockIdx.x == 0 && blockIdx.y == 0 && wave == 0) write_slots(p, lens, R, tid_lane);
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
    const int e8 = min(it.t1, full), tw = it.t0 + 32 * token_wave;   // the wave's finished blocks

    // The chains of loads that a part begins with overlap: the table entries of the first 64 steps
    // (a subtile per lane and 32 steps), the queries, then the entries' scales and codes.
    const int32_t* table = p.c.table + head * p.c.blocks_per_head;
    auto entry_token = [&](int i0) {
      return max(min(tw + (i0 + (lane >> 1)) * kRound + (lane & 1) * 16, e8 - 16), 0);
    };
    const int entry0 = table[entry_token(0) >> sh], entry1 = table[entry_token(32) >> sh];

    // queries: row r of the tile in column `col`, channels i*64 + quad*16 + h*8 + e
    h8 q[RT][2 * N];
    float qs[RT];
    int lim[RT];
    int lm[RT];
    int lim_lo = 0x7fffffff;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      lm[r] = row_limit(p, it.b, it.ctx, row0 + r * 16 + col);
      lim[r] = lm[r] < 0 ? 0x7fffffff : lm[r];       // rows without a query see everything
      lim_lo = min(lim_lo, lim[r]);
    }
    Raw raw[RT][2 * N];
    load_queries<D, RT>(p, it.b, g, row0, col, quad, lm, raw);
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) lim_lo = min(lim_lo, __shfl_xor(lim_lo, o));
    lim_lo = __builtin_amdgcn_readfirstlane(lim_lo);

    const int steps = e8 > tw ? (e8 - tw + kRound - 1) / kRound : 0;
    struct Entry { uint32_t sub; float sk, lsv; };
    auto entry_of = [&](int e, int i0) {
      const int t = entry_token(i0);
      e = min(max(e, 0), p.c.n_blocks - 1);
      const Pair sc = p.c.scales[e];
      return Entry{((uint32_t)e << (sh - 3)) + ((uint32_t)(t & (T - 1)) >> 4), key_scale(sc.x, sc.y),
                       log_scale(sc.y)};
    };
    const uint32_t v_sub = (uint32_t)T >> 4;          // from a key subtile to its value subtile
    auto load = [&](Tile<D>& x, const Entry& en, int i) {
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const int l = 2 * (i & 31) + a;
        const uint32_t sub = __builtin_amdgcn_readlane(en.sub, l);
        x.sk[a] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(en.sk), l));
        x.lsv[a] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(en.lsv), l));
        const uint8_t* kb = p.c.codes + (uint64_t)sub * (16 * D) + lane * 16;
        const uint8_t* vb = p.c.codes + (uint64_t)(sub + v_sub) * (16 * D) + lane * 16;
#pragma unroll
        for (int n = 0; n < N; ++n)
          x.k[a][n] = load_codes<RG>(kb + n * 1024);
#pragma unroll
        for (int n = 0; n < N; ++n)
          x.v[a][n] = load_codes<RG>(vb + n * 1024);
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

    scale_queries<D, RT>(p, raw, q, qs);

    State<D, RT> s;
    reset(s);
    const SubSums sums = {SUMS ? p.sub + head * p.sub_per_head * p.rows : nullptr, row0, p.rows};
    // ---- finished blocks
    auto compute = [&](const Tile<D>& y, int i) {
      const int t = tw + i * kRound;
      f4 sc[1][RT][2];
      float fk[1][RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[0][r][0] = sc[0][r][1] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          h8 k[2];
#pragma unroll
          for (int a = 0; a < 2; ++a) k[a] = code8<E4M3>(y.k[a][n][2 * h], y.k[a][n][2 * h + 1]);
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int a = 0; a < 2; ++a) sc[0][r][a] = mfma_f16(k[a], q[r][2 * n + h], sc[0][r][a]);
        }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        fk[0][r][0] = y.sk[0] * qs[r];
        fk[0][r][1] = y.sk[1] * qs[r];
      }
      float d[2], pr[RT][8];
      begin_steps<D, RT, 1>(s, sc, fk, lim, lim_lo, t, e8, y.lsv, quad, d);
      finish_step<D, RT, SUMS ? kSubSums : kPlain>(s, sc[0], fk[0], d, t, e8, col, quad, sums, pr);
      h8 ph[RT];
      to_operand<RT>(pr, ph);
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

    if (full < it.t1)
      unfinished_block<D, RT, SUMS>(p, s, it.b, g, it.ctx, it.ctx, full + 32 * token_wave, kRound, row0,
                                    lim, lim_lo, sums, fresh(tid_lane));

    lane = fresh(tid_lane);
    col = lane & 15;
    quad = lane >> 4;
    // ---- the token waves' states merged, normalized and written as the part's partial
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float l = quad_sum(s.l[r]);
      if (quad == 0) {
        sm[wave][r * 16 + col] = s.m[r];
        sl[wave][r * 16 + col] = l;
      }
    }
    __syncthreads();
    const int64_t slot0 = ((int64_t)(blockIdx.x + it.b) * p.c.n_kv + g) * p.rows;
    const float vref = exp2_fast(s.lv);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int group = wave % RG;
      float M = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < TW; ++w) M = fmaxf(M, sm[w * RG + group][r * 16 + col]);
      float L = 0.0f, own = 0.0f;
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float mw = sm[w * RG + group][r * 16 + col], lw = sl[w * RG + group][r * 16 + col];
        const float a = mw == M ? 1.0f : exp2_fast(mw - M);
        // a wave without tokens: sum 0 (NaN stays)
        L += lw * a;
        if (w == token_wave) own = a;
      }
      const float f = L == 0.0f ? 0.0f : own / L;
      if (token_wave == 0 && quad == 0 && row0 + r * 16 + col < p.rows)
        p.part_ml[slot0 + row0 + r * 16 + col] = {M, L};
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        f4 v = s.o[r][c] * f;                         // at most the largest code, then the scale
        v *= vref;
        *reinterpret_cast<f4*>(&so[wave][col][c * 16 + quad * 4]) = v;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < RG * 16 * D / 4; i += 256) {
        const int gr = i / (16 * D / 4), row = i / (D / 4) % 16, ch = i % (D / 4) * 4;
        const int to = gr * (16 * RT) + r * 16 + row;
        if (to < p.rows) {
          f4 v = *reinterpret_cast<const f4*>(&so[gr][row][ch]);
#pragma unroll
          for (int w = 1; w < TW; ++w) v += *reinterpret_cast<const f4*>(&so[w * RG + gr][row][ch]);
          *reinterpret_cast<f4*>(p.part_o + (slot0 + to) * D + ch) = v;
        }
      }
      __syncthreads();
    }
    at = pl.start + units_of(pl.ctx);
    if (at >= at_end || !find_unit(p, lens, at, tid_lane, &pl)) return;
  }
}

// Four channels of an output row.
__device__ __forceinline__ void store_out(uint16_t* to, f4 v, int bf16, int wide) {
  union { _Float16 h[4]; __bf16 b[4]; uint16_t u[4]; u2 w; } x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (bf16) x.b[e] = (__bf16)v[e];
    else x.h[e] = (_Float16)v[e];
  }
  if (wide) {
    *reinterpret_cast<u2*>(to) = x.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = x.u[e];
  }
}

// ---- chunk --------------------------------------------------------------------------
// More than 64 query rows of a KV head: the matrix products bound it (4 d flops per row and token
// against 2 d bytes per token).  A workgroup takes 128 rows, 32 a wave, so that a wave's state
// and operands fit 256 registers and two workgroups share a compute unit: one's softmax runs
// beside the other's products.  Tiles of 64 tokens are converted to fp16 once per workgroup, into
// LDS in the operands' order (a wave's operand is 1 KiB in a row: no bank conflicts): two buffers,
// one barrier a tile, the codes of the next tile already in registers.  512 query tokens of 32 heads
// over 32768 tokens of 8 KV heads: 326 us, 844 TFLOP/s, matrix cores busy a third and vector ALU
// half of the cycles.
//
// Workgroups of the same codes (row tiles of one KV head and range) have consecutive places on one
// XCD, whose L2 then serves all but the first of them.
constexpr int kTile = 64;                   // tokens

template <int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void dense_chunk_kernel(const DenseAttnParams p) {
  constexpr int N = D / 64, CT = D / 16, RT = 2;
  constexpr int kFrag = 1024;               // bytes of a wave's operand
  constexpr int kKeys = 4 * 2 * N * kFrag, kValues = 2 * CT * kFrag;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][kKeys + kValues];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int tiles = (p.rows + kChunkRows - 1) / kChunkRows;
  // (range, KV head) pairs go round the XCDs, row tiles of a pair stay on one, the last (which
  // sees most) first
  const int xcd = blockIdx.x & 7, place = blockIdx.x >> 3;
  const int pair = place / tiles * 8 + xcd, tile = tiles - 1 - place % tiles;
  if (pair >= p.ranges * p.c.n_kv) return;
  const int g = pair % p.c.n_kv, range = pair / p.c.n_kv;
  const int row0 = tile * kChunkRows + wave * (16 * RT);
  const int sh = p.c.shift, T = 1 << sh;
  const Lens lens = first_lens(p, lane);
  const int R = range_units(p, lens, lane);
  if (blockIdx.x == 0 && wave == 0) write_slots(p, lens, R, lane);
  Place pl;
  int at = range * R;
  const int at_end = at + R;
  if (!find_unit(p, lens, at, lane, &pl)) return;
  for (;;) {
    const int b = pl.b, ctx = pl.ctx;
    const int t0 = (at - pl.start) * kUnit;
    const int t1 = min(min(at_end - pl.start, units_of(ctx)) * kUnit, ctx);
    const int full = ctx & ~(T - 1);
    const int64_t head = (int64_t)b * p.c.n_kv + g;
    const int q_len = p.q_len ? min(max(p.q_len[b], 0), p.n_q) : p.n_q;
    // query tokens of the workgroup's rows, and how far the last of them sees
    const int j_lo = tile * kChunkRows / p.group;
    const int j_hi = min((tile * kChunkRows + kChunkRows - 1) / p.group, q_len - 1);
    const int sees = min(ctx - q_len + j_hi + 1, ctx);
    if (j_lo < q_len) {
      int lim[RT], lm[RT], lim_lo = 0x7fffffff;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        lm[r] = row_limit(p, b, ctx, row0 + r * 16 + col);
        lim[r] = lm[r] < 0 ? 0x7fffffff : lm[r];
        lim_lo = min(lim_lo, lim[r]);
      }
#pragma unroll
      for (int o = 8; o >= 1; o >>= 1) lim_lo = min(lim_lo, __shfl_xor(lim_lo, o));
      lim_lo = __builtin_amdgcn_readfirstlane(lim_lo);
      h8 q[RT][2 * N];
      float qs[RT];
      {
        Raw raw[RT][2 * N];
        load_queries<D, RT>(p, b, g, row0, col, quad, lm, raw);
        scale_queries<D, RT>(p, raw, q, qs);
      }
      State<D, RT> s;
      reset(s);
      const SubSums none = {nullptr, 0, 0};
      // row i of the first factor: ones over subtile i / 8's tokens (its lane: row col)
      h8 ones;
#pragma unroll
      for (int e = 0; e < 8; ++e) ones[e] = (e < 4) == (col < 8) ? (_Float16)1.0f : (_Float16)0.0f;

      const int e8 = min(min(t1, full), (sees + 15) & ~15);
      const int n = e8 > t0 ? (e8 - t0 + kTile - 1) / kTile : 0;
      const int32_t* table = p.c.table + head * p.c.blocks_per_head;
      // entries of 16 tiles, a subtile per lane
      struct Entry { uint32_t sub; float sk, lsv; };
      auto entries = [&](int i0) {
        const int t = max(min(t0 + i0 * kTile + lane * 16, e8 - 16), 0);
        const int e = min(max(table[t >> sh], 0), p.c.n_blocks - 1);
        const Pair sc = p.c.scales[e];
        return Entry{((uint32_t)e << (sh - 3)) + ((uint32_t)(t & (T - 1)) >> 4), key_scale(sc.x, sc.y),
                     log_scale(sc.y)};
      };
      const uint32_t v_sub = (uint32_t)T >> 4;
      // A thread's codes of a tile: key units tid + 256 i (subtile, then 16-byte unit); value units of
      // the two subtiles of a 32-token step.
      constexpr int kUnits = 16 * D / 16;           // 16-byte units of a subtile
      constexpr int KL = 4 * kUnits / 256;          // 2 (D 128) or 1
      u4 kc[KL], vc[2];
      Entry now, next;
      auto subtile = [&](const Entry& en, int i, int st) {
        return (uint32_t)__builtin_amdgcn_readlane(en.sub, (i & 15) * 4 + st);
      };
      const int tid = threadIdx.x;
      auto load = [&](const Entry& en, int i) {
#pragma unroll
        for (int k = 0; k < KL; ++k) {
          const int u = wave * 64 + k * 256, st = u / kUnits;
          kc[k] = *reinterpret_cast<const u4*>(p.c.codes + (uint64_t)subtile(en, i, st) * (16 * D) +
                                               (u % kUnits + lane) * 16);
        }
        if (wave * 64 < 2 * kUnits) {
          const int u = wave * 64, sp = u / kUnits;
#pragma unroll
          for (int a = 0; a < 2; ++a)
            vc[a] = *reinterpret_cast<const u4*>(
                p.c.codes + (uint64_t)(subtile(en, i, sp * 2 + a) + v_sub) * (16 * D) +
                (u % kUnits + lane) * 16);
        }
      };
      auto store = [&](uint8_t* buf) {
#pragma unroll
        for (int k = 0; k < KL; ++k) {
          const int u = tid + k * 256, st = u / kUnits, w = u % kUnits, i = w >> 6;
          uint8_t* to = buf + (st * 2 * N + 2 * i) * kFrag + (w & 63) * 16;
          *reinterpret_cast<h8*>(to) = code8<E4M3>(kc[k][0], kc[k][1]);
          *reinterpret_cast<h8*>(to + kFrag) = code8<E4M3>(kc[k][2], kc[k][3]);
        }
        if (wave * 64 < 2 * kUnits) {
          const int sp = tid / kUnits, w = tid % kUnits, i = w >> 6;
          uint8_t* to = buf + kKeys + (sp * CT + 4 * i) * kFrag + (w & 63) * 16;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<h8*>(to + j * kFrag) = code8<E4M3>(vc[0][j], vc[1][j]);
        }
      };
      __syncthreads();                              // the buffers' last readers are done
      if (n > 0) {
        now = entries(0);
        next = entries(16);
        load(now, 0);
        store(lds[0]);
        load(now, min(1, n - 1));
      }
      __syncthreads();
      for (int i = 0; i < n; ++i) {
        // the scales of this tile (its entries may be replaced below)
        float sk[4], lsv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int l = (i & 15) * 4 + k;
          sk[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(now.sk), l));
          lsv[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(now.lsv), l));
        }
        const uint8_t* buf = lds[i & 1];
        const int t = t0 + i * kTile;
        // both steps' scores first: the second's exponentials run beside the first's products
        f4 sc[2][RT][2];
        float fk[2][RT][2], d[4];
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int a = 0; a < 2; ++a) {
#pragma unroll
            for (int r = 0; r < RT; ++r) sc[st][r][a] = (f4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < 2 * N; ++k) {
              const h8 kf = *reinterpret_cast<const h8*>(buf + ((st * 2 + a) * 2 * N + k) * kFrag + lane * 16);
#pragma unroll
              for (int r = 0; r < RT; ++r) sc[st][r][a] = mfma_f16(kf, q[r][k], sc[st][r][a]);
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) fk[st][r][a] = sk[st * 2 + a] * qs[r];
          }
        begin_steps<D, RT, 2>(s, sc, fk, lim, lim_lo, t, e8, lsv, quad, d);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          float pr[RT][8];
          finish_step<D, RT, kNoSums>(s, sc[st], fk[st], d + 2 * st, t, e8, col, quad, none, pr);
          h8 ph[RT];
          to_operand<RT>(pr, ph);
          // The sums by one more product, of rows that are one over a subtile's tokens: the lanes of
          // quads 0 and 1 get the first subtile's sum, the others the second's (each twice).  Where
          // the value scales make the operand small, fp16 would drop tokens from the sums: added
          // in fp32 (twice, as above).
          const float d0 = d[2 * st], d1 = d[2 * st + 1];
          const float low = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(fminf(d0, d1))));
          if (low >= -4.0f) {
            const float back = exp2_fast(-(quad < 2 ? d0 : d1));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
              const f4 sum = mfma_f16(ones, ph[r], (f4){0.0f, 0.0f, 0.0f, 0.0f});
              s.l[r] = __builtin_fmaf(sum[0], back, s.l[r]);
            }
          } else {
            const float b0 = 2.0f * exp2_fast(-d0), b1 = 2.0f * exp2_fast(-d1);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
              const float x = (pr[r][0] + pr[r][1]) + (pr[r][2] + pr[r][3]);
              const float y = (pr[r][4] + pr[r][5]) + (pr[r][6] + pr[r][7]);
              s.l[r] = __builtin_fmaf(y, b1, __builtin_fmaf(x, b0, s.l[r]));
            }
          }
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            const h8 vf = *reinterpret_cast<const h8*>(buf + kKeys + (st * CT + c) * kFrag + lane * 16);
#pragma unroll
            for (int r = 0; r < RT; ++r) s.o[r][c] = mfma_f16(vf, ph[r], s.o[r][c]);
          }
        }
        // the next tile's codes, in registers since the last one, and the loads of the one after
        if (i + 1 < n) store(lds[(i + 1) & 1]);
        if (((i + 1) & 15) == 0) {
          now = next;
          next = entries(i + 17);
        }
        // (tile i + 2 lies in the next 16 when i + 1 ends these)
        if (i + 2 < n) load(((i + 2) & 15) == 0 ? next : now, i + 2);
        __syncthreads();
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) s.l[r] *= 0.5f;
      if (full < t1 && sees > full)
        unfinished_block<D, RT, false>(p, s, b, g, ctx, min(ctx, sees), full, 32, row0, lim, lim_lo, none,
                                       fresh(lane));

      const float vref = exp2_fast(s.lv);
      // one range: the whole sequence was seen, and this is the output; else a partial
      const int64_t slot0 = ((int64_t)(range + b) * p.c.n_kv + g) * p.rows;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int row = row0 + r * 16 + col;
        const float L = quad_sum(s.l[r]);
        const float f = L == 0.0f ? 0.0f : 1.0f / L;
        if (p.ranges == 1) {
          if (lm[r] >= 0) {
            const int jq = row / p.group, iq = row % p.group;
            uint16_t* out = p.out + b * p.os_b + jq * p.os_t + (g * p.group + iq) * p.os_h + quad * 4;
#pragma unroll
            for (int c = 0; c < CT; ++c) {
              f4 v = s.o[r][c] * f;
              v *= vref;
              store_out(out + c * 16, v, p.c.bf16, p.out_wide);
            }
          }
        } else if (row < p.rows) {
          if (quad == 0) p.part_ml[slot0 + row] = {s.m[r], L};
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            f4 v = s.o[r][c] * f;
            v *= vref;
            *reinterpret_cast<f4*>(p.part_o + (slot0 + row) * D + c * 16 + quad * 4) = v;
          }
        }
      }
    }
    at = pl.start + units_of(ctx);
    if (at >= at_end || !find_unit(p, lens, at, lane, &pl)) return;
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
  const Slots sl = p.slots[b];
  const int first = sl.first, count = sl.count, ctx = sl.ctx;
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
  const Slots sl = p.slots[b];
  const int first = sl.first, count = sl.count, ctx = sl.ctx;
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

// The same for the chunk kernel's many rows: a wave takes four rows at once, sixteen lanes a row for
// the parts' references and sums.  With one range the rows are written already, but for
// sequences without tokens.
template <int D>
__global__ __launch_bounds__(256) void dense_combine_rows_kernel(const DenseAttnParams p) {
  constexpr int C = D / 64, K = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.y, b = blockIdx.z, row0 = (blockIdx.x * 4 + wave) * K;
  const Slots sl = p.slots[b];
  const int first = sl.first, count = sl.count, ctx = sl.ctx;
  if ((p.ranges == 1 && count > 0) || row0 >= p.rows) return;
  const int n = min(K, p.rows - row0), i16 = lane & 15;
  const int64_t step = (int64_t)p.c.n_kv * p.rows;
  const int64_t slot0 = ((int64_t)first * p.c.n_kv + g) * p.rows + row0;
  const Pair* ml = p.part_ml + slot0 + min(lane >> 4, n - 1);
  auto part = [&](int i) { return i < count ? ml[i * step] : Pair{-__builtin_inff(), 0.0f}; };
  const Pair head = part(i16);
  float m = head.x;
  for (int i = 16 + i16; i < count; i += 16) m = fmaxf(m, ml[i * step].x);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.0f, o[K][C] = {};
  for (int i0 = 0; i0 < count; i0 += 16) {
    const Pair x = i0 ? part(i0 + i16) : head;
    const float f = x.x == m ? x.y : x.y * exp2_fast(x.x - m);
    l += f;
    const int most = min(16, count - i0);
#pragma unroll 4
    for (int u = 0; u < most; ++u)
#pragma unroll
      for (int r = 0; r < K; ++r) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), r * 16 + u));
        const int64_t slot = slot0 + (i0 + u) * step + min(r, n - 1);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float v = p.part_o[slot * D + lane * C + c];
          o[r][c] += w == 0.0f ? 0.0f : w * v;
        }
      }
  }
#pragma unroll
  for (int x = 1; x < 16; x <<= 1) l += __shfl_xor(l, x);
#pragma unroll
  for (int r = 0; r < K; ++r) {
    const int row = row0 + r;
    const float lr = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l), r * 16));
    if (row_limit(p, b, ctx, row) < 0) continue;
    const int jq = row / p.group, iq = row % p.group;
    uint16_t* out = p.out + b * p.os_b + jq * p.os_t + (g * p.group + iq) * p.os_h + lane * C;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float v = lr == 0.0f ? 0.0f : o[r][c] / lr;
      out[c] = p.c.bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v)
                        : __builtin_bit_cast(uint16_t, (_Float16)v);
    }
  }
}

template <int D, bool E4M3, int RT, int RG>
void launch_split(const DenseAttnParams& p, hipStream_t st) {
  const dim3 grid(p.ranges, p.c.n_kv);
  if (p.weights) hipLaunchKernelGGL((dense_split_kernel<D, E4M3, RT, RG, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((dense_split_kernel<D, E4M3, RT, RG, false>), grid, dim3(256), 0, st, p);
}

template <int D, bool E4M3>
void launch_rows(const DenseAttnParams& p, hipStream_t st) {
  if (p.rows <= 16) launch_split<D, E4M3, 1, 1>(p, st);
  else if (p.rows <= 32) launch_split<D, E4M3, 2, 1>(p, st);
  else if (p.rows <= 48) launch_split<D, E4M3, 3, 1>(p, st);
  else if (p.rows <= kSplitRows) launch_split<D, E4M3, 2, 2>(p, st);
  else {
    const int tiles = (p.rows + kChunkRows - 1) / kChunkRows;
    const int pairs = (p.ranges * p.c.n_kv + 7) / 8 * 8;
    hipLaunchKernelGGL((dense_chunk_kernel<D, E4M3>), dim3(pairs * tiles), dim3(256), 0, st, p);
  }
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
  if (p.rows > kSplitRows) {
    const dim3 grid((p.rows + 15) / 16, p.c.n_kv, p.c.batch);
    if (p.c.d == 128) hipLaunchKernelGGL(dense_combine_rows_kernel<128>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(dense_combine_rows_kernel<64>, grid, dim3(256), 0, st, p);
    return (int)hipGetLastError();
  }
  const int J = (p.max_ctx + (1 << p.c.shift) - 1) >> p.c.shift;
  const dim3 grid(p.rows + (p.weights ? (J + 255) / 256 : 0), p.c.n_kv, p.c.batch);
  if (p.c.d == 128) hipLaunchKernelGGL(dense_combine_kernel<128>, grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(dense_combine_kernel<64>, grid, dim3(256), 0, st, p);
  return (int)hipGetLastError();
}

}  // namespace starkv
