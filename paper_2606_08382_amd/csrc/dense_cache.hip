// The 8-bit cache of an uncompressed layer: append, read-back and eviction.
#include <hip/hip_runtime.h>

#include "dense.h"

namespace starkv {

namespace {

typedef uint32_t u4c __attribute__((ext_vector_type(4)));
typedef float f2c __attribute__((ext_vector_type(2)));
typedef uint16_t us2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float from16(uint32_t u, int bf16) {
  return bf16 ? __uint_as_float(u << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)u);
}
__device__ __forceinline__ uint16_t to_f16(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// Element offsets of (row, channel) inside a (sequence, KV head)'s 16-bit tail planes.
__device__ __forceinline__ int tail_value(int row, int ch, int d) {
  return ((row >> 4) * d + ch) * 16 + (row & 15);
}

// Eight elements of a row.
__device__ __forceinline__ u4c load8(const uint16_t* a, int wide) {
  if (wide) return *reinterpret_cast<const u4c*>(a);
  union { u4c v; uint16_t h[8]; } w;
#pragma unroll
  for (int e = 0; e < 8; ++e) w.h[e] = a[e];
  return w.v;
}

// ------------------------------------------------------------------------------ append
//
// One workgroup per 64 tokens (or a block of 128) of the blocks that the new tokens touch, KV head
// and keys or values.  A block that they finish is gathered into LDS (its earlier tokens from the 16-bit tail), its
// absolute maximum taken on the bit patterns, and its codes written in the order that the
// attention's matrix operands take (see the header).  The first workgroup also moves the new
// tokens of the last two blocks into the tail: it is the only one that reads the tail, and it
// does so before it writes.  Bound by HBM in bulk (4 x 131072 tokens of 8 heads: 655 to 690 us, 4.7 to
// 4.9 TB/s) and by latency below (64 tokens 7 us, 4096 tokens of two sequences 17).
//
// Codes are RN(x / s), decided exactly.  Borders between two codes have few bits (at most 8 in the
// significand), so a quotient may be replaced by any value on the same side of the nearest 8-bit
// number b: b itself if the quotient equals it, else b moved by one unit of fp32 towards the
// quotient, as the sign of the residual x - b s tells, which fma gives exactly.
// INT8 seldom needs that: the products of x with two reciprocals of s, 2^-22 below and above,
// enclose the quotient, and where all sixteen codes of a thread come out alike from both they are
// right.  (E4M3's coarse grid meets the quotients of 16-bit values far more often, in nearly every
// wave.)  Scales below 2^-60 and their rows are multiplied by 2^100 first, so that the
// residual does not underflow.  Measured against an fp32 division with residuals for all values:
// 4 x 131072 tokens of 8 heads in INT8 852 -> 655 us.
struct Quantizer {
  float lift, s, inv;
  __device__ __forceinline__ Quantizer(float scale) {
    lift = scale < 0x1p-60f ? 0x1p100f : 1.0f;
    s = scale * lift;
    inv = s > 0.0f ? 1.0f / s : 0.0f;
  }
  __device__ __forceinline__ float quotient(float x) const {
    const uint32_t b = (__float_as_uint(x * inv) + 0x8000u) & 0xffff0000u;
    const float r = __builtin_fmaf(-__uint_as_float(b), s, x);
    const int towards = (int)(__float_as_uint(r) ^ __float_as_uint(x)) >> 31 | 1;
    return __uint_as_float(r != 0.0f ? b + towards : b);
  }
};

// Four codes from quotients x * f.
template <bool E4M3>
__device__ __forceinline__ uint32_t pack_codes(const float* x, float f) {
  if constexpr (E4M3) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, v, true);
  } else {
    // x f + 1.5 2^23 + 128 in one rounding: the code, offset by 128, is the sum's low byte
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(__builtin_fmaf(x[i], f, 12583040.0f));
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u);
    const uint32_t b = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
    return a | b;
  }
}

// Sixteen codes.
template <bool E4M3>
__device__ __forceinline__ u4c quantize16(const Quantizer& qz, float* x) {
  u4c v;
  bool decided = false;
  if (qz.lift != 1.0f) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= qz.lift;
  } else if constexpr (!E4M3) {
    uint32_t differ = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = pack_codes<E4M3>(x + 4 * e, qz.inv * (1.0f + 0x1p-22f));
      differ |= v[e] ^ pack_codes<E4M3>(x + 4 * e, qz.inv * (1.0f - 0x1p-22f));
    }
    decided = differ == 0;
  }
  if (!decided) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = qz.quotient(x[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack_codes<E4M3>(x + 4 * e, 1.0f);
  }
  return v;
}

template <int D, bool E4M3, int SH>
__global__ __launch_bounds__(256) void dense_append_kernel(const DenseAppendParams p) {
  constexpr int T = 1 << SH, W = T < 64 ? 64 : T;   // tokens of a block, of a workgroup
  constexpr int kBlocks = W / T, kRow = D + 8, C8 = D / 8;   // (LDS row: 16 bytes of padding)
  __shared__ __attribute__((aligned(16))) uint16_t rows[W * kRow];
  __shared__ uint32_t wave_top[kBlocks][4];
  const int tid = threadIdx.x;
  const int g = blockIdx.y, b = blockIdx.z >> 1, kv = blockIdx.z & 1, bf16 = p.c.bf16;
  const int64_t first = p.pos[b];
  const int m = p.n_new_dev ? min(max(p.n_new_dev[b], 0), p.n_new) : p.n_new;
  const int64_t hi64 = first + m;
  const int lo = (int)min(max(first, (int64_t)0), (int64_t)p.c.capacity);
  const int hi = (int)min(max(hi64, (int64_t)0), (int64_t)p.c.capacity);
  if (lo >= hi) return;
  const int j0 = (lo >> SH) + blockIdx.x * kBlocks, last = (hi - 1) >> SH;
  if (j0 > last) return;
  const int n = min((hi >> SH) - j0, kBlocks);      // finished blocks of the workgroup
  const int64_t head = (int64_t)b * p.c.n_kv + g;
  const int32_t* table = p.c.table + head * p.c.blocks_per_head;
  uint16_t* tail = p.c.tails + (head * 2 + kv) * (2 * T * D);
  const uint16_t* x = p.x[kv] + b * p.xs_b[kv] + g * p.xs_h[kv] - first * p.xs_t[kv];
  const int64_t xt = p.xs_t[kv];
  const int wide = p.wide[kv];

  if (n > 0) {
    int entry[kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) entry[k] = k < n ? table[j0 + k] : -1;
    // a block's rows take whole waves of every pass, so its maximum is one over waves
    constexpr int kPass = 256 / C8;                 // rows of a pass
    us2 most[kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) most[k] = (us2){0, 0};
#pragma unroll
    for (int r0 = 0; r0 < W; r0 += kPass) {
      const int r = r0 + tid / C8, c = (tid % C8) * 8, t = j0 * T + r;
      if (r >= n * T) continue;
      union { u4c v; uint16_t h[8]; } w;
      if (t >= lo) {
        w.v = load8(x + t * xt + c, wide);
      } else {
        const int tr = t & (2 * T - 1);
        if (kv == 0) {
          w.v = *reinterpret_cast<const u4c*>(tail + tr * D + c);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) w.h[e] = tail[tail_value(tr, c + e, D)];
        }
      }
      *reinterpret_cast<u4c*>(rows + r * kRow + c) = w.v;
      // |x| as an integer: the order of the 16-bit patterns is that of the values, with the
      // infinity and NaNs on top
#pragma unroll
      for (int k = 0; k < kBlocks; ++k)
        if (r >> SH == k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            most[k] = __builtin_elementwise_max(most[k], __builtin_bit_cast(us2, w.v[e] & 0x7fff7fffu));
    }
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) {
      uint32_t top = max((uint32_t)most[k][0], (uint32_t)most[k][1]);
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
      if ((tid & 63) == 0) wave_top[k][tid >> 6] = top;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) {
      if (entry[k] < 0 || entry[k] >= p.c.n_blocks) continue;
      const uint32_t top = max(max(wave_top[k][0], wave_top[k][1]), max(wave_top[k][2], wave_top[k][3]));
      const bool bad = top >= (bf16 ? 0x7f80u : 0x7c00u);
      const float scale = bad ? __builtin_nanf("") : from16(top, bf16) / (E4M3 ? 448.0f : 127.0f);
      if (tid == 0) reinterpret_cast<float*>(p.c.scales)[2 * (int64_t)entry[k] + kv] = scale;
      const Quantizer qz(bad ? 0.0f : scale);
      uint8_t* dst = p.c.codes + (int64_t)entry[k] * (2 * T * D) + kv * (T * D);
#pragma unroll
      for (int i0 = 0; i0 < T * D / 16; i0 += 256) {
        const int i = i0 + tid;
        if (T * D / 16 < 256 && i >= T * D / 16) continue;
        const int st = i / D, u = i % D;            // subtile, its 16-byte unit
        const int grp = u >> 6, a = (u >> 4) & 3, l = u & 15;
        float q[16];
        if (kv == 0) {                              // token l, channels grp*64 + 16a ..
          union { u4c v[2]; uint16_t h[16]; } w;
          const uint16_t* s = rows + (k * T + st * 16 + l) * kRow + grp * 64 + a * 16;
          w.v[0] = *reinterpret_cast<const u4c*>(s);
          w.v[1] = *reinterpret_cast<const u4c*>(s + 8);
#pragma unroll
          for (int e = 0; e < 16; ++e) q[e] = from16(w.h[e], bf16);
        } else {                                    // tokens 4a .., channels grp*64 + 16 jt + l
#pragma unroll
          for (int e = 0; e < 16; ++e)
            q[e] = from16(rows[(k * T + st * 16 + 4 * a + (e & 3)) * kRow + grp * 64 + (e >> 2) * 16 + l], bf16);
        }
        if (bad) {
#pragma unroll
          for (int e = 0; e < 16; ++e) q[e] = 0.0f;
        }
        *reinterpret_cast<u4c*>(dst + (int64_t)i * 16) = quantize16<E4M3>(qz, q);
      }
    }
  }
  if (blockIdx.x == 0) {
    const int from = max(lo, (last - 1) << SH);
    if (kv == 0) {                                  // rows, eight channels a thread
#pragma unroll 4
      for (int i = tid; i < (hi - from) * C8; i += 256) {
        const int t = from + i / C8, c = i % C8 * 8;
        *reinterpret_cast<u4c*>(tail + (t & (2 * T - 1)) * D + c) = load8(x + t * xt + c, wide);
      }
    } else {                                        // eight tokens of a channel a thread
      const int t8 = from & ~7, n8 = (hi - t8 + 7) >> 3;
#pragma unroll 2
      for (int i = tid; i < n8 * D; i += 256) {
        const int t = t8 + i / D * 8, c = i % D;
        union { u4c v; uint16_t h[8]; } w;
        uint16_t* to = tail + tail_value(t & (2 * T - 1), c, D);
        if (t >= from && t + 8 <= hi) {
#pragma unroll
          for (int e = 0; e < 8; ++e) w.h[e] = x[(t + e) * xt + c];
          *reinterpret_cast<u4c*>(to) = w.v;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (t + e >= from && t + e < hi) to[e] = x[(t + e) * xt + c];
        }
      }
    }
  }
}

// -------------------------------------------------------------------------------- read
//
// One workgroup per 32 tokens (two subtiles), KV head and keys or values: rows are put together in
// LDS and leave in whole rows, since a thread's 16 bytes of codes lie across four rows (values)
// or 16 threads' across 16 rows (keys).  4130 rows of 2 x 8 heads to fp32: 15 us, 5.6 TB/s (53 us
// when each thread wrote its own values).
template <bool E4M3>
__device__ __forceinline__ float code_value(uint32_t byte) {
  if constexpr (E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
  else return (float)((int)byte - 128);
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void dense_read_kernel(const DenseReadParams p) {
  constexpr int kRow = D + 4;
  __shared__ __attribute__((aligned(16))) float rows[32 * kRow];
  const int g = blockIdx.y, b = blockIdx.z >> 1, kv = blockIdx.z & 1;
  void* out = p.out[kv];
  if (!out) return;
  const int sh = p.c.shift, T = 1 << sh, bf16 = p.c.bf16;
  const int64_t start = p.start[b];
  const int ctx = min(max(p.ctx_len[b], 0), p.c.capacity);
  const int full = ctx & ~(T - 1);
  const int64_t head = (int64_t)b * p.c.n_kv + g;
  const uint16_t* tail = p.c.tails + (head * 2 + kv) * (2 * T * D);
  const int64_t t0 = ((start >> 4) + (int64_t)blockIdx.x * 2) * 16;   // first token
  for (int i = threadIdx.x; i < 2 * D; i += 256) {
    const int st = i / D, u = i % D, grp = u >> 6, a = (u >> 4) & 3, l = u & 15;
    const int64_t ts = t0 + st * 16;
    float q[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) q[e] = 0.0f;
    if (ts >= 0 && ts < full) {
      int entry = p.c.table[head * p.c.blocks_per_head + (ts >> sh)];
      entry = min(max(entry, 0), p.c.n_blocks - 1);
      const float s = reinterpret_cast<const float*>(p.c.scales)[2 * (int64_t)entry + kv];
      union { u4c v; uint8_t c[16]; } w;
      w.v = *reinterpret_cast<const u4c*>(p.c.codes + (int64_t)entry * (2 * T * D) + kv * (T * D) +
                                          ((ts & (T - 1)) >> 4) * (16 * D) + u * 16);
#pragma unroll
      for (int e = 0; e < 16; ++e) q[e] = code_value<E4M3>(w.c[e]) * s;
    } else if (ts >= full && ts < ctx) {
      // (the ring's rows beyond the last token hold anything)
      const int tr = (int)ts & (2 * T - 1);
      if (kv == 0) {
        union { u4c v[2]; uint16_t h[16]; } w;
        const u4c* src = reinterpret_cast<const u4c*>(tail + (tr + l) * D + grp * 64 + a * 16);
        w.v[0] = src[0];
        w.v[1] = src[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) q[e] = ts + l < ctx ? from16(w.h[e], bf16) : 0.0f;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          union { f2c v; uint16_t h[4]; } w;
          w.v = *reinterpret_cast<const f2c*>(tail + tail_value(tr + 4 * a, grp * 64 + j * 16 + l, D));
#pragma unroll
          for (int r = 0; r < 4; ++r) q[4 * j + r] = ts + 4 * a + r < ctx ? from16(w.h[r], bf16) : 0.0f;
        }
      }
    }
    if (kv == 0) {
      float* to = rows + (st * 16 + l) * kRow + grp * 64 + a * 16;
#pragma unroll
      for (int e = 0; e < 16; ++e) to[e] = q[e];
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        rows[(st * 16 + 4 * a + (e & 3)) * kRow + grp * 64 + (e >> 2) * 16 + l] = q[e];
    }
  }
  __syncthreads();
  const int64_t o0 = b * p.os_b[kv] + g * p.os_h[kv] - start * p.os_t[kv];
  constexpr int kFour = D / 4;                      // a thread writes four channels
  for (int i = threadIdx.x; i < 32 * kFour; i += 256) {
    const int64_t t = t0 + i / kFour;
    if (t < start || t >= start + p.n) continue;
    const int c = i % kFour * 4;
    const float* f = rows + i / kFour * kRow + c;
    const int64_t at = o0 + t * p.os_t[kv] + c;
    if (p.out_dtype == STARKV_DT_F32) {
      float* o = static_cast<float*>(out) + at;
      if (p.wide[kv]) {
        *reinterpret_cast<float4*>(o) = *reinterpret_cast<const float4*>(f);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = f[e];
      }
    } else {
      uint16_t* o = static_cast<uint16_t*>(out) + at;
      union { f2c v; uint16_t h[4]; } w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w.h[e] = p.out_dtype == STARKV_DT_BF16 ? to_bf16(f[e]) : to_f16(f[e]);
      if (p.wide[kv]) {
        *reinterpret_cast<f2c*>(o) = w.v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = w.h[e];
      }
    }
  }
}

// ------------------------------------------------------------------------------- evict
//
// One workgroup per (sequence, KV head).  Element k*1024 + thread of the head's blocks stays in
// registers (NPT per thread), so that in-place outputs cannot overtake inputs.  The weight of the
// last block that stays is found by four 8-bit radix passes over order-preserving integer keys;
// ranks come from ballots in index order, which also settles ties by the lower index.
// Bound by its chain of barriers, not by its 16 bytes per block: 7 us for 1024 blocks of 256 heads
// and for 2048 of 32.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.0f);      // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive rank of this thread's flagged elements in index order (element k*1024 + thread).
// counts: 16 * NPT ints of LDS.  Ends with a barrier.
template <int NPT>
__device__ __forceinline__ int ordered_ranks(uint32_t flags, int* counts, int* rank, int tid) {
  const int wave = tid >> 6, lane = tid & 63;
  int below[NPT];
#pragma unroll
  for (int k = 0; k < NPT; ++k) {
    const uint64_t m = __ballot((flags >> k) & 1);
    below[k] = __popcll(m & ((1ull << lane) - 1));
    if (lane == 0) counts[k * 16 + wave] = __popcll(m);
  }
  __syncthreads();
  if (wave == 0) {                                   // exclusive scan of 16*NPT counts
    constexpr int PL = (16 * NPT + 63) / 64;
    int v[PL], sum = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int at = lane * PL + i;
      v[i] = sum;
      sum += at < 16 * NPT ? counts[at] : 0;
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(incl, o);
      if (lane >= o) incl += y;
    }
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const int at = lane * PL + i;
      if (at < 16 * NPT) counts[at] = v[i] + incl - sum;
    }
    if (lane == 63) counts[16 * NPT] = incl;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NPT; ++k) rank[k] = counts[k * 16 + wave] + below[k];
  const int total = counts[16 * NPT];
  __syncthreads();
  return total;
}

template <int NPT>
__global__ __launch_bounds__(1024) void dense_evict_kernel(const DenseEvictParams p, int write_ctx) {
  __shared__ int counts[16 * NPT + 1];
  __shared__ int hist[256];
  __shared__ uint32_t sel_prefix;
  __shared__ int sel_need;
  const int tid = threadIdx.x, b = blockIdx.x / p.n_kv;
  const int J = p.blocks_per_head;
  const int64_t base = (int64_t)blockIdx.x * J;
  const int ctx = min(max(p.ctx_len[b], 0), p.capacity);
  const int n = ctx >> p.shift;
  const int left = n - (n > p.keep ? (n - p.keep) & ~1 : 0);
  if (write_ctx && tid == 0 && blockIdx.x % p.n_kv == 0) p.ctx_out[b] = ctx - ((n - left) << p.shift);

  float w[NPT];
  int entry[NPT];
#pragma unroll
  for (int k = 0; k < NPT; ++k) {
    const int i = k * 1024 + tid;
    w[k] = i < J ? p.weights[base + i] : 0.0f;
    entry[k] = i < J ? p.table[base + i] : 0;
  }
  uint32_t kept = 0;
  if (left == n) {
#pragma unroll
    for (int k = 0; k < NPT; ++k) kept |= (uint32_t)(k * 1024 + tid < n) << k;
  } else {
    uint32_t free = 0;                               // blocks that are chosen by weight
#pragma unroll
    for (int k = 0; k < NPT; ++k) {
      const int i = k * 1024 + tid;
      const bool must = i < p.sink || (i >= n - p.recent && i < n);
      kept |= (uint32_t)must << k;
      free |= (uint32_t)(!must && i < n) << k;
    }
    int need = left - p.sink - p.recent;             // of the free ones; less than there are
    uint32_t prefix = 0;
    if (need > 0) {
      for (int bit = 24; bit >= 0; bit -= 8) {       // the need-th largest key, 8 bits at a time
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NPT; ++k) {
          const uint32_t key = weight_key(w[k]);
          const bool same = bit == 24 || (key >> (bit + 8)) == (prefix >> (bit + 8));
          if (((free >> k) & 1) && same) atomicAdd(&hist[(key >> bit) & 255], 1);
        }
        __syncthreads();
        if (tid < 64) {                              // lane l: bins 255-4l .. 252-4l
          int c[4], sum = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) { c[i] = hist[255 - 4 * tid - i]; sum += c[i]; }
          int incl = sum;
#pragma unroll
          for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(incl, o);
            if (tid >= o) incl += y;
          }
          int above = incl - sum;                    // keys in larger bins
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (above < need && above + c[i] >= need) {
              sel_prefix = prefix | (uint32_t)(255 - 4 * tid - i) << bit;
              sel_need = need - above;
            }
            above += c[i];
          }
        }
        __syncthreads();
        prefix = sel_prefix;
        need = sel_need;
        __syncthreads();
      }
      uint32_t tie = 0;
#pragma unroll
      for (int k = 0; k < NPT; ++k) {
        const uint32_t key = weight_key(w[k]);
        const bool f = (free >> k) & 1;
        kept |= (uint32_t)(f && key > prefix) << k;
        tie |= (uint32_t)(f && key == prefix) << k;
      }
      int rank[NPT];
      ordered_ranks<NPT>(tie, counts, rank, tid);
#pragma unroll
      for (int k = 0; k < NPT; ++k) kept |= (uint32_t)(((tie >> k) & 1) && rank[k] < need) << k;
    }
  }
  // outputs may be in place: every input has arrived before the barriers that follow
#pragma unroll
  for (int k = 0; k < NPT; ++k) asm volatile("" ::"v"(entry[k]), "v"(w[k]));
  int rank[NPT];
  ordered_ranks<NPT>(kept, counts, rank, tid);
#pragma unroll
  for (int k = 0; k < NPT; ++k) {
    const int i = k * 1024 + tid;
    if (i >= J) continue;
    const bool stay = (kept >> k) & 1;
    // kept blocks first, then the others below n in order, then the rest in place
    const int to = i >= n ? i : stay ? rank[k] : left + i - rank[k];
    p.table_out[base + to] = entry[k];
    if (stay) p.weights_out[base + to] = w[k];
    else if (i == n) p.weights_out[base + left] = w[k];
    // zeros behind the unfinished block's entry (which is absent where n == J)
    if (i > left || (i == left && n == J && left < n)) p.weights_out[base + i] = 0.0f;
  }
}

// Lengths of an in-place eviction, once every workgroup has read the old ones.
__global__ void dense_evict_ctx_kernel(const DenseEvictParams p) {
  const int b = blockIdx.x * 64 + threadIdx.x;
  if (b >= p.batch) return;
  const int ctx = min(max(p.ctx_len[b], 0), p.capacity);
  const int n = ctx >> p.shift;
  p.ctx_out[b] = ctx - ((n > p.keep ? (n - p.keep) & ~1 : 0) << p.shift);
}

}  // namespace

namespace {
template <int D, bool E4M3>
void launch_append(const DenseAppendParams& p, dim3 grid, hipStream_t st) {
#define SK_APPEND(SH) hipLaunchKernelGGL((dense_append_kernel<D, E4M3, SH>), grid, dim3(256), 0, st, p)
  if (p.c.shift == 4) SK_APPEND(4);
  else if (p.c.shift == 5) SK_APPEND(5);
  else if (p.c.shift == 6) SK_APPEND(6);
  else SK_APPEND(7);
#undef SK_APPEND
}
}  // namespace

int launch_dense_append(const DenseAppendParams& p, void* stream) {
  const int T = 1 << p.c.shift, per = T < 64 ? 64 / T : 1;   // blocks of a workgroup
  const int64_t touched = ((int64_t)p.n_new + 2 * T - 2) >> p.c.shift;
  const int64_t blocks = touched < p.c.blocks_per_head ? touched : p.c.blocks_per_head;
  const dim3 grid((uint32_t)((blocks + per - 1) / per), p.c.n_kv, p.c.batch * 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p.c.d == 128) {
    if (p.c.e4m3) launch_append<128, true>(p, grid, st);
    else launch_append<128, false>(p, grid, st);
  } else {
    if (p.c.e4m3) launch_append<64, true>(p, grid, st);
    else launch_append<64, false>(p, grid, st);
  }
  return (int)hipGetLastError();
}

int launch_dense_read(const DenseReadParams& p, void* stream) {
  // 16-token subtiles that n rows can touch, two to a workgroup
  const int64_t subs = ((int64_t)p.n + 30) >> 4;
  const dim3 grid((uint32_t)((subs + 1) / 2), p.c.n_kv, p.c.batch * 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p.c.d == 128) {
    if (p.c.e4m3) hipLaunchKernelGGL((dense_read_kernel<128, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((dense_read_kernel<128, false>), grid, dim3(256), 0, st, p);
  } else {
    if (p.c.e4m3) hipLaunchKernelGGL((dense_read_kernel<64, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((dense_read_kernel<64, false>), grid, dim3(256), 0, st, p);
  }
  return (int)hipGetLastError();
}

int launch_dense_evict(const DenseEvictParams& p, void* stream) {
  const dim3 grid(p.batch * p.n_kv);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int in_place = p.ctx_out == p.ctx_len;
  const int per = (p.blocks_per_head + 1023) / 1024;
#define SK_EVICT(NPT) hipLaunchKernelGGL(dense_evict_kernel<NPT>, grid, dim3(1024), 0, st, p, !in_place)
  if (per <= 1) SK_EVICT(1);
  else if (per <= 2) SK_EVICT(2);
  else if (per <= 4) SK_EVICT(4);
  else if (per <= 8) SK_EVICT(8);
  else if (per <= 16) SK_EVICT(16);
  else SK_EVICT(32);
#undef SK_EVICT
  int e = (int)hipGetLastError();
  if (e == 0 && in_place) {
    hipLaunchKernelGGL(dense_evict_ctx_kernel, dim3((p.batch + 63) / 64), dim3(64), 0, st, p);
    e = (int)hipGetLastError();
  }
  return e;
}

}  // namespace starkv
