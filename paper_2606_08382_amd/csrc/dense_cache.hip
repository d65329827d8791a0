// The 8-bit cache of an uncompressed layer: append, read-back and eviction.
#include <hip/hip_runtime.h>

#include "dense.h"

namespace starkv {

namespace {

typedef uint32_t u4c __attribute__((ext_vector_type(4)));
typedef float f2c __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float from16(uint32_t u, int bf16) {
  return bf16 ? __uint_as_float(u << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)u);
}
__device__ __forceinline__ uint16_t to_f16(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// Element offsets of (row, channel) inside a (sequence, KV head)'s 16-bit tail planes.
__device__ __forceinline__ int tail_value(int row, int ch, int d) {
  return ((row >> 4) * d + ch) * 16 + (row & 15);
}

// ------------------------------------------------------------------------------ append
//
// One workgroup per block that the new tokens touch, KV head and keys or values.  A block
// that they finish is gathered into LDS (its earlier tokens from the 16-bit tail), its
// absolute maximum taken on the bit patterns, and its codes written in the order that the
// attention's matrix operands take (see the header).  The first workgroup also moves the new
// tokens of the last two blocks into the tail: it is the only one that reads the tail, and it
// does so before it writes.
//
// Codes are RN(x / s) without a second rounding: the fp32 quotient, less than one unit in the
// last place off, is moved to an odd significand on the true quotient's side unless it is
// exact (the sign of the residual x - q s decides, and fma gives that sign exactly).  No border
// between two codes has an odd 24-bit significand, so rounding the odd value rounds the quotient.
// Scales below 2^-60 and their rows are multiplied by 2^100 first, so that the residual does
// not underflow.
struct Quantizer {
  float lift, s, inv;
  __device__ __forceinline__ Quantizer(float scale) {
    lift = scale < 0x1p-60f ? 0x1p100f : 1.0f;
    s = scale * lift;
    inv = s > 0.0f ? 1.0f / s : 0.0f;
  }
  __device__ __forceinline__ float quotient(float x) const {
    x *= lift;
    float q = x * inv;
    q = __builtin_fmaf(__builtin_fmaf(-q, s, x), inv, q);
    const float r = __builtin_fmaf(-q, s, x);
    const uint32_t u = __float_as_uint(q);
    const bool out = (r > 0.0f) == (x > 0.0f);        // away from zero
    const uint32_t odd = out ? u + 1 : u - 1;
    return r != 0.0f && !(u & 1) && q != 0.0f ? __uint_as_float(odd) : q;
  }
};

template <bool E4M3>
__device__ __forceinline__ uint32_t pack_codes(const float* q) {
  if constexpr (E4M3) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], v, true);
  } else {
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = (int)__builtin_rintf(fminf(fmaxf(q[i], -127.0f), 127.0f)) + 128;
      v |= (uint32_t)c << (8 * i);
    }
    return v;
  }
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void dense_append_kernel(const DenseAppendParams p) {
  constexpr int kRow = D + 8;                       // LDS row: 16 bytes of padding
  __shared__ __attribute__((aligned(16))) uint16_t rows[128 * kRow];
  __shared__ uint32_t wave_top[4];
  const int tid = threadIdx.x;
  const int g = blockIdx.y, b = blockIdx.z >> 1, kv = blockIdx.z & 1;
  const int sh = p.c.shift, T = 1 << sh, bf16 = p.c.bf16;
  const int64_t first = p.pos[b];
  const int m = p.n_new_dev ? min(max(p.n_new_dev[b], 0), p.n_new) : p.n_new;
  const int64_t hi64 = first + m;
  const int lo = (int)min(max(first, (int64_t)0), (int64_t)p.c.capacity);
  const int hi = (int)min(max(hi64, (int64_t)0), (int64_t)p.c.capacity);
  if (lo >= hi) return;
  const int j = (lo >> sh) + blockIdx.x, last = (hi - 1) >> sh;
  if (j > last) return;
  const int64_t head = (int64_t)b * p.c.n_kv + g;
  uint16_t* tail = p.c.tails + (head * 2 + kv) * (2 * T * D);
  const uint16_t* x = p.x[kv] + b * p.xs_b[kv] + g * p.xs_h[kv] - first * p.xs_t[kv];
  const int64_t xt = p.xs_t[kv];
  const int wide = p.wide[kv];

  if (hi >= (j + 1) << sh) {                        // the block is finished
    uint32_t top = 0;
    constexpr int C8 = D / 8;
    for (int i = tid; i < T * C8; i += 256) {
      const int r = i / C8, c = (i % C8) * 8, t = (j << sh) + r;
      union { u4c v; uint16_t h[8]; } w;
      if (t >= lo) {
        const uint16_t* a = x + t * xt + c;
        if (wide) {
          w.v = *reinterpret_cast<const u4c*>(a);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) w.h[e] = a[e];
        }
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
      for (int e = 0; e < 8; ++e) top = max(top, (uint32_t)(w.h[e] & 0x7fff));
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
    top = max(max(wave_top[0], wave_top[1]), max(wave_top[2], wave_top[3]));
    const bool bad = top >= (bf16 ? 0x7f80u : 0x7c00u);
    const float scale = bad ? __builtin_nanf("") : from16(top, bf16) / (E4M3 ? 448.0f : 127.0f);
    const int entry = p.c.table[head * p.c.blocks_per_head + j];
    if (entry >= 0 && entry < p.c.n_blocks) {
      if (tid == 0) reinterpret_cast<float*>(p.c.scales)[2 * (int64_t)entry + kv] = scale;
      const Quantizer qz(bad ? 0.0f : scale);
      uint8_t* dst = p.c.codes + (int64_t)entry * (2 * T * D) + kv * (T * D);
      for (int i = tid; i < T * D / 16; i += 256) {
        const int st = i / D, u = i % D;            // subtile, its 16-byte unit
        const int grp = u >> 6, a = (u >> 4) & 3, l = u & 15;
        float q[16];
        if (kv == 0) {                              // token l, channels grp*64 + 16a ..
          union { u4c v[2]; uint16_t h[16]; } w;
          const uint16_t* s = rows + (st * 16 + l) * kRow + grp * 64 + a * 16;
          w.v[0] = *reinterpret_cast<const u4c*>(s);
          w.v[1] = *reinterpret_cast<const u4c*>(s + 8);
#pragma unroll
          for (int e = 0; e < 16; ++e) q[e] = from16(w.h[e], bf16);
        } else {                                    // tokens 4a .., channels grp*64 + 16 jt + l
#pragma unroll
          for (int e = 0; e < 16; ++e)
            q[e] = from16(rows[(st * 16 + 4 * a + (e & 3)) * kRow + grp * 64 + (e >> 2) * 16 + l], bf16);
        }
        union { u4c v; uint32_t w[4]; } z;
#pragma unroll
        for (int e = 0; e < 16; ++e) q[e] = bad ? 0.0f : qz.quotient(q[e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) z.w[e] = pack_codes<E4M3>(q + 4 * e);
        *reinterpret_cast<u4c*>(dst + (int64_t)i * 16) = z.v;
      }
    }
  }
  if (blockIdx.x == 0) {
    const int from = max(lo, (last - 1) << sh);
    for (int i = tid; i < (hi - from) * D; i += 256) {
      const int t = from + i / D, c = i % D, tr = t & (2 * T - 1);
      tail[kv == 0 ? tr * D + c : tail_value(tr, c, D)] = x[t * xt + c];
    }
  }
}

// -------------------------------------------------------------------------------- read
//
// One workgroup per four 16-token subtiles of the requested rows, KV head and keys or values;
// a thread takes a 16-byte unit of codes.
template <int D, bool E4M3>
__device__ __forceinline__ float code_value(uint32_t byte) {
  if constexpr (E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
  else return (float)((int)byte - 128);
}

__device__ __forceinline__ void store_as(void* out, int64_t at, float f, int dtype) {
  if (dtype == STARKV_DT_F32) static_cast<float*>(out)[at] = f;
  else static_cast<uint16_t*>(out)[at] = dtype == STARKV_DT_BF16 ? to_bf16(f) : to_f16(f);
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void dense_read_kernel(const DenseReadParams p) {
  const int g = blockIdx.y, b = blockIdx.z >> 1, kv = blockIdx.z & 1;
  void* out = p.out[kv];
  if (!out) return;
  const int sh = p.c.shift, T = 1 << sh, bf16 = p.c.bf16;
  const int64_t start = p.start[b];
  const int ctx = min(max(p.ctx_len[b], 0), p.c.capacity);
  const int full = ctx & ~(T - 1);
  const int64_t head = (int64_t)b * p.c.n_kv + g;
  const uint16_t* tail = p.c.tails + (head * 2 + kv) * (2 * T * D);
  const int64_t o0 = b * p.os_b[kv] + g * p.os_h[kv] - start * p.os_t[kv];
  const int64_t ot = p.os_t[kv];
  const int64_t s0 = (start >> 4) + (int64_t)blockIdx.x * 4;
  for (int i = threadIdx.x; i < 4 * D; i += 256) {
    const int64_t t0 = (s0 + i / D) * 16;           // first token of the subtile
    const int u = i % D, grp = u >> 6, a = (u >> 4) & 3, l = u & 15;
    float q[16];
    if (t0 >= 0 && t0 < full) {
      int entry = p.c.table[head * p.c.blocks_per_head + (t0 >> sh)];
      entry = min(max(entry, 0), p.c.n_blocks - 1);
      const float s = reinterpret_cast<const float*>(p.c.scales)[2 * (int64_t)entry + kv];
      const uint8_t* src = p.c.codes + (int64_t)entry * (2 * T * D) + kv * (T * D) +
                           ((t0 & (T - 1)) >> 4) * (16 * D) + u * 16;
      union { u4c v; uint8_t c[16]; } w;
      w.v = *reinterpret_cast<const u4c*>(src);
#pragma unroll
      for (int e = 0; e < 16; ++e) q[e] = code_value<D, E4M3>(w.c[e]) * s;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t t = t0 + (kv == 0 ? l : 4 * a + (e & 3));
      const int c = grp * 64 + (kv == 0 ? 16 * a + e : (e >> 2) * 16 + l);
      if (t < start || t >= start + p.n) continue;
      float f = 0.0f;
      if (t >= 0 && t < ctx) {
        if (t < full) {
          f = q[e];
        } else {
          const int tr = (int)t & (2 * T - 1);
          f = from16(tail[kv == 0 ? tr * D + c : tail_value(tr, c, D)], bf16);
        }
      }
      store_as(out, o0 + t * ot + c, f, p.out_dtype);
    }
  }
}

// ------------------------------------------------------------------------------- evict
//
// One workgroup per (sequence, KV head).  Element k*1024 + thread of the head's blocks stays in
// registers (NPT per thread), so that in-place outputs cannot overtake inputs.  The weight of the
// last block that stays is found by four 8-bit radix passes over order-preserving integer keys;
// ranks come from ballots in index order, which also settles ties by the lower index.
// Bound by its chain of barriers, not by its 16 bytes per block.
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

int launch_dense_append(const DenseAppendParams& p, void* stream) {
  const int T = 1 << p.c.shift;
  const int64_t touched = ((int64_t)p.n_new + 2 * T - 2) >> p.c.shift;
  const dim3 grid((uint32_t)(touched < p.c.blocks_per_head ? touched : p.c.blocks_per_head),
                  p.c.n_kv, p.c.batch * 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p.c.d == 128) {
    if (p.c.e4m3) hipLaunchKernelGGL((dense_append_kernel<128, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((dense_append_kernel<128, false>), grid, dim3(256), 0, st, p);
  } else {
    if (p.c.e4m3) hipLaunchKernelGGL((dense_append_kernel<64, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((dense_append_kernel<64, false>), grid, dim3(256), 0, st, p);
  }
  return (int)hipGetLastError();
}

int launch_dense_read(const DenseReadParams& p, void* stream) {
  // 16-token subtiles that n rows can touch, four to a workgroup
  const int64_t subs = ((int64_t)p.n + 30) >> 4;
  const dim3 grid((uint32_t)((subs + 3) / 4), p.c.n_kv, p.c.batch * 2);
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
