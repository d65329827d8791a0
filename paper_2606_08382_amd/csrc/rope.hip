// Rotary positions of query and key heads (starkv_rope).
//
// y_p = x_p cos a - x_q sin a, y_q = x_q cos a + x_p sin a for the channel pairs (p, q) of the
// first R channels, a = position * f_j; the rest is copied.  Bound by its bytes, one read and
// one write of every element, as long as the angles cost little: an angle belongs to (token,
// pair) and serves every head, so a thread takes one unit of pairs (16-byte accesses) of a
// token and computes its angles once for two heads.  16384 tokens of 40 heads of 128 in bf16: 60 us,
// 5.6 TB/s.
//
// An angle is position * f / 2 pi in turns, in fp64, minus its nearest integer (exact), and only
// then fp32: at position 2^31 the turn's fraction is still known to 2^-22.  sincospif takes it
// in half turns, so nothing is lost to a reduction by pi.
#include <hip/hip_runtime.h>

#include "dense.h"

namespace starkv {

namespace {

typedef uint32_t u4r __attribute__((ext_vector_type(4)));

template <int DT>
struct Elem;
template <>
struct Elem<STARKV_DT_F16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float load(uint16_t u) {
    return (float)__builtin_bit_cast(_Float16, u);
  }
  static __device__ __forceinline__ uint16_t store(float f) {
    return __builtin_bit_cast(uint16_t, (_Float16)f);
  }
};
template <>
struct Elem<STARKV_DT_BF16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float load(uint16_t u) {
    return __uint_as_float((uint32_t)u << 16);
  }
  static __device__ __forceinline__ uint16_t store(float f) {
    return __builtin_bit_cast(uint16_t, (__bf16)f);
  }
};
template <>
struct Elem<STARKV_DT_F32> {
  typedef uint32_t raw;
  static __device__ __forceinline__ float load(uint32_t u) { return __uint_as_float(u); }
  static __device__ __forceinline__ uint32_t store(float f) { return __float_as_uint(f); }
};

// cos and sin of pair j at this position.
__device__ __forceinline__ void angle(const RopeParams& p, int pos, int j, float* c, float* s) {
  const double t = (double)pos * p.turns[j];
  const float r = (float)(t - __builtin_rint(t));
  sincospif(2.0f * r, s, c);
  *c *= p.gain;
  *s *= p.sine;
}

// Sixteen bytes of a row.  Calls larger than the caches pass them by (336 MB: 60 us against 68);
// the rows of smaller ones stay for what reads them next.
template <bool STREAM>
__device__ __forceinline__ u4r load16(const void* a) {
  const u4r* v = static_cast<const u4r*>(a);
  if constexpr (STREAM) return __builtin_nontemporal_load(v);
  else return *v;
}
template <bool STREAM>
__device__ __forceinline__ void store16(void* a, u4r x) {
  u4r* v = static_cast<u4r*>(a);
  if constexpr (STREAM) __builtin_nontemporal_store(x, v);
  else *v = x;
}

// WIDE: units of E = 16 bytes of pairs (HALF: E channels of either half; INTERLEAVED: E/2
// neighbouring pairs), then of E copied channels.  Otherwise a unit is one pair or one channel.
template <int DT, bool IL, bool WIDE, bool STREAM>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams p) {
  typedef Elem<DT> El;
  typedef typename El::raw raw;
  constexpr int E = WIDE ? 16 / (int)sizeof(raw) : 1;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int u = (int)(id % p.units);
  const int64_t rest = id / p.units;
  const int hg = (int)(rest % p.head_groups);
  const int64_t tok = rest / p.head_groups;
  if (tok >= p.tokens) return;
  const int64_t b = tok / p.n, t = tok % p.n;
  const raw* x = static_cast<const raw*>(p.x) + b * p.xs_b + t * p.xs_t;
  raw* o = static_cast<raw*>(p.out) + b * p.os_b + t * p.os_t;
  const int h0 = hg * p.heads_per_thread, h1 = min(h0 + p.heads_per_thread, p.heads);
  if (u >= p.rot_units) {                    // channels that are not rotated
    const int c = p.rotary + (u - p.rot_units) * E;
    if (p.x == p.out) return;
    for (int h = h0; h < h1; ++h) {
      const raw* a = x + (int64_t)h * p.xs_h + c;
      raw* z = o + (int64_t)h * p.os_h + c;
      if constexpr (WIDE) store16<STREAM>(z, load16<STREAM>(a));
      else *z = *a;
    }
    return;
  }
  const int pos = p.positions[tok];
  constexpr int NP = !WIDE ? 1 : (IL ? E / 2 : E);   // pairs of the unit
  float cs[NP], sn[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) angle(p, pos, u * NP + i, &cs[i], &sn[i]);
  if constexpr (!WIDE) {
    const int c0 = IL ? 2 * u : u, c1 = IL ? 2 * u + 1 : u + p.rotary / 2;
    for (int h = h0; h < h1; ++h) {
      const raw* xr = x + (int64_t)h * p.xs_h;
      raw* orow = o + (int64_t)h * p.os_h;
      const float a = El::load(xr[c0]), e = El::load(xr[c1]);
      orow[c0] = El::store(a * cs[0] - e * sn[0]);
      orow[c1] = El::store(e * cs[0] + a * sn[0]);
    }
  } else if constexpr (IL) {
    union V { u4r v; raw r[E]; };
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
      V a, z;
      a.v = load16<STREAM>(x + (int64_t)h * p.xs_h + u * E);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float e = El::load(a.r[2 * i]), f = El::load(a.r[2 * i + 1]);
        z.r[2 * i] = El::store(e * cs[i] - f * sn[i]);
        z.r[2 * i + 1] = El::store(f * cs[i] + e * sn[i]);
      }
      store16<STREAM>(o + (int64_t)h * p.os_h + u * E, z.v);
    }
  } else {
    union V { u4r v; raw r[E]; };
    const int half = p.rotary / 2;
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
      const raw* xr = x + (int64_t)h * p.xs_h + u * E;
      V a, e, y, z;
      a.v = load16<STREAM>(xr);
      e.v = load16<STREAM>(xr + half);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float f = El::load(a.r[i]), g = El::load(e.r[i]);
        y.r[i] = El::store(f * cs[i] - g * sn[i]);
        z.r[i] = El::store(g * cs[i] + f * sn[i]);
      }
      raw* orow = o + (int64_t)h * p.os_h + u * E;
      store16<STREAM>(orow, y.v);
      store16<STREAM>(orow + half, z.v);
    }
  }
}

template <int DT, bool IL>
void launch(const RopeParams& p, bool wide, dim3 grid, hipStream_t st) {
  if (!wide) hipLaunchKernelGGL((rope_kernel<DT, IL, false, false>), grid, dim3(256), 0, st, p);
  else if (p.streaming) hipLaunchKernelGGL((rope_kernel<DT, IL, true, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((rope_kernel<DT, IL, true, false>), grid, dim3(256), 0, st, p);
}

template <int DT>
void launch_type(const RopeParams& p, bool wide, dim3 grid, hipStream_t st) {
  if (p.interleaved) launch<DT, true>(p, wide, grid, st);
  else launch<DT, false>(p, wide, grid, st);
}

}  // namespace

int launch_rope(const RopeParams& p, bool wide, void* stream) {
  const int64_t threads = p.tokens * p.head_groups * p.units;
  const dim3 grid((uint32_t)((threads + 255) / 256));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p.dtype == STARKV_DT_F32) launch_type<STARKV_DT_F32>(p, wide, grid, st);
  else if (p.dtype == STARKV_DT_BF16) launch_type<STARKV_DT_BF16>(p, wide, grid, st);
  else launch_type<STARKV_DT_F16>(p, wide, grid, st);
  return (int)hipGetLastError();
}

}  // namespace starkv
