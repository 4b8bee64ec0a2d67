// Device helpers of the kernels that work on groups of eight consecutive
// columns: loads and stores of a group, the dropout mask of a group, scale and
// conversion of a group to 8-bit floats.
#pragma once
#include "layup_internal.h"

namespace layup {

// A group of eight elements as it lies in memory.  The vector accesses carry
// the alignment of one element: gfx950 takes 128-bit global accesses at any
// address, so rows of odd length need no code of their own.
template <class T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
  typedef u32x4 V __attribute__((aligned(2)));
  u32x4 v;
  __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const V*>(p); }
  // v's elements k, k + 1, ... and zeros behind them, 0 < k < 8
  __device__ __forceinline__ void drop_front(int k) {
    if (k & 4) v = u32x4{v[2], v[3], 0, 0};
    if (k & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (k & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  }
  __device__ __forceinline__ void load_some(const bf16_t* p, int n) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) v[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
  }
  __device__ __forceinline__ void zero() { v = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int e) const {
    return __builtin_bit_cast(float, e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
  static __device__ __forceinline__ float round(float x) { return bf2f(f2bf(x)); }
  static __device__ __forceinline__ void store(bf16_t* p, const float (&f)[8]) {
    *reinterpret_cast<V*>(p) = u32x4{pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]), pack_bf2(f[4], f[5]), pack_bf2(f[6], f[7])};
  }
  static __device__ __forceinline__ void store_part(bf16_t* p, const float (&f)[8], int n) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = f2bf(f[e]);
  }
};
template <>
struct Raw8<float> {
  typedef f32x4 V __attribute__((aligned(4)));
  f32x4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *reinterpret_cast<const V*>(p);
    hi = *reinterpret_cast<const V*>(p + 4);
  }
  __device__ __forceinline__ void drop_front(int k) {
    const f32x4 z{0.f, 0.f, 0.f, 0.f};
    if (k & 4) lo = hi, hi = z;
    if (k & 2) lo = f32x4{lo[2], lo[3], hi[0], hi[1]}, hi = f32x4{hi[2], hi[3], 0.f, 0.f};
    if (k & 1) lo = f32x4{lo[1], lo[2], lo[3], hi[0]}, hi = f32x4{hi[1], hi[2], hi[3], 0.f};
  }
  __device__ __forceinline__ void load_some(const float* p, int n) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) {
        if (e < 4) lo[e] = p[e];
        else hi[e - 4] = p[e];
      }
  }
  __device__ __forceinline__ void zero() { lo = hi = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? lo[e] : hi[e - 4]; }
  static __device__ __forceinline__ float round(float x) { return x; }
  static __device__ __forceinline__ void store(float* p, const float (&f)[8]) {
    *reinterpret_cast<V*>(p) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<V*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
  }
  static __device__ __forceinline__ void store_part(float* p, const float (&f)[8], int n) {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < n) p[e] = f[e];
  }
};

// Columns c .. c + 7 of a row of d; behind its end zeros.  The group that the
// end cuts is loaded as the row's last eight elements, like any other, and
// shifted down by finish_group once all loads of a thread are on their way
// (loads element by element, or a shift behind each load, cost a round trip to
// memory each: 1003 x 1237 forward 11 us, now 7).  WHOLE: d is a multiple of 8.
template <bool WHOLE = false, class T>
__device__ __forceinline__ void load_group(Raw8<T>& r, const T* row, int64_t c, int64_t d) {
  if (c < d && (WHOLE || d >= 8)) r.load(row + (WHOLE || c + 8 <= d ? c : d - 8));
  else r.zero();
}
template <bool WHOLE = false, class T>
__device__ __forceinline__ void finish_group(Raw8<T>& r, const T* row, int64_t c, int64_t d) {
  if constexpr (!WHOLE) {
    if (d < 8) {
      if (c == 0) r.load_some(row, (int)d);
    } else if (c < d && c + 8 > d) {
      r.drop_front((int)(c + 8 - d));
    }
  }
}
// Stores around the caches are not used: alone they gain (8192 x 768 forward and
// backward 45 -> 43 us, an 8192 x 2048 quantiser 14.9 -> 12.9), but whoever reads
// the result next pays for it (a linear layer's operands and products, 8192 x
// 4096 x 1024: 192 -> 216).
template <bool WHOLE = false, class T>
__device__ __forceinline__ void store_group(T* p, const float (&f)[8], int64_t n) {
  if (WHOLE || n >= 8) Raw8<T>::store(p, f);
  else Raw8<T>::store_part(p, f, (int)n);
}

// Philox4x32-10: two 32 x 32 -> 64 products a round.
__device__ __forceinline__ u32x4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

__device__ __forceinline__ uint64_t mask_offset(const Mask& K) { return K.offset + (K.offset_dev ? *K.offset_dev : 0); }

// Dropout of columns 8 group .. 8 group + 7 of a row.
__device__ __forceinline__ void drop_group(float (&f)[8], uint32_t group, uint32_t row, const Mask& K, uint64_t offset) {
  const u32x4 w = philox(group, row, (uint32_t)offset, (uint32_t)(offset >> 32), K.k0, K.k1);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // the 16 bits in the high half, against the threshold there (the low bits
    // of an odd column's word do not change the comparison)
    const uint32_t u = e & 1 ? w[e >> 1] : w[e >> 1] << 16;
    f[e] = u >= K.thr ? f[e] * K.scale : 0.f;
  }
}

// ------------------------------------------------------------- reductions
// Exchanges within a wave without LDS: lane l takes the value of lane l ^ 1,
// l ^ 2 (within four lanes), 7 - l (of eight) and 15 - l (of sixteen).  After
// the steps before, each of these lanes holds the sum (maximum) of the other
// half of the group.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_MIRROR8 = 0x141, DPP_MIRROR16 = 0x140;
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, v))); }

// Sum over groups of G = 16, 32 or 64 lanes; every lane gets the same bits.
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp<DPP_XOR1>(v);
  v += dpp<DPP_XOR2>(v);
  v += dpp<DPP_MIRROR8>(v);
  v += dpp<DPP_MIRROR16>(v);
  if constexpr (G >= 32) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1];
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  if constexpr (G >= 64) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1];
    v = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  }
  return v;
}
// Maximum over groups of 16 lanes.
__device__ __forceinline__ uint32_t lanes16_max(uint32_t v) {
  v = max(v, dpp<DPP_XOR1>(v));
  v = max(v, dpp<DPP_XOR2>(v));
  v = max(v, dpp<DPP_MIRROR8>(v));
  return max(v, dpp<DPP_MIRROR16>(v));
}

// ------------------------------------------------------------ 8-bit floats
// |f| for the scale of a block: what is not finite does not count.
__device__ __forceinline__ uint32_t finite_bits(float f) {
  const uint32_t a = __builtin_bit_cast(uint32_t, f) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}

// Exponent byte of a block whose largest magnitude has the bits `amax` (as an
// integer, magnitudes order like floats): amax = m 2^E and the format's
// largest value is 1.75 2^TOP, so the scale is 2^(E - TOP), twice that where
// m > 1.75.  A subnormal amax has E < -126, which the clamp covers.
template <int TOP>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if (amax == 0) return 127;
  const int b = (int)(amax >> 23) - TOP + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(b, 1);
}
// 2^-(byte - 127)
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// Eight values times inv in 8 bits, round to nearest even; TOP 8: E4M3, 15:
// E5M2.  Scaled finite values are within the format; the rest becomes NaN.
template <int TOP>
__device__ __forceinline__ u32x2 to_fp8(const float (&f)[8], float inv) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __builtin_isfinite(f[e]) ? f[e] * inv : __builtin_nanf("");
  u32x2 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = 0;
    if constexpr (TOP == 8) {
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w, true);
    } else {
      w = __builtin_amdgcn_cvt_pk_bf8_f32(v[4 * h], v[4 * h + 1], w, false);
      w = __builtin_amdgcn_cvt_pk_bf8_f32(v[4 * h + 2], v[4 * h + 3], w, true);
    }
    o[h] = (uint32_t)w;
  }
  return o;
}

}  // namespace layup
