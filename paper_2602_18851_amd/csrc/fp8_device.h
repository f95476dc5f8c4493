// 8-bit codes and their scales, shared by the kernels that quantise.
#pragma once

#include "device_util.h"

namespace sn_dev {

// Exponent of the block scale 2^e: the smallest e >= -126 with amax / 2^e <=
// 1.75 * 2^top (448: top 8; 57344: top 15).  amax = f 2^g, 1 <= f < 2: e = g -
// top, one more where f > 1.75.  Adding just less than a quarter of the mantissa's
// range carries into the exponent exactly then.  amax_bits are the bits of a
// non-negative float.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits, int top) {
  const int e = (int)((amax_bits + 0x1fffffu) >> 23) - 127 - top;
  return e < -126 ? -126 : e;
}

// The scale 2^e and the factor 2^-e that divides by it exactly; NaN both where the block
// holds an infinity or a NaN.
__device__ __forceinline__ void block_scale(uint32_t amax_bits, int top, float& scale, float& inverse) {
  const int e = scale_exponent(amax_bits, top);
  const bool bad = amax_bits >= 0x7f800000u;
  scale = __uint_as_float(bad ? 0x7fc00000u : (uint32_t)(127 + e) << 23);
  inverse = __uint_as_float(bad ? 0x7fc00000u : (uint32_t)(127 - e) << 23);
}

// Wide loads and stores at any alignment of the element, which global memory instructions of this
// target take (an address that is not a multiple of 16 costs the second line it touches).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// Eight neighbouring values of a row as they are stored.
template <typename T>
struct Eight {
  static constexpr int W = sizeof(T) / 2;  // 16-byte words
  u32x4 w[W];
  __device__ __forceinline__ float value(int e) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t x = w[0][e >> 1];
      return __uint_as_float(e & 1 ? x & 0xffff0000u : x << 16);
    } else {
      return __uint_as_float(w[e >> 2][e & 3]);
    }
  }
  __device__ __forceinline__ uint32_t magnitude(int e) const { return __float_as_uint(value(e)) & 0x7fffffffu; }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = u32x4{0, 0, 0, 0};
  }
  // Columns c .. c + 7 of a row of n; zeros from n on.
  __device__ __forceinline__ void load(const T* p, int c, int n) {
    if (c + 8 <= n) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j] = *reinterpret_cast<const u32x4_any*>(reinterpret_cast<const char*>(p) + 16 * j);
      return;
    }
    clear();
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (c + e < n) {
        if constexpr (sizeof(T) == 2)
          w[0][e >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, p[e]) << (16 * (e & 1));
        else
          w[e >> 2][e & 3] = __float_as_uint(p[e]);
      }
  }
};

constexpr int format_top(bool e5m2) { return e5m2 ? 15 : 8; }

// Four codes of four values, lowest byte first, rounded to nearest even.
template <bool E5M2>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (E5M2) {
    const int lo = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, lo, true);
  } else {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
  }
}

// Keeps the first n of the four bytes of a word (n <= 0: none).
__device__ __forceinline__ uint32_t keep_bytes(uint32_t w, int n) {
  return n >= 4 ? w : n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u);
}

// Maximum over the 16 lanes of a row of lanes, in every one of them.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
#define SN_ROR(n) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x120 + (n), 0xf, 0xf, false))
  SN_ROR(8);
  SN_ROR(4);
  SN_ROR(2);
  SN_ROR(1);
#undef SN_ROR
  return x;
}

}  // namespace sn_dev
