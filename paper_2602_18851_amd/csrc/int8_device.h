// 8-bit integers with a scale for each row, shared by the kernels that quantise.
#pragma once

#include "fp8_device.h"

namespace sn_dev {

typedef int i32x4 __attribute__((ext_vector_type(4)));  // MFMA int8 operand and 16 x 16 accumulator of one lane

// The scale max|x| / 127, rounded once, 2^-126 at least, and about its reciprocal; NaN and
// zero (so that all codes are zero) where the row holds an infinity or a NaN.  amax_bits
// are the bits of a non-negative float.
__device__ __forceinline__ void int8_scale(uint32_t amax_bits, float& scale, float& inverse) {
  const bool bad = amax_bits >= 0x7f800000u;
  const float s = fmaxf(__uint_as_float(amax_bits) / 127.f, 0x1p-126f);
  scale = bad ? __uint_as_float(0x7fc00000u) : s;
  inverse = bad ? 0.f : 1.f / s;
}

// x / scale rounded to the nearest whole number, ties to even, as if the quotient were exact.
// x * inverse is off by less than 127 * 2^-22, so the first candidate is right or one beside a quotient next to a tie. The
// rest x - q scale is exact: both terms are multiples of 2^(e - 24), 2^e <= scale < 2^(e + 1) (x too, being
// scale / 2 at least where q is not zero), and it stays below 2^e.
__device__ __forceinline__ int int8_code(float x, float scale, float inverse) {
  const float q = rintf(x * inverse);
  const float rest = 2.f * fmaf(-q, scale, x), off = fabsf(rest);
  const int i = (int)q;
  const bool next = off > scale || (off == scale && (i & 1));
  return i + (next ? (rest > 0.f ? 1 : -1) : 0);
}

__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  const uint32_t lo = __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x0c0c0400u);
  return lo | hi << 16;
}

// Codes of columns c .. c + 7 of a row of n values; zeros from n on.  A product with the scale's reciprocal that is 2^-13
// away from every tie (as all of a wave's are in nine cases of ten) is on the right side of it; added to 1.5 2^23,
// it rounds to a whole number in the low bits.
template <typename T>
__device__ __forceinline__ uint2 int8_codes(const Eight<T>& v, int64_t c, int64_t n, float scale, float inverse) {
  constexpr float kRound = 12582912.f;
  uint32_t u[8];
  float off = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = inverse == 0.f ? 0.f : v.value(e) * inverse, r = t + kRound;
    u[e] = __float_as_uint(r);
    off = fmaxf(off, fabsf(t - (r - kRound)));
  }
  if (__ballot(off > 0.5f - 0x1p-13f)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = inverse == 0.f ? 0u : (uint32_t)int8_code(v.value(e), scale, inverse);
  }
  const uint2 w = make_uint2(pack4((int)u[0], (int)u[1], (int)u[2], (int)u[3]), pack4((int)u[4], (int)u[5], (int)u[6], (int)u[7]));
  if (c + 8 <= n) return w;
  return make_uint2(keep_bytes(w.x, (int)(n - c)), keep_bytes(w.y, (int)(n - c) - 4));
}

}  // namespace sn_dev
