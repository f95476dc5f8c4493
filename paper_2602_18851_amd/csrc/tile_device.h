// What the kernels of 8-bit products share: the order of tiles, ranges of loads, ragged edges, waits.
#pragma once

#include "fp8_device.h"

namespace sn_dev {

// Place of tile t: bands of kBand tiles in m, column after column of a band, so that the tiles
// that run at one time on an XCD share few rows of A and of B in its L2.
// 8192^3 of 8-bit floats to bf16: 467 us column by column, 443, 432 and 427 in bands of 16, 8 and 4.
constexpr int kBand = 4;
__device__ __forceinline__ void place(int t, int tiles_m, int tiles_n, int64_t& bm, int64_t& bn) {
  const int band = t / (kBand * tiles_n), first = band * kBand, in = t - first * tiles_n;
  const int rows = min(kBand, tiles_m - first);
  bm = first + in % rows;
  bn = in / rows;
}

// Zeroes the bytes of a 16-byte chunk from byte n on.
__device__ __forceinline__ void keep_chunk(u32x4& q, int n) {
#pragma unroll
  for (int e = 0; e < 4; ++e) q[e] = keep_bytes(q[e], n - 4 * e);
}

// Bytes from a matrix row to the end of the last row of its tile, for the range check of loads:
// the rows there are, up to the 16-byte chunk that holds column k - 1.
__device__ __forceinline__ uint32_t range_bytes(int64_t row, int64_t rows, int tile, int64_t ld, int64_t k) {
  if (row >= rows) return 0;
  const int64_t last = (rows - row < tile ? rows - row : tile) - 1;
  return (uint32_t)(last * ld + ((k + 15) & ~int64_t(15)));
}

// Four neighbouring elements of C, of which n are there.
template <typename TC>
__device__ __forceinline__ void store4(TC* p, const f32x4& v, int n) {
  typedef TC vec __attribute__((ext_vector_type(4)));
  typedef vec vec_any __attribute__((aligned(sizeof(TC))));
  if (n >= 4) {
    *reinterpret_cast<vec_any*>(p) = vec{(TC)v[0], (TC)v[1], (TC)v[2], (TC)v[3]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) p[e] = (TC)v[e];
}

__device__ __forceinline__ void bare_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
// At most N vector-memory operations outstanding and every LDS read complete.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((N >> 4) << 14));
}

}  // namespace sn_dev
