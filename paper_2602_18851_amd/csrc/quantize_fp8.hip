// Block quantiser: a matrix to 8-bit codes with a power-of-two scale for each block of 128, in either
// direction or both from one reading (spectral_quantize_fp8).
//
// A block's scale is the smallest 2^e, e >= -126, with max |x| / 2^e <= R.
// Dividing by it is exact, so a code is x / 2^e rounded once, and the codes do
// not depend on how the quotient is formed.  Against scales max |x| / R, the
// codes lose range at the small end (at most one octave), not digits.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "entry_util.h"
#include "fp8_device.h"
#include "quantize_fp8.h"

namespace {

using namespace sn_dev;
using sn::QuantArgs;

// One workgroup takes a 128 x 128 tile: thread t holds rows 8 (t / 16) .. + 7
// of columns 8 (t % 16) .. + 7 in registers, so x is read once for both
// directions: a row block's maximum lies in 16 neighbouring lanes, a column
// block's in the 16 row groups.  Codes of the transpose go through LDS, 8 bytes
// (8 rows of a column) at a time, to leave as 16-byte chunks of 128-byte rows.
// In LDS a column's 16 slots of 8 bytes are permuted by the column group, so
// that the 16 lanes of a row group write to different banks.  Bound by memory:
// 8192 x 8192 bf16 by rows 34 us (5.9 TB/s; 41 with the values held as float),
// both ways 48 (5.6), float32 by tiles both ways 80 (5.0), 4097 x 3001 float32 both ways 17 (4.4; 29 with
// rows of odd alignment read one element at a time).
template <typename T, bool E5M2, bool TILES, bool ROW, bool COL>
__global__ void __launch_bounds__(256, 4) quantize_kernel(QuantArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t tcodes[COL ? 128 * 128 : 16];
  __shared__ uint32_t wave_max[4][128];
  __shared__ __attribute__((aligned(16))) float col_inv[128];
  const int t = threadIdx.x, cg = t & 15, rg = t >> 4, wv = t >> 6;
  const int64_t tr = blockIdx.x / a.tiles_c, tc = blockIdx.x % a.tiles_c;
  const int64_t r0 = tr * 128, c0 = tc * 128;
  const int nr = (int)(a.rows - r0 < 128 ? a.rows - r0 : 128);  // rows and columns of this tile
  const int nc = (int)(a.cols - c0 < 128 ? a.cols - c0 : 128);
  const int rl = 8 * rg, cl = 8 * cg;

  Eight<T> v[8];
  const T* src = static_cast<const T*>(a.x) + r0 * a.ld_x + c0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (rl + i < nr) {
      v[i].load(src + (rl + i) * a.ld_x + cl, cl, nc);
    } else {
      v[i].clear();
    }
  }

  // maxima of the bits of |x|: an infinity, and a NaN above it, stay
  constexpr int TOP = format_top(E5M2);
  float rinv[8];  // factor of each of this thread's rows
  if constexpr (TILES) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, v[i].magnitude(e));
    m = max16(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((t & 63) == 0) wave_max[0][wv] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) m = max(m, wave_max[0][w]);
    float s, inv;
    block_scale(m, TOP, s, inv);
    if (t == 0) {
      if (ROW) a.row_scale[tc * ((a.rows + 127) / 128) + tr] = s;
      if (COL) a.col_scale[tr * a.tiles_c + tc] = s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) rinv[i] = inv;
  } else if constexpr (ROW) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, v[i].magnitude(e));
      float s;
      block_scale(max16(m), TOP, s, rinv[i]);
      if (cg == i && rl + i < nr) a.row_scale[tc * a.rows + r0 + rl + i] = s;
    }
  }

  if constexpr (ROW) {
    const int room = (nc + 15) & ~15;  // columns written: zeros from nc on
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint2 w = make_uint2(
          encode4<E5M2>(v[i].value(0) * rinv[i], v[i].value(1) * rinv[i], v[i].value(2) * rinv[i], v[i].value(3) * rinv[i]),
          encode4<E5M2>(v[i].value(4) * rinv[i], v[i].value(5) * rinv[i], v[i].value(6) * rinv[i], v[i].value(7) * rinv[i]));
      if (cl + 8 > nc) w = make_uint2(keep_bytes(w.x, nc - cl), keep_bytes(w.y, nc - cl - 4));
      if (rl + i < nr && cl < room) *reinterpret_cast<uint2*>(a.row_codes + (r0 + rl + i) * a.ld_row + c0 + cl) = w;
    }
  }

  if constexpr (COL) {
    __builtin_amdgcn_sched_barrier(0);  // the codes by rows first: fewer registers, more waves
    if constexpr (!TILES) {
      uint32_t m[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m[e] = max(m[e], v[i].magnitude(e));
        m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], 16));
        m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], 32));
      }
      if ((t & 63) < 16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) wave_max[wv][cl + e] = m[e];
      }
      __syncthreads();
      if (t < 128) {
        float s, inv;
        block_scale(max(max(wave_max[0][t], wave_max[1][t]), max(wave_max[2][t], wave_max[3][t])), TOP, s, inv);
        col_inv[t] = inv;
        if (t < nc) a.col_scale[tr * a.cols + c0 + t] = s;
      }
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = v[i].value(e) * (TILES ? rinv[i] : col_inv[cl + e]);
      uint2 w = make_uint2(encode4<E5M2>(f[0], f[1], f[2], f[3]), encode4<E5M2>(f[4], f[5], f[6], f[7]));
      if (rl + 8 > nr) w = make_uint2(keep_bytes(w.x, nr - rl), keep_bytes(w.y, nr - rl - 4));
      *reinterpret_cast<uint2*>(tcodes + 128 * (cl + e) + 8 * (rg ^ cg)) = w;
    }
    __syncthreads();
    const int part = t & 7;  // 16 rows of a column
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = (t >> 3) + 32 * j;
      const uint2 lo = *reinterpret_cast<const uint2*>(tcodes + 128 * c + 8 * ((2 * part) ^ (c >> 3)));
      const uint2 hi = *reinterpret_cast<const uint2*>(tcodes + 128 * c + 8 * ((2 * part + 1) ^ (c >> 3)));
      if (c < nc && 16 * part < nr)  // zeros from row nr on
        *reinterpret_cast<u32x4*>(a.col_codes + (c0 + c) * a.ld_col + r0 + 16 * part) =
            u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
}

template <typename T, bool E5M2, bool TILES>
void launch3(const QuantArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)(((a.rows + 127) / 128) * a.tiles_c));
  if (a.row_codes && a.col_codes)
    quantize_kernel<T, E5M2, TILES, true, true><<<grid, 256, 0, st>>>(a);
  else if (a.row_codes)
    quantize_kernel<T, E5M2, TILES, true, false><<<grid, 256, 0, st>>>(a);
  else
    quantize_kernel<T, E5M2, TILES, false, true><<<grid, 256, 0, st>>>(a);
}

template <typename T>
void launch1(const QuantArgs& a, bool e5m2, bool tiles, hipStream_t st) {
  if (e5m2)
    tiles ? launch3<T, true, true>(a, st) : launch3<T, true, false>(a, st);
  else
    tiles ? launch3<T, false, true>(a, st) : launch3<T, false, false>(a, st);
}

}  // namespace

namespace sn {

void launch_quantize(QuantArgs a, bool bf16, bool e5m2, bool tiles, hipStream_t st) {
  a.tiles_c = (int32_t)((a.cols + 127) / 128);
  bf16 ? launch1<__bf16>(a, e5m2, tiles, st) : launch1<float>(a, e5m2, tiles, st);
}

}  // namespace sn

using namespace sn;

extern "C" SN_API int spectral_quantize_fp8(const void* x, int64_t rows, int64_t cols, int64_t ld_x, int32_t dtype,
                                            int32_t format, int32_t tiles, uint8_t* row_codes, int64_t ld_row,
                                            float* row_scale, uint8_t* col_codes, int64_t ld_col, float* col_scale,
                                            void* hip_stream) {
  if (dtype != SN_F32 && dtype != SN_BF16) return refuse(SN_EDTYPE, "x must be SN_F32 or SN_BF16");
  if (format != SN_E4M3 && format != SN_E5M2) return refuse(SN_EDTYPE, "format must be SN_E4M3 or SN_E5M2");
  if (tiles != 0 && tiles != 1) return refuse(SN_EINVAL, "tiles must be 0 or 1");
  if (rows < 0 || cols < 0) return refuse(SN_EINVAL, "rows and cols must be >= 0");
  if (ld_x == 0) ld_x = cols;
  if (ld_x < cols) return refuse(SN_EINVAL, "ld_x must be >= cols");
  if (!row_codes && !col_codes) return refuse(SN_ENULL, "row_codes and col_codes are both NULL");
  if ((row_codes && ld_row < cols) || (col_codes && ld_col < rows))
    return refuse(SN_EINVAL, "ld_row must be >= cols and ld_col >= rows");
  if ((row_codes && (ld_row % 16 || !aligned(row_codes, 16))) || (col_codes && (ld_col % 16 || !aligned(col_codes, 16))))
    return refuse(SN_EINVAL, "code rows must be 16-byte aligned");
  if (rows == 0 || cols == 0) return SN_OK;
  if (!x || (row_codes && !row_scale) || (col_codes && !col_scale))
    return refuse(SN_ENULL, "x and the scales of the requested codes must not be NULL");
  if (!aligned(x, dtype == SN_F32 ? 4 : 2) || !aligned(row_scale, 4) || !aligned(col_scale, 4))
    return refuse(SN_EINVAL, "x and the scales must be aligned to their type");
  if (rows > (int64_t(1) << 40) || cols > (int64_t(1) << 40) || ld_x > (int64_t(1) << 40) ||
      ((rows + 127) / 128) * ((cols + 127) / 128) >= (int64_t(1) << 24))
    return refuse(SN_EINVAL, "rows x cols must stay below 2^24 tiles of 128 x 128");
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = check_stream(st)) return rc;
  QuantArgs a{};
  a.x = x;
  a.rows = rows;
  a.cols = cols;
  a.ld_x = ld_x;
  a.row_codes = row_codes;
  a.ld_row = ld_row;
  a.row_scale = row_scale;
  a.col_codes = col_codes;
  a.ld_col = ld_col;
  a.col_scale = col_scale;
  launch_quantize(a, dtype == SN_BF16, format == SN_E5M2, tiles != 0, st);
  return launched("quantise");
}
