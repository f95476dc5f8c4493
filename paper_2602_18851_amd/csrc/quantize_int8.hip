// Quantiser by rows: a matrix to 8-bit integers with a scale for each row (spectral_quantize_int8).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "entry_util.h"
#include "int8_device.h"
#include "quantize_int8.h"

namespace {

using namespace sn_dev;
using sn::QuantInt8Args;

// LANES lanes take a row, which they hold in registers, 8 values of every 8 LANES in HELD groups, so x is
// read once; rows that are too long for that (HELD 0) are read a second time for their codes.  Bound by memory: 8192 x 8192
// bf16 34-38 us, of inputs that no cache holds 37 (5.4 TB/s; 42 with every quotient checked for ties), 4097 x 3001 float32 12-13.5 us
// (4.6).  Codes stored past the
// caches take 34, but the product that follows reads them.
template <typename T, int LANES, int HELD>
__global__ void __launch_bounds__(256) quantize_int8_kernel(QuantInt8Args a) {
  __shared__ uint32_t wave_max[4];
  const int t = threadIdx.x, l = t % LANES;
  const int64_t room = (a.cols + 15) & ~int64_t(15);  // columns written
  auto row_max = [&](uint32_t m) {
    m = max16(m);
    if constexpr (LANES >= 64) {
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    }
    if constexpr (LANES == 256) {
      __syncthreads();  // the row before has been read
      if ((t & 63) == 0) wave_max[t >> 6] = m;
      __syncthreads();
      m = max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3]));
    }
    return m;
  };
  // the row of a workgroup of LANES 256 is the same for all, so its barriers are met by all
  for (int64_t r = (int64_t)blockIdx.x * (256 / LANES) + t / LANES; r < a.rows;
       r += (int64_t)gridDim.x * (256 / LANES)) {
    const T* x = static_cast<const T*>(a.x) + r * a.ld_x;
    int8_t* codes = a.codes + r * a.ld;
    auto read = [&](Eight<T>& v, int64_t c) {
      if (c < a.cols)
        v.load(x + c, 0, (int)min(a.cols - c, (int64_t)8));
      else
        v.clear();
    };
    auto top = [&](const Eight<T>& v, uint32_t m) {
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, v.magnitude(e));
      return m;
    };
    float scale, inverse;
    if constexpr (HELD > 0) {
      Eight<T> v[HELD];
#pragma unroll
      for (int i = 0; i < HELD; ++i) read(v[i], 8 * (l + LANES * i));
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < HELD; ++i) m = top(v[i], m);
      int8_scale(row_max(m), scale, inverse);
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        const int64_t c = 8 * (l + LANES * i);
        if (c < room) *reinterpret_cast<uint2*>(codes + c) = int8_codes(v[i], c, a.cols, scale, inverse);
      }
    } else {
      uint32_t m = 0;
#pragma unroll 4
      for (int64_t c = 8 * l; c < a.cols; c += 8 * LANES) {
        Eight<T> v;
        read(v, c);
        m = top(v, m);
      }
      int8_scale(row_max(m), scale, inverse);
#pragma unroll 4
      for (int64_t c = 8 * l; c < room; c += 8 * LANES) {
        Eight<T> v;
        read(v, c);
        *reinterpret_cast<uint2*>(codes + c) = int8_codes(v, c, a.cols, scale, inverse);
      }
    }
    if (l == 0) a.scale[r] = scale;
  }
}

template <typename T>
void launch1(const QuantInt8Args& a, hipStream_t st) {
  auto grid = [&](int lanes) {
    return dim3((uint32_t)std::min<int64_t>((a.rows + 256 / lanes - 1) / (256 / lanes), 1 << 20));
  };
  if (a.cols <= 128)
    quantize_int8_kernel<T, 16, 1><<<grid(16), 256, 0, st>>>(a);
  else if (a.cols <= 512)
    quantize_int8_kernel<T, 64, 1><<<grid(64), 256, 0, st>>>(a);
  else if (a.cols <= 2048)
    quantize_int8_kernel<T, 256, 1><<<grid(256), 256, 0, st>>>(a);
  else if (a.cols <= 4096)
    quantize_int8_kernel<T, 256, 2><<<grid(256), 256, 0, st>>>(a);
  else if (a.cols <= 8192)
    quantize_int8_kernel<T, 256, 4><<<grid(256), 256, 0, st>>>(a);
  else
    quantize_int8_kernel<T, 256, 0><<<grid(256), 256, 0, st>>>(a);
}

}  // namespace

namespace sn {

void launch_quantize_int8(const QuantInt8Args& a, bool bf16, hipStream_t st) {
  bf16 ? launch1<__bf16>(a, st) : launch1<float>(a, st);
}

}  // namespace sn

using namespace sn;

extern "C" SN_API int spectral_quantize_int8(const void* x, int64_t rows, int64_t cols, int64_t ld_x, int32_t dtype,
                                             int8_t* codes, int64_t ld, float* scale, void* hip_stream) {
  if (dtype != SN_F32 && dtype != SN_BF16) return refuse(SN_EDTYPE, "x must be SN_F32 or SN_BF16");
  if (rows < 0 || cols < 0) return refuse(SN_EINVAL, "rows and cols must be >= 0");
  constexpr int64_t kMost = int64_t(1) << 40;
  if (rows > kMost || cols > kMost || ld_x > kMost || ld > kMost)
    return refuse(SN_EINVAL, "rows, cols, ld_x and ld must stay below 2^40");
  if (ld_x == 0) ld_x = cols;
  if (ld_x < cols || ld < cols) return refuse(SN_EINVAL, "ld_x and ld must be >= cols");
  if (ld % 16 || !aligned(codes, 16)) return refuse(SN_EINVAL, "code rows must be 16-byte aligned");
  if (rows == 0) return SN_OK;
  if ((cols > 0 && (!x || !codes)) || !scale) return refuse(SN_ENULL, "x, codes and scale must not be NULL");
  if (!aligned(x, dtype == SN_F32 ? 4 : 2) || !aligned(scale, 4))
    return refuse(SN_EINVAL, "x and scale must be aligned to their type");
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = check_stream(st)) return rc;
  launch_quantize_int8({x, rows, cols, ld_x, codes, ld, scale}, dtype == SN_BF16, st);
  return sn::launched("quantise");
}
