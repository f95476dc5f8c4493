// Internal interface of the quantiser by rows (quantize_int8.hip), which the
// products run for a plain operand.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace sn {

struct QuantInt8Args {
  const void* x;
  int64_t rows, cols, ld_x;
  int8_t* codes;
  int64_t ld;
  float* scale;  // [rows]
};

// Queues the kernel (rows, cols >= 1; arguments checked by the caller).
void launch_quantize_int8(const QuantInt8Args& a, bool bf16, hipStream_t st);

}  // namespace sn
