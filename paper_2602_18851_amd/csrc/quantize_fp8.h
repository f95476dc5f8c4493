// Internal interface of the block quantiser (quantize_fp8.hip), which the
// products run for a plain operand.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace sn {

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ld_x;
  uint8_t* row_codes;
  int64_t ld_row;
  float* row_scale;  // [ceil(cols / 128)][rows or row tiles]
  uint8_t* col_codes;
  int64_t ld_col;
  float* col_scale;  // [ceil(rows / 128)][cols or column tiles]
  int32_t tiles_c;   // column tiles
};

// Queues the kernel (rows, cols >= 1; arguments checked by the caller).
void launch_quantize(QuantArgs a, bool bf16, bool e5m2, bool tiles, hipStream_t st);

}  // namespace sn
