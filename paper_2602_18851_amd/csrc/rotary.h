// Internal interface of the rotary kernels (rotary.hip), which the logit consumer runs on its planes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "spectral.h"

namespace sn {

constexpr int kMaxPairs = 128;  // rot_dim <= 256

// What a launch needs of a plan, passed by value: pair frequencies in turns per position.
struct RotaryTable {
  double turns[kMaxPairs];
  double amplitude;
  int32_t pairs, head_dim, interleaved;
};

// Checks a plan and forms its table.
int rotary_table(const sn_rotary* p, RotaryTable& t);

// Turns the hi and lo bf16 planes [layers][seq][n_heads * head_dim] of Q and K in place.
int launch_rotary_planes(const RotaryTable& t, int64_t layers, int64_t seq, const int64_t* positions, int64_t q_heads,
                         int64_t k_heads, uint16_t* qh, uint16_t* ql, uint16_t* kh, uint16_t* kl, hipStream_t st);

}  // namespace sn
