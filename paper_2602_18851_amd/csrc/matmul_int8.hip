// Products of 8-bit integers with a scale for each row (spectral_matmul_int8):
//   C[i][j] = sA[i] sB[j] sum_c A[i][c] B[j][c].
// The sums are exact, in 32 bits on the matrix cores (k stays below 2^17), in whatever order and
// parts: every kernel gives the same bits.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "entry_util.h"
#include "int8_device.h"
#include "quantize_int8.h"
#include "tile_device.h"

namespace {

using namespace sn_dev;

struct IntArgs {
  const uint8_t* a;
  const uint8_t* b;
  const float* sa;
  const float* sb;
  void* c;
  int64_t m, n, k;
  int64_t ld_a, ld_b, ld_c;
  int64_t sa_row, sb_row;
  int32_t tiles_m, tiles_n;
  int32_t splits, blocks_per_split;  // workgroups that share a tile's sum over k, and the 128-column blocks of each
  int32_t* parts;                    // their sums [splits][m][ld_parts], with splits > 1
  int64_t ld_parts;
  int32_t c_bf16;  // C's type, for the kernel that takes either
};

// Sums over 64 columns of 16 x 16 elements: a lane gives 16 bytes of row lane % 16 of each; any 16
// columns, the same ones in x and y.
__device__ __forceinline__ i32x4 multiply64(const u32x4& x, const u32x4& y, const i32x4& sum) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, x), __builtin_bit_cast(i32x4, y), sum, 0, 0, 0);
}

// A scale as fraction and power of two, so that the product of two scales and a sum leaves float32's range
// only where C does.
struct Scale {
  float fraction;
  int power;
};
__device__ __forceinline__ Scale scale_of(const float* s) {
  const float v = *s;
  return Scale{__builtin_amdgcn_frexp_mantf(v), __builtin_amdgcn_frexp_expf(v)};
}
__device__ __forceinline__ float scaled(int sum, const Scale& x, const Scale& y) {
  return __builtin_ldexpf((float)sum * (x.fraction * y.fraction), x.power + y.power);
}

// Row m, columns n .. n + 3 of C from their sums.
template <typename TC>
__device__ __forceinline__ void finish4(const IntArgs& a, int64_t m, int64_t n, const i32x4& sum, const Scale& sa,
                                        const Scale (&sb)[4]) {
  f32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = scaled(sum[e], sa, sb[e]);
  store4(static_cast<TC*>(a.c) + m * a.ld_c + n, r, (int)min(a.n - n, (int64_t)4));
}
// The scales of those columns; past the last the last one's.
__device__ __forceinline__ void column_scales(const IntArgs& a, int64_t n, Scale (&sb)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) sb[e] = scale_of(a.sb + min(n + e, a.n - 1) * a.sb_row);
}

// Tiles of 128 x 128 by 4 waves of 64 x 64, two workgroups to a compute unit, or by 8 waves of 64 x 32.  Blocks of 128
// columns come through two stages in LDS, the next requested before the current one is multiplied.  The
// products are formed transposed (rows from B): a lane holds four neighbouring columns of one row of C.
constexpr int kT = 128;
constexpr int kTStage = 2 * kT * 128;  // rows of A, of B

template <typename TC, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) tile_kernel(IntArgs a) {
  constexpr int ROWS = kT / WAVES;   // rows of each matrix a wave stages
  constexpr int NJ = 16 / WAVES;     // columns of 16 x 16 blocks of a wave: 64 or 32 columns of C
  // one array: with two, the compiler waits for every load into LDS before it reads either
  __shared__ __attribute__((aligned(16))) uint8_t stage[2 * kTStage];
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int per_xcd = gridDim.x / 8;
  const int unit = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (unit >= a.tiles_m * a.tiles_n * a.splits) return;  // whole workgroup
  const int tile = unit / a.splits, split = unit % a.splits;
  int64_t bm, bn;
  place(tile, a.tiles_m, a.tiles_n, bm, bn);

  const int64_t am = bm * kT + ROWS * wv, bnr = bn * kT + ROWS * wv;  // rows this wave stages
  const __amdgpu_buffer_rsrc_t ra = make_rsrc(a.a + am * a.ld_a, range_bytes(am, a.m, ROWS, a.ld_a, a.k));
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.b + bnr * a.ld_b, range_bytes(bnr, a.n, ROWS, a.ld_b, a.k));
  auto issue = [&](int kb) {
    uint8_t* st = stage + (kb & 1) * kTStage;
    stage_issue<ROWS, 0>(ra, st + 128 * ROWS * wv, 128u * (uint32_t)kb, (uint32_t)a.ld_a, lane, ROWS * wv);
    stage_issue<ROWS, 0>(rb, st + 128 * (kT + ROWS * wv), 128u * (uint32_t)kb, (uint32_t)a.ld_b, lane, ROWS * wv);
  };

  const int wm = wv / (WAVES / 2), wn = wv % (WAVES / 2);  // rows from 64 wm, columns from 16 NJ wn
  i32x4 acc[4][NJ];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  // this workgroup's blocks of columns; the last of all may be ragged
  const int kb0 = split * a.blocks_per_split, n_kb = min((int)((a.k + 127) / 128), kb0 + a.blocks_per_split);
  auto block = [&](int kb, auto last_tag) {
    constexpr bool LAST = decltype(last_tag)::value;  // columns from k on are whatever the rows hold there
    const uint8_t* ta = stage + (kb & 1) * kTStage;
    const uint8_t* tb = ta + kT * 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int keep = (int)(a.k - (int64_t)kb * 128) - 16 * (4 * h + q);
      u32x4 fa[4], fb[NJ];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        fa[r] = stage_chunk(ta, 64 * wm + 16 * r + s, 4 * h + q);
        if constexpr (LAST) keep_chunk(fa[r], keep);
      }
#pragma unroll
      for (int r = 0; r < NJ; ++r) {
        fb[r] = stage_chunk(tb, 16 * (NJ * wn + r) + s, 4 * h + q);
        if constexpr (LAST) keep_chunk(fb[r], keep);
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = multiply64(fb[j], fa[i], acc[i][j]);
    }
  };
  auto landed = [&]() {
    wait_loads<0>();
    bare_barrier();  // every wave's part of the block, and the one before it fully read
  };
  if (kb0 < n_kb) issue(kb0);
#pragma unroll 1
  for (int kb = kb0; kb + 1 < n_kb; ++kb) {
    landed();
    issue(kb + 1);
    block(kb, std::false_type{});
  }
  if (kb0 < n_kb) {
    landed();
    block(n_kb - 1, std::true_type{});
  }

#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t n = bn * kT + 16 * (NJ * wn + j) + 4 * q;
    if (n >= a.n) continue;
    Scale sb[4];
    if (a.splits == 1) column_scales(a, n, sb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t m = bm * kT + 64 * wm + 16 * i + s;
      if (m >= a.m) continue;
      if (a.splits > 1)  // rows of the parts are whole groups of four
        *reinterpret_cast<i32x4*>(a.parts + ((int64_t)split * a.m + m) * a.ld_parts + n) = acc[i][j];
      else
        finish4<TC>(a, m, n, acc[i][j], scale_of(a.sa + m * a.sa_row), sb);
    }
  }
}

// Products of few tiles: tiles of 64 x 64 by 4 waves of 32 x 32, so that four times as many workgroups share the product, with a
// ring of kSStages blocks of columns in LDS: a workgroup alone on its compute unit hides its loads' latency itself.
// 1001 x 999 x 3001: 10.7-12 us for 24 blocks one after the other, bound by their latency (a call with tiles of 128 x 128 in
// four parts: 20); 1000^3, 8 blocks, 7-7.5.
constexpr int kST = 64, kSStages = 4;
constexpr int kSStage = 2 * kST * 128;

template <typename TC>
__global__ void __launch_bounds__(256, 2) small_kernel(IntArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t stage[kSStages * kSStage];
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int per_xcd = gridDim.x / 8;
  const int unit = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (unit >= a.tiles_m * a.tiles_n * a.splits) return;  // whole workgroup
  const int tile = unit / a.splits, split = unit % a.splits;
  int64_t bm, bn;
  place(tile, a.tiles_m, a.tiles_n, bm, bn);
  const int64_t am = bm * kST + 16 * wv, bnr = bn * kST + 16 * wv;  // rows this wave stages
  const uint8_t* const pa = a.a + am * a.ld_a;
  const uint8_t* const pb = a.b + bnr * a.ld_b;
  const uint32_t len_a = range_bytes(am, a.m, 16, a.ld_a, a.k), len_b = range_bytes(bnr, a.n, 16, a.ld_b, a.k);
  const int kb0 = split * a.blocks_per_split, n_kb = min((int)((a.k + 127) / 128), kb0 + a.blocks_per_split);
  // past the last block: empty ranges, which keep the count of loads
  auto issue = [&](int kb) {
    uint8_t* st = stage + (kb % kSStages) * kSStage;
    const bool in = kb < n_kb;
    stage_issue<16, 0>(make_rsrc(pa, in ? len_a : 0u), st + 128 * 16 * wv, 128u * (uint32_t)kb, (uint32_t)a.ld_a, lane, 16 * wv);
    stage_issue<16, 0>(make_rsrc(pb, in ? len_b : 0u), st + 128 * (kST + 16 * wv), 128u * (uint32_t)kb, (uint32_t)a.ld_b, lane,
                       16 * wv);
  };
  const int wm = wv >> 1, wn = wv & 1;
  i32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int x = 0; x < kSStages - 1; ++x) issue(kb0 + x);
#pragma unroll 1
  for (int kb = kb0; kb < n_kb; ++kb) {
    wait_loads<4 * (kSStages - 2)>();  // all but the loads of the kSStages - 2 blocks after this one
    bare_barrier();                    // every wave's part of the block, and the one before it fully read
    issue(kb + kSStages - 1);
    const uint8_t* ta = stage + (kb % kSStages) * kSStage;
    const uint8_t* tb = ta + kST * 128;
    u32x4 fa[2][2], fb[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        fa[r][h] = stage_chunk(ta, 32 * wm + 16 * r + s, 4 * h + q);
        fb[r][h] = stage_chunk(tb, 32 * wn + 16 * r + s, 4 * h + q);
      }
    if (128 * (kb + 1) > a.k) {  // columns from k on are whatever the rows hold there
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) keep_chunk(fa[r][h], (int)(a.k - (int64_t)kb * 128) - 16 * (4 * h + q));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = multiply64(fb[j][h], fa[i][h], acc[i][j]);
  }
  wait_loads<0>();  // the last loads have left the LDS alone before the workgroup gives it up

#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t n = bn * kST + 32 * wn + 16 * j + 4 * q;
    if (n >= a.n) continue;
    Scale sb[4];
    if (a.splits == 1) column_scales(a, n, sb);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t m = bm * kST + 32 * wm + 16 * i + s;
      if (m >= a.m) continue;
      if (a.splits > 1)
        *reinterpret_cast<i32x4*>(a.parts + ((int64_t)split * a.m + m) * a.ld_parts + n) = acc[i][j];
      else
        finish4<TC>(a, m, n, acc[i][j], scale_of(a.sa + m * a.sa_row), sb);
    }
  }
}

// Large products: tiles of 256 x 256 by 8 waves of 128 x 64, two per SIMD.  A step is
// a block of 128 columns, two stages of 64 KB in LDS.  A wave takes 64 rows of each half (128 rows) of A and 64 rows of B,
// so a step falls into two phases of 64 x 64 (32 products of 16 x 16 x 64):
//   phase           0                    1
//   reads           A0, B                A1
//   multiplies      A0 B                 A1 B
//   requests        A1 of step k + 1     A0, B of step k + 2
// A phase is a memory part and a product part with a bare barrier after each, and
// waves 4-7 run half a phase behind waves 0-3, so on every SIMD one wave multiplies
// while the other reads.
// Nothing is read or refilled too early:
//   - before the barrier that ends a memory part every wave waits until what the next phase reads has landed. That
//     was requested two phases before it: since then 8 loads, of the two phases after, are outstanding at most;
//   - a memory part ends with its reads complete, a barrier before any wave
//     requests into their place.
// Requests past the last step read nothing (an empty range) and keep the count.
// 8192^3: 421-429 us (2.6 POP/s; tiles of 128 x 128 563), bound by power.
constexpr int kBT = 256;
constexpr int kBHalf = 128 * 128;
constexpr int kBStage = 4 * kBHalf;  // A0, A1, B

template <typename TC>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) big_kernel(IntArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t stage[2 * kBStage];
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int per_xcd = gridDim.x / 8;
  const int tile = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (tile >= a.tiles_m * a.tiles_n) return;  // whole workgroup
  int64_t bm, bn;
  place(tile, a.tiles_m, a.tiles_n, bm, bn);

  // this wave stages rows 16 wv .. + 15 of every 128
  const uint8_t* base[4];
  uint32_t len[4];
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int64_t row = (h < 2 ? bm : bn) * kBT + 128 * (h & 1) + 16 * wv;
    base[h] = h < 2 ? a.a + row * a.ld_a : a.b + row * a.ld_b;
    len[h] = range_bytes(row, h < 2 ? a.m : a.n, 16, h < 2 ? a.ld_a : a.ld_b, a.k);
  }
  const uint32_t rb[2] = {(uint32_t)a.ld_a, (uint32_t)a.ld_b};
  const int n_k = (int)((a.k + 127) / 128), n_full = (int)(a.k / 128);
  const int sr = lane >> 3, p = lane & 7;
  uint32_t voff[2][2];  // operand, row group of 8
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      voff[o][j] = (uint32_t)sr * rb[o] + 16u * (uint32_t)(p ^ stage_swz(16 * wv + 8 * j + sr));
  auto issue = [&](int h, int k) {  // this wave's part of half tile h of step k
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base[h], k < n_k ? len[h] : 0u);
    uint8_t* dst = stage + (k & 1) * kBStage + h * kBHalf + 2048 * wv;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst + 1024 * j), 16, voff[h >> 1][j],
                                               8u * j * rb[h >> 1] + 128u * (uint32_t)k, 0, 0);
  };
  enum { A0 = 0, A1 = 1, B0 = 2, B1 = 3 };

  const int wm = wv >> 2, wn = wv & 3;  // 64 rows of each A half from 64 wm, of B from 64 wn
  i32x4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  u32x4 fa[4][2], fb[4][2];  // [16 rows][half of the block's columns]
  auto read = [&](u32x4 (&f)[4][2], int k, int row) {
    const uint8_t* src = stage + (k & 1) * kBStage + 128 * row;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < 2; ++c) f[r][c] = stage_chunk(src, 16 * r + s, 4 * c + q);
  };
  // zeroes columns >= k of operands of the ragged step
  auto mask = [&](u32x4 (&f)[4][2]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int keep = (int)(a.k - (int64_t)n_full * 128) - 16 * (4 * c + q);
#pragma unroll
      for (int r = 0; r < 4; ++r) keep_chunk(f[r][c], keep);
    }
  };
  auto products = [&](int i0) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i0 + i][j] = multiply64(fb[j][c], fa[i][c], acc[i0 + i][j]);
    __builtin_amdgcn_s_setprio(0);
  };
  auto request = [&](int k) {
    issue(A0, k);
    issue(B0, k);
    issue(B1, k);
  };
  auto step = [&](int k, auto ragged_tag) {
    constexpr bool RAGGED = decltype(ragged_tag)::value;
    // phase 0
    read(fa, k, 64 * wm);
    read(fb, k, 256 + 64 * wn);
    issue(A1, k + 1);
    wait_loads<8>();
    bare_barrier();
    if constexpr (RAGGED) {
      mask(fa);
      mask(fb);
    }
    products(0);
    bare_barrier();
    // phase 1
    read(fa, k, 128 + 64 * wm);
    request(k + 2);
    wait_loads<8>();
    bare_barrier();
    if constexpr (RAGGED) mask(fa);
    products(4);
    bare_barrier();
  };
  request(0);
  issue(A1, 0);
  request(1);
  wait_loads<8>();  // what phase 0 of step 0 reads
  bare_barrier();
  if (wm == 1) bare_barrier();  // waves 4-7: half a phase behind
#pragma unroll 1
  for (int k = 0; k < n_full; ++k) step(k, std::false_type{});
  if (n_full < n_k) step(n_full, std::true_type{});
  if (wm == 0) bare_barrier();
  wait_loads<0>();  // the last loads have left the LDS alone before the workgroup gives it up

  // lane: row 128 (i / 4) + 64 wm + 16 (i % 4) + s, columns 64 wn + 16 j + 4 q .. + 3
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t n = bn * kBT + 64 * wn + 16 * j + 4 * q;
    if (n >= a.n) continue;
    Scale sb[4];
    column_scales(a, n, sb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t m = bm * kBT + 128 * (i >> 2) + 64 * wm + 16 * (i & 3) + s;
      if (m < a.m) finish4<TC>(a, m, n, acc[i][j], scale_of(a.sa + m * a.sa_row), sb);
    }
  }
}

// Adds the parts of C.
template <typename TC>
__global__ void __launch_bounds__(256) join_kernel(IntArgs a) {
  const int64_t per_row = a.ld_parts / 4, all = a.m * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / per_row, n = 4 * (i % per_row);
    const int32_t* p = a.parts + m * a.ld_parts + n;
    i32x4 r = *reinterpret_cast<const i32x4*>(p);
    for (int z = 1; z < a.splits; ++z) r += *reinterpret_cast<const i32x4*>(p + z * a.m * a.ld_parts);
    Scale sb[4];
    column_scales(a, n, sb);
    finish4<TC>(a, m, n, r, scale_of(a.sa + m * a.sa_row), sb);
  }
}

// Few rows of A: every byte of B is used once or a few times, so B's rate from memory bounds the call, and B
// goes straight to registers.  A workgroup takes 16 TN rows of B against all rows of A (16 TM), its 8 waves
// every eighth block of columns each; their sums meet in LDS.  A plain A (PLAIN 1: bf16, 2: float32) that
// fits LDS is quantised by every workgroup for itself, which saves a launch.  One bf16 row against 8192 x 8192: 13.8 us
// (4.9 TB/s); 16.4 when B was requested after the row was quantised.
constexpr int kFewWaves = 8;
constexpr int64_t kPlainBytes = 48 << 10;  // LDS for the codes of a plain A

// LDS of a row of its codes: whole blocks, and 16 bytes that put the rows' chunks into different banks.
constexpr int64_t plain_row(int64_t k) { return (k + 127) / 128 * 128 + 16; }

// Quantises the rows of a plain A into LDS, as the quantiser does, all lanes on each row.
template <typename T>
__device__ __forceinline__ void stage_plain(const IntArgs& a, uint8_t* codes, float* scale, uint32_t (*wave_max)[kFewWaves]) {
  const int k = (int)a.k, m = (int)a.m, row = (int)plain_row(a.k), lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  for (int r = 0; r < m; ++r) {
    uint32_t top = 0;
    const T* x = reinterpret_cast<const T*>(a.a) + r * a.ld_a;
#pragma unroll 2
    for (int c = 8 * threadIdx.x; c < k; c += 8 * 64 * kFewWaves) {
      Eight<T> v;
      v.load(x + c, c, k);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, v.magnitude(e));
    }
    top = max16(top);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (lane == 0) wave_max[r][wv] = top;
  }
  __syncthreads();
  for (int r = 0; r < m; ++r) {
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = max(top, wave_max[r][w]);
    float sc, inv;
    int8_scale(top, sc, inv);
    if (threadIdx.x == 0) scale[r] = sc;
    const T* x = reinterpret_cast<const T*>(a.a) + r * a.ld_a;
#pragma unroll 2
    for (int c = 8 * threadIdx.x; c < row - 16; c += 8 * 64 * kFewWaves) {
      Eight<T> v;
      v.clear();
      if (c < k) v.load(x + c, c, k);
      *reinterpret_cast<uint2*>(codes + r * row + c) = int8_codes(v, c, k, sc, inv);
    }
  }
  __syncthreads();
}

// The same for one row of up to kHeldRow columns, held in registers; its barriers wait for no load, so that those of B go on.
// Longer ones do not fit there and are quantised before B is requested: bf16 against 8192 x 14336 29.7 us, from codes 21.8, and
// against 8192 x 28672 50.6 and 37.8.
constexpr int kHeldRow = 2 * 8 * 64 * kFewWaves;
template <typename T>
struct HeldRow {
  Eight<T> v[2];
  __device__ __forceinline__ void load(const IntArgs& a) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = 8 * (threadIdx.x + 64 * kFewWaves * i);
      v[i].clear();
      if (c < (int)a.k) v[i].load(reinterpret_cast<const T*>(a.a) + c, c, (int)a.k);
    }
  }
  __device__ __forceinline__ void stage(const IntArgs& a, uint8_t* codes, float* scale, uint32_t* wave_max) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, v[i].magnitude(e));
    top = max16(top);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = top;
    wait_loads<63>();
    bare_barrier();
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = max(top, wave_max[w]);
    float sc, inv;
    int8_scale(top, sc, inv);
    if (threadIdx.x == 0) *scale = sc;
    const int room = (int)((a.k + 127) / 128 * 128);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = 8 * (threadIdx.x + 64 * kFewWaves * i);
      if (c < room) *reinterpret_cast<uint2*>(codes + c) = int8_codes(v[i], c, a.k, sc, inv);
    }
    wait_loads<63>();
    bare_barrier();
  }
};

template <int TM, int TN, int PLAIN>
__global__ void __launch_bounds__(64 * kFewWaves, TM * TN == 1 ? 4 : 2) few_rows_kernel(IntArgs a) {
  static_assert(PLAIN == 0 || TM <= 2, "a plain A has 32 rows at most");
  constexpr int AHEAD = 4;
  __shared__ i32x4 sums[kFewWaves][TM * TN][64];
  __shared__ uint32_t wave_max[PLAIN ? 16 * TM : 1][kFewWaves];
  __shared__ float plain_scale[PLAIN ? 16 * TM : 1];
  extern __shared__ __attribute__((aligned(16))) uint8_t plain_codes[];  // PLAIN: [m][plain_row(k)]
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int k = (int)a.k, n_kb = (k + 127) / 128, n_full = k / 128;
  const int64_t n0 = (int64_t)blockIdx.x * 16 * TN;
  using T = typename std::conditional<PLAIN == 1, __bf16, float>::type;

  // rows past the last read the last one's, their results are dropped
  const uint8_t* pa[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = min((int64_t)(16 * i + s), a.m - 1);
    pa[i] = PLAIN ? plain_codes + m * plain_row(k) : a.a + m * a.ld_a;
  }
  const uint8_t* pb[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) pb[j] = a.b + min(n0 + 16 * j + s, a.n - 1) * a.ld_b;

  i32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};

  struct Side {
    u32x4 b[TN][2], a[TM][2];
  };
  // columns c .. c + 15 and c + 64 .. c + 79 of a row; in the block that column k ends in, zeros from k on
  auto read = [&](u32x4 (&v)[2], const uint8_t* row, int c, auto last) {
    constexpr bool LAST = decltype(last)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v[h] = u32x4{0, 0, 0, 0};
      if (!LAST || c + 64 * h < k) v[h] = *reinterpret_cast<const u32x4*>(row + c + 64 * h);
      if constexpr (LAST) keep_chunk(v[h], k - c - 64 * h);
    }
  };
  auto load = [&](Side& t, int kb, auto last) {
#pragma unroll
    for (int j = 0; j < TN; ++j) read(t.b[j], pb[j], 128 * kb + 16 * q, last);
    if constexpr (PLAIN == 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) read(t.a[i], pa[i], 128 * kb + 16 * q, last);
    }
  };
  auto multiply = [&](Side& t, int kb) {
    if constexpr (PLAIN != 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) read(t.a[i], pa[i], 128 * kb + 16 * q, std::false_type{});
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = multiply64(t.b[j][h], t.a[i][h], acc[i][j]);
  };
  // this wave's full blocks wv, wv + 8, ..: `count` of them, in groups of AHEAD
  const int count = n_full > wv ? (n_full - wv + kFewWaves - 1) / kFewWaves : 0, groups = count / AHEAD;
  int kb = wv, g = 0;
  if constexpr (PLAIN != 0) {
    if (TM == 1 && a.m == 1 && k <= kHeldRow && n_full >= kFewWaves * AHEAD) {  // the same for all waves
      HeldRow<T> row;
      row.load(a);
      Side t[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) load(t[u], kb + kFewWaves * u, std::false_type{});
      row.stage(a, plain_codes, plain_scale, wave_max[0]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) multiply(t[u], kb + kFewWaves * u);
      kb += kFewWaves * AHEAD;
      g = 1;
    } else {
      stage_plain<T>(a, plain_codes, plain_scale, wave_max);
    }
  }
#pragma unroll 1
  for (; g < groups; ++g, kb += kFewWaves * AHEAD) {
    Side t[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(t[u], kb + kFewWaves * u, std::false_type{});
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) multiply(t[u], kb + kFewWaves * u);
  }
  // what is left: fewer than AHEAD full blocks and, for one wave, the ragged one
#pragma unroll 1
  for (; kb < n_full; kb += kFewWaves) {
    Side t;
    load(t, kb, std::false_type{});
    multiply(t, kb);
  }
  if (kb < n_kb) {
    Side t;
    load(t, kb, std::true_type{});
    multiply(t, kb);
  }

#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) sums[wv][i * TN + j][lane] = acc[i][j];
  __syncthreads();
#pragma unroll 1
  for (int t = wv; t < TM * TN; t += kFewWaves) {
    i32x4 r = sums[0][t][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) r += sums[w][t][lane];
    const int64_t m = 16 * (t / TN) + s, n = n0 + 16 * (t % TN) + 4 * q;
    if (m >= a.m || n >= a.n) continue;
    Scale sb[4];
    column_scales(a, n, sb);
    const Scale sa = scale_of(PLAIN ? plain_scale + m : a.sa + m * a.sa_row);
    if (a.c_bf16)
      finish4<__bf16>(a, m, n, r, sa, sb);
    else
      finish4<float>(a, m, n, r, sa, sb);
  }
}

// What a call runs: sn_matmul_kernel, and its workgroups of so many threads.
struct Run {
  int32_t kernel, threads;
  int64_t workgroups;
};

void launch_tiles(const IntArgs& a, const Run& run, hipStream_t st) {
  const dim3 g((uint32_t)run.workgroups);
  if (run.kernel == SN_MATMUL_BIG)
    a.c_bf16 ? big_kernel<__bf16><<<g, 512, 0, st>>>(a) : big_kernel<float><<<g, 512, 0, st>>>(a);
  else if (run.kernel == SN_MATMUL_SMALL)
    a.c_bf16 ? small_kernel<__bf16><<<g, 256, 0, st>>>(a) : small_kernel<float><<<g, 256, 0, st>>>(a);
  else if (run.kernel == SN_MATMUL_TILE_8)
    a.c_bf16 ? tile_kernel<__bf16, 8><<<g, 512, 0, st>>>(a) : tile_kernel<float, 8><<<g, 512, 0, st>>>(a);
  else
    a.c_bf16 ? tile_kernel<__bf16, 4><<<g, 256, 0, st>>>(a) : tile_kernel<float, 4><<<g, 256, 0, st>>>(a);
  if (a.splits > 1) {
    const dim3 j((uint32_t)std::min<int64_t>((a.m * (a.ld_parts / 4) + 255) / 256, 4096));
    a.c_bf16 ? join_kernel<__bf16><<<j, 256, 0, st>>>(a) : join_kernel<float><<<j, 256, 0, st>>>(a);
  }
}

void launch_few(const IntArgs& a, const Run& run, int plain, hipStream_t st) {
  const int t = (int)((a.m + 15) / 16);
  const dim3 g((uint32_t)run.workgroups);
  constexpr int W = 64 * kFewWaves;
  const size_t lds = plain ? (size_t)(a.m * plain_row(a.k)) : 0;
  if (plain == 1) return t == 1 ? few_rows_kernel<1, 1, 1><<<g, W, lds, st>>>(a) : few_rows_kernel<2, 1, 1><<<g, W, lds, st>>>(a);
  if (plain == 2) return t == 1 ? few_rows_kernel<1, 1, 2><<<g, W, lds, st>>>(a) : few_rows_kernel<2, 1, 2><<<g, W, lds, st>>>(a);
  switch (t) {
    case 1: return few_rows_kernel<1, 1, 0><<<g, W, 0, st>>>(a);
    case 2: return few_rows_kernel<2, 2, 0><<<g, W, 0, st>>>(a);
    default: return few_rows_kernel<4, 2, 0><<<g, W, 0, st>>>(a);
  }
}

// ------------------------------------------------------------------ host side

using sn::aligned;
using sn::refuse;

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Whether there is a kernel for so few rows: 33 to 48 (40 rows 33 us against 8192 x 8192) are never
// cheaper than the tiles of 64 x 64 (16.7).
constexpr bool few_rows(int64_t m) { return m <= 32 || (m > 48 && m <= 64); }

// The kernel of a product, and over how many workgroups a tile's sum is split: the cheapest by these costs in us.  A
// launch's start and end, and a block of 128 columns: 64 x 64 tiles, one to a compute unit 0.29, two 0.39 (128 x 8192 x 8192
// 22 us, 256 28.8, 512 54); 128 x 128 0.65 and 0.97 (512 x 8192 x 8192 45, 1024 66); 256 x 256, one to a unit, 1.62
// (8192^3 421).  Parts are written, read and joined at 5.5 TB/s in a launch more: 512 x 512 x 16384 35 us in one part of 64 x
// 64 tiles, 21 in 16 of 128 x 128.  Few rows: 512 or 1024 columns of C at a time, each wave an eighth of the columns of A (1 row
// against 8192 x 8192 13.7, 64 rows 27.5).
struct Way {
  int kernel;
  int splits, blocks_per_split;
  double cost;
};

Way choose(int64_t m, int64_t n, int64_t k, bool f32) {
  auto up = [](int64_t x, int64_t t) { return (x + t - 1) / t; };
  const int64_t n_kb = std::max<int64_t>(up(k, 128), 1);
  Way best{SN_MATMUL_BIG, 1, (int)n_kb, 8.0 + 1.62 * (double)(up(up(m, kBT) * up(n, kBT), 256) * n_kb)};
  auto tiles = [&](int kernel, int64_t size, double start, double alone, double both) {
    const int64_t all = up(m, size) * up(n, size);
    for (int64_t s = 1; s <= 16 && (s == 1 || 2 * s <= n_kb); ++s) {
      const int64_t per = up(n_kb, s), wgs = all * s, rest = wgs % 512;
      if (s > 1 && (s - 1) * per >= n_kb) continue;  // a split without blocks
      double c = start + (double)per * ((double)(wgs / 512) * both + (rest == 0 ? 0.0 : rest <= 256 ? alone : both));
      if (s > 1) c += 5.5 + (double)(8 * s + (f32 ? 4 : 2)) * (double)m * (double)n / 5.5e6;
      if (c < best.cost) best = Way{kernel, (int)s, (int)per, c};
    }
  };
  tiles(SN_MATMUL_TILE_4, kT, 5.0, 0.65, 0.97);
  tiles(SN_MATMUL_SMALL, kST, 4.0, 0.29, 0.39);
  // 512 lanes for 16 columns of C have to stay below the 2^32 of a launch
  if (few_rows(m) && n <= (int64_t(1) << 27) - 16) {
    const int t = (int)((m + 15) / 16);
    const double block = t == 1 ? 0.66 : t == 2 ? 1.8 : 2.9;
    const double cost = 3.0 + std::max(1.0, (double)up(n, t == 1 ? 16 : 32) / 256.0) * (double)up(n_kb, kFewWaves) * block;
    if (cost <= best.cost) best = Way{SN_MATMUL_FEW_ROWS, 1, (int)n_kb, cost};
  }
  return best;
}

struct Plan {
  Run run;
  int32_t tiles_m, tiles_n;
  int32_t splits, blocks_per_split;
  int64_t off_parts, ld_parts;
  bool plain_a;
  bool fuse;         // the kernel for few rows, which quantises a plain A itself
  int64_t ld_codes;  // of a plain A's codes
  int64_t off_scale, bytes;
};

// Checks the description and fills in its defaults.
int resolve(sn_matmul_int8& p, Plan& pl) {
  const bool plain = p.a_type == SN_F32 || p.a_type == SN_BF16;
  if (!plain && p.a_type != SN_I8) return refuse(SN_EDTYPE, "a_type must be SN_I8, SN_F32 or SN_BF16");
  if (p.c_type != SN_F32 && p.c_type != SN_BF16) return refuse(SN_EDTYPE, "c_type must be SN_F32 or SN_BF16");
  if (p.m < 0 || p.n < 0 || p.k < 0) return refuse(SN_EINVAL, "m, n and k must be >= 0");
  constexpr int64_t kMost = int64_t(1) << 40, kMostRows = int64_t(1) << 34, kMostLd = int64_t(1) << 22;
  if (p.m > kMostRows || p.n > kMostRows || p.ld_a > kMost || p.ld_b > kMost || p.ld_c > kMost)
    return refuse(SN_EINVAL, "m, n or a row stride is too large");
  if (p.k >= (1 << 17)) return refuse(SN_EINVAL, "k must stay below 2^17");
  if (p.ld_a == 0) p.ld_a = plain ? p.k : round_up(p.k, 16);
  if (p.ld_b == 0) p.ld_b = round_up(p.k, 16);
  if (p.ld_c == 0) p.ld_c = p.n;
  if (p.ld_a < p.k || p.ld_b < p.k || p.ld_c < p.n)
    return refuse(SN_EINVAL, "ld_a and ld_b must be >= k, ld_c >= n");
  if ((!plain && (p.ld_a % 16 || p.ld_a >= kMostLd)) || p.ld_b % 16 || p.ld_b >= kMostLd)
    return refuse(SN_EINVAL, "code rows must be multiples of 16 bytes, below 2^22");
  for (int64_t* s : {&p.sa_row, &p.sb_row}) {
    if (*s == SN_STRIDE_ZERO)
      *s = 0;
    else if (*s == 0)
      *s = 1;
    if (*s < 0 || *s > kMost) return refuse(SN_EINVAL, "scale strides must be >= 0 and below 2^40");
  }
  const int64_t small = ((p.m + 127) / 128) * ((p.n + 127) / 128);
  if (small >= (int64_t(1) << 22)) return refuse(SN_EINVAL, "m x n must stay below 2^22 tiles of 128 x 128");
  pl = Plan{};
  pl.plain_a = plain;
  pl.splits = 1;
  if (p.m == 0 || p.n == 0) return SN_OK;
  const Way way = choose(p.m, p.n, p.k, p.c_type == SN_F32);
  const bool few = way.kernel == SN_MATMUL_FEW_ROWS;
  pl.fuse = few && plain && p.m <= 32 && p.m * plain_row(p.k) <= kPlainBytes;
  if (plain && !pl.fuse) {
    pl.ld_codes = round_up(p.k, 16);
    pl.off_scale = round_up(p.m * pl.ld_codes, 256);
    pl.bytes = pl.off_scale + round_up(p.m * 4, 256);
  }
  if (few) {
    const int64_t cols = p.m <= 16 || pl.fuse ? 16 : 32;  // of C that a workgroup takes
    pl.run = Run{SN_MATMUL_FEW_ROWS, 64 * kFewWaves, (p.n + cols - 1) / cols};
    return SN_OK;
  }
  const int64_t size = way.kernel == SN_MATMUL_BIG ? kBT : way.kernel == SN_MATMUL_SMALL ? kST : kT;
  pl.tiles_m = (int32_t)((p.m + size - 1) / size);
  pl.tiles_n = (int32_t)((p.n + size - 1) / size);
  pl.splits = way.splits;
  pl.blocks_per_split = way.blocks_per_split;
  if (pl.splits > 1) {
    pl.off_parts = pl.bytes;
    pl.ld_parts = round_up(p.n, 4);
    pl.bytes += round_up(pl.splits * p.m * pl.ld_parts * 4, 256);
  }
  const int64_t units = (int64_t)pl.tiles_m * pl.tiles_n * pl.splits;
  // a 128 x 128 tile alone on its compute unit: 8 waves; else two of 4
  pl.run.kernel = way.kernel == SN_MATMUL_TILE_4 && units <= 256 ? SN_MATMUL_TILE_8 : way.kernel;
  pl.run.threads = pl.run.kernel == SN_MATMUL_BIG || pl.run.kernel == SN_MATMUL_TILE_8 ? 512 : 256;
  pl.run.workgroups = (units + 7) / 8 * 8;  // whole rounds of the XCDs
  return SN_OK;
}

}  // namespace

extern "C" SN_API int spectral_matmul_int8_workspace_bytes(const sn_matmul_int8* desc, int64_t* bytes) {
  if (!desc || !bytes) return refuse(SN_ENULL, "p and bytes must not be NULL");
  sn_matmul_int8 p = *desc;
  Plan pl;
  if (int rc = resolve(p, pl)) return rc;
  *bytes = pl.bytes;
  return SN_OK;
}

extern "C" SN_API int spectral_matmul_int8_kernel(const sn_matmul_int8* desc, int32_t* kernel, int32_t* parts,
                                                  int64_t* workgroups, int32_t* threads) {
  if (!desc || !kernel || !parts || !workgroups || !threads)
    return refuse(SN_ENULL, "p, kernel, parts, workgroups and threads must not be NULL");
  sn_matmul_int8 p = *desc;
  Plan pl;
  if (int rc = resolve(p, pl)) return rc;
  *kernel = pl.run.kernel;
  *parts = pl.run.kernel == 0 ? 0 : pl.splits;
  *workgroups = pl.run.workgroups;
  *threads = pl.run.threads;
  return SN_OK;
}

extern "C" SN_API int spectral_matmul_int8(const sn_matmul_int8* desc, const void* a, const float* sa, const int8_t* b,
                                           const float* sb, void* c, void* workspace, int64_t workspace_bytes,
                                           void* hip_stream) {
  if (!desc) return refuse(SN_ENULL, "p must not be NULL");
  sn_matmul_int8 p = *desc;
  Plan pl;
  if (int rc = resolve(p, pl)) return rc;
  if (p.m == 0 || p.n == 0) return SN_OK;
  if (!c || !sb || (!pl.plain_a && !sa) || (p.k > 0 && (!a || !b)))
    return refuse(SN_ENULL, "a, sa (of codes), b, sb and c must not be NULL");
  if (pl.plain_a ? !aligned(a, p.a_type == SN_F32 ? 4 : 2) : !aligned(a, 16) || !aligned(sa, 4))
    return refuse(SN_EINVAL, "codes must be 16-byte aligned, a plain A and scales aligned to their type");
  if (!aligned(b, 16) || !aligned(sb, 4) || !aligned(c, p.c_type == SN_F32 ? 4 : 2))
    return refuse(SN_EINVAL, "codes must be 16-byte aligned, scales and C aligned to their type");
  if (pl.bytes > 0) {
    if (!workspace) return refuse(SN_ENULL, "workspace must not be NULL");
    if (workspace_bytes < pl.bytes)
      return refuse(SN_EINVAL, "workspace too small (spectral_matmul_int8_workspace_bytes)");
    if (!aligned(workspace, 256)) return refuse(SN_EINVAL, "workspace must be 256-byte aligned");
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = sn::check_stream(st)) return rc;

  IntArgs g{};
  g.a = static_cast<const uint8_t*>(a);
  g.b = reinterpret_cast<const uint8_t*>(b);
  g.sa = sa;
  g.sb = sb;
  g.c = c;
  g.m = p.m;
  g.n = p.n;
  g.k = p.k;
  g.ld_a = p.ld_a;
  g.ld_b = p.ld_b;
  g.ld_c = p.ld_c;
  g.sa_row = p.sa_row;
  g.sb_row = p.sb_row;
  g.c_bf16 = p.c_type == SN_BF16;
  if (pl.plain_a && !pl.fuse) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    float* scale = reinterpret_cast<float*>(ws + pl.off_scale);
    sn::launch_quantize_int8({a, p.m, p.k, p.ld_a, reinterpret_cast<int8_t*>(ws), pl.ld_codes, scale},
                             p.a_type == SN_BF16, st);
    if (int rc = sn::launched("quantise")) return rc;
    g.a = ws;
    g.ld_a = pl.ld_codes;
    g.sa = scale;
    g.sa_row = 1;
  }
  g.splits = pl.splits;
  g.blocks_per_split = pl.blocks_per_split;
  g.parts = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + pl.off_parts);
  g.ld_parts = pl.ld_parts;
  g.tiles_m = pl.tiles_m;
  g.tiles_n = pl.tiles_n;
  if (pl.run.kernel == SN_MATMUL_FEW_ROWS)
    launch_few(g, pl.run, !pl.fuse ? 0 : p.a_type == SN_BF16 ? 1 : 2, st);
  else
    launch_tiles(g, pl.run, st);
  return sn::launched("product");
}
