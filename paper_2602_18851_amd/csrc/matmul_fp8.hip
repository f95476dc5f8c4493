// Products of 8-bit matrices with a scale for each block of 128 (spectral_matmul_fp8):
//   C[i][j] = sum_b sA[b][i] sB[b][j] sum_{c in b} A[i][c] B[j][c].
// A block's inner sum starts from zero on the matrix cores; the vector ALUs add
// it to C with the blocks' scales, in float32.
//
// Which matrix instruction depends on C's type.  The 8-bit one (16x16x128, the
// depth of a block) adds the products of 8 neighbouring columns at the exponent of the
// largest, dropping what lies 14 bits below it: measured, 1 + 2^-13 is kept
// and 1 + 2^-14 is not, while different eights are added in float32.  On normal values a
// block's sum is off by 1.5e-5 of itself: nothing in a C of bf16 (2^-8), nor beside
// the codes' own rounding (2^-4), but more than a float32 C stands for.  A
// float32 C takes the codes as float16, which holds both formats exactly, and the float16
// instruction, whose products are exact and summed in float32 (1e-8 of the sum), at half the rate.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "entry_util.h"
#include "fp8_device.h"
#include "quantize_fp8.h"

namespace {

using namespace sn_dev;

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct MatArgs {
  const uint8_t* a;
  const uint8_t* b;
  const float* sa;
  const float* sb;
  void* c;
  int64_t m, n, k;
  int64_t ld_a, ld_b, ld_c;
  int64_t sa_block, sa_row, sb_block, sb_row;
  int32_t a_shift, b_shift;  // log2 of the rows that share a scale (0 or 7)
  int32_t tiles_m, tiles_n;
  int32_t splits, blocks_per_split;  // workgroups that share a tile's sum over k, and the 128-column blocks of each
  float* parts;                      // their sums [splits][m][ld_parts], with splits > 1
  int64_t ld_parts;
  int32_t c_bf16;  // C's type, for the kernel that takes either
};

// One 16 x 16 block of the inner sums over 128 columns: rows from x (format
// FX: 0 E4M3, 1 E5M2), columns from y.  A lane gives 32 bytes of row lane % 16 of
// each; any 32 columns, the same ones in x and y.
template <int FX, int FY>
__device__ __forceinline__ f32x4 block_product(const i32x8& x, const i32x8& y) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, f32x4{0.f, 0.f, 0.f, 0.f}, FX, FY, 0, 0, 0, 0);
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Place of tile t: bands of kBand tiles in m, column after column of a band, so that the tiles
// that run at one time on an XCD share few rows of A and of B in its L2.
// 8192^3 to bf16: 467 us column by column, 443, 432 and 427 in bands of 16, 8 and 4.
constexpr int kBand = 4;
__device__ __forceinline__ void place(int t, int tiles_m, int tiles_n, int64_t& bm, int64_t& bn) {
  const int band = t / (kBand * tiles_n), first = band * kBand, in = t - first * tiles_n;
  const int rows = min(kBand, tiles_m - first);
  bm = first + in % rows;
  bn = in / rows;
}

// Eight codes as float16, exactly (NaN codes as NaN).
template <int F>
__device__ __forceinline__ f16x8 widen(uint32_t w0, uint32_t w1) {
  f16x2 h[4];
  if constexpr (F == 0) {
    h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.f, false);
    h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.f, true);
    h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.f, false);
    h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.f, true);
  } else {
    // E5M2 is the upper byte of a float16
    h[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0u, w0, 0x010c000cu));
    h[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0u, w0, 0x030c020cu));
    h[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0u, w1, 0x010c000cu));
    h[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0u, w1, 0x030c020cu));
  }
  return f16x8{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
}

__device__ __forceinline__ i32x8 join(const u32x4& lo, const u32x4& hi) {
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
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

// Tiles of 128 x 128 by 4 waves of 64 x 64, two workgroups to a compute unit, or by 8 waves of 64 x 32.  Blocks of
// 128 columns and the scales of their rows come through two stages in LDS, the next requested before the current one is
// multiplied (three or four stages gain nothing: by 4 waves, 512 x 8192 x 8192 46.6 and 46.4 us, two 45.7).  The products are
// formed transposed (rows from B): a lane holds four neighbouring columns of one row of C, with one scale of A.  Scales
// through LDS, a block ahead, and not read as they are needed: by 4 waves, 4096^3 to float32 139 instead of 230 us, 256 x
// 8192 x 8192 to bf16 46 instead of 66 (by 8 waves 31.6).
constexpr int kT = 128;
constexpr int kTStage = 2 * kT * 128 + 2 * kT * 4;  // rows of A, of B, then their scales

template <int FA, int FB, bool ROWS_B, typename TC, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) tile_kernel(MatArgs a) {
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
  // and scales of 64 rows, of A in waves 0 and 1, of B in 2 and 3; rows past the last take the last one's
  const bool sc_a = wv < 2;
  const int64_t sc_row0 = (sc_a ? bm : bn) * kT + 64 * (wv & 1), sc_rows = sc_a ? a.m : a.n;
  const float* sc_at = (sc_a ? a.sa : a.sb) +
                       (min(sc_row0 + lane, sc_rows - 1) >> (sc_a ? a.a_shift : a.b_shift)) * (sc_a ? a.sa_row : a.sb_row);
  const int64_t sc_block = sc_a ? a.sa_block : a.sb_block;
  auto issue = [&](int kb) {
    uint8_t* st = stage + (kb & 1) * kTStage;
    stage_issue<ROWS, 0>(ra, st + 128 * ROWS * wv, 128u * (uint32_t)kb, (uint32_t)a.ld_a, lane, ROWS * wv);
    stage_issue<ROWS, 0>(rb, st + 128 * (kT + ROWS * wv), 128u * (uint32_t)kb, (uint32_t)a.ld_b, lane, ROWS * wv);
    if (wv < 4) __builtin_amdgcn_global_load_lds(sc_at + kb * sc_block, (lds_void*)(st + 2 * kT * 128 + 256 * wv), 4, 0, 0);
  };

  const int wm = wv / (WAVES / 2), wn = wv % (WAVES / 2);  // rows from 64 wm, columns from 16 NJ wn
  f32x4 acc[4][NJ];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // this workgroup's blocks of columns; the last of all may be ragged
  const int kb0 = split * a.blocks_per_split, n_kb = min((int)((a.k + 127) / 128), kb0 + a.blocks_per_split);
  auto block = [&](int kb, auto last_tag) {
    constexpr bool LAST = decltype(last_tag)::value;  // columns from k on are whatever the rows hold there
    const uint8_t* ta = stage + (kb & 1) * kTStage;
    const uint8_t* tb = ta + kT * 128;
    const float* sc = reinterpret_cast<const float*>(ta + 2 * kT * 128);
    u32x4 fa[4][2], fb[NJ][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int keep = (int)(a.k - (int64_t)kb * 128) - 16 * (4 * h + q);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        fa[r][h] = stage_chunk(ta, 64 * wm + 16 * r + s, 4 * h + q);
        if constexpr (LAST) keep_chunk(fa[r][h], keep);
      }
#pragma unroll
      for (int r = 0; r < NJ; ++r) {
        fb[r][h] = stage_chunk(tb, 16 * (NJ * wn + r) + s, 4 * h + q);
        if constexpr (LAST) keep_chunk(fb[r][h], keep);
      }
    }
    float sa[4];
    f32x4 sb[ROWS_B ? NJ : 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) sa[i] = sc[64 * wm + 16 * i + s];
    if constexpr (ROWS_B) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) sb[j] = *reinterpret_cast<const f32x4*>(sc + kT + 16 * (NJ * wn + j) + 4 * q);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) sa[i] *= sc[kT + 16 * NJ * wn];
    }
    auto add = [&](int i, int j, const f32x4& part) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(part[e], ROWS_B ? sa[i] * sb[j][e] : sa[i], acc[i][j][e]);
    };
    if constexpr (sizeof(TC) == 2) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          add(i, j, block_product<FB, FA>(join(fb[j][0], fb[j][1]), join(fa[i][0], fa[i][1])));
    } else {
      // two columns of 16 x 16 blocks at a time: their sums and codes as float16 stay in registers
#pragma unroll
      for (int jj = 0; jj < NJ; jj += 2) {
        f32x4 part[4][2];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const int w = 2 * (h & 1);
          f16x8 hb[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) hb[j] = widen<FB>(fb[jj + j][h >> 1][w], fb[jj + j][h >> 1][w + 1]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f16x8 ha = widen<FA>(fa[i][h >> 1][w], fa[i][h >> 1][w + 1]);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                  hb[j], ha, h == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[i][j], 0, 0, 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) add(i, jj + j, part[i][j]);
      }
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
  for (int i = 0; i < 4; ++i) {
    const int64_t m = bm * kT + 64 * wm + 16 * i + s;
    if (m >= a.m) continue;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t n = bn * kT + 16 * (NJ * wn + j) + 4 * q;
      if (n >= a.n) continue;
      if (a.splits > 1)  // rows of the parts are whole groups of four
        *reinterpret_cast<f32x4*>(a.parts + ((int64_t)split * a.m + m) * a.ld_parts + n) = acc[i][j];
      else
        store4(static_cast<TC*>(a.c) + m * a.ld_c + n, acc[i][j], (int)min(a.n - n, (int64_t)4));
    }
  }
}

// Large products: tiles of 256 x 256 by 8 waves of 128 x 64, two per SIMD.  A step is
// a block of 128 columns, two stages of 64 KB in LDS and the scales of its rows
// of A and B.  A wave takes 64 rows of each half (128 rows) of A and 64 rows of B,
// so a step falls into two phases of 64 x 64 (16 products of 16 x 16 x 128):
//   phase           0                    1
//   reads           A0, B, scales        A1
//   multiplies      A0 B                 A1 B
//   requests        A1 of step k + 1     A0, B and scales of step k + 2
// A phase is a memory part and a product part with a bare barrier after each, and
// waves 4-7 run half a phase behind waves 0-3, so on every SIMD one wave multiplies
// while the other reads.  (8192^3 before the order of tiles below: 518 us in four phases of 64 x 32, 467
// in two.)
// Nothing is read or refilled too early:
//   - before the barrier that ends a memory part every wave waits until what the next phase reads has landed. That
//     was requested two phases before it: since then 9 loads, of the two phases after, are outstanding at most;
//   - a memory part ends with its reads complete, a barrier before any wave
//     requests into their place.
// Requests past the last step read nothing (an empty range; scales: the last block again)
// and keep the count.
constexpr int kBT = 256;
constexpr int kBHalf = 128 * 128;
constexpr int kBStage = 4 * kBHalf;  // A0, A1, B

template <int FA, int FB, bool ROWS_B>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) big_kernel(MatArgs a) {
  // two stages, then of each the scales of the tile's rows of A and of B; one array: with two, the compiler waits
  // for every load into LDS before it reads either
  __shared__ __attribute__((aligned(16))) uint8_t stage[2 * kBStage + 2 * 2 * kBT * 4];
  float* const scales = reinterpret_cast<float*>(stage + 2 * kBStage);
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
  // waves 0-3 stage the scales of 64 rows of A each, waves 4-7 of B; rows past the last take the last one's
  const bool sc_a = wv < 4;
  const int64_t sc_row0 = sc_a ? bm * kBT : bn * kBT, sc_rows = sc_a ? a.m : a.n, sc_step = sc_a ? a.sa_row : a.sb_row;
  const int sc_shift = sc_a ? a.a_shift : a.b_shift;
  const int64_t sc_at = min(sc_row0 + 64 * (wv & 3) + lane, sc_rows - 1) >> sc_shift;
  const float* sc_base = (sc_a ? a.sa : a.sb) + (sc_row0 >> sc_shift) * sc_step;
  const uint32_t sc_off = (uint32_t)((sc_at - (sc_row0 >> sc_shift)) * sc_step * 4);
  const int64_t sc_block = sc_a ? a.sa_block : a.sb_block;
  auto issue_scales = [&](int k) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(uni(sc_base + (k < n_k ? k : n_k - 1) * sc_block), 0x7fffffffu);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(scales + (k & 1) * 2 * kBT + 64 * wv), 4, sc_off, 0, 0, 0);
  };
  enum { A0 = 0, A1 = 1, B0 = 2, B1 = 3 };

  const int wm = wv >> 2, wn = wv & 3;  // 64 rows of each A half from 64 wm, of B from 64 wn
  f32x4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 fa[4][2], fb[4][2];  // [16 rows][half of the block's columns]
  float sa[8];               // scale of row 128 (i / 4) + 64 wm + 16 (i % 4) + s, times B's where that is one
  f32x4 sb[ROWS_B ? 4 : 1];  // scales of rows 64 wn + 16 j + 4 q .. + 3 of B
  auto read = [&](u32x4 (&f)[4][2], int k, int row) {
    const uint8_t* src = stage + (k & 1) * kBStage + 128 * row;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < 2; ++c) f[r][c] = stage_chunk(src, 16 * r + s, 4 * c + q);
  };
  auto read_scales = [&](int k) {
    const float* src = scales + (k & 1) * 2 * kBT;
#pragma unroll
    for (int i = 0; i < 8; ++i) sa[i] = src[128 * (i >> 2) + 64 * wm + 16 * (i & 3) + s];
    if constexpr (ROWS_B) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sb[j] = *reinterpret_cast<const f32x4*>(src + kBT + 64 * wn + 16 * j + 4 * q);
    } else {
      const float b = src[kBT + 64 * wn];
#pragma unroll
      for (int i = 0; i < 8; ++i) sa[i] *= b;
    }
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
    // kFlight block sums are under way before the first is added to C, so that the matrix cores never wait for the
    // additions nor these for them; in this order, which the compiler's own does not keep
    constexpr int kFlight = 4;
    f32x4 part[kFlight];
    auto multiply = [&](int t) {
      part[t % kFlight] = block_product<FB, FA>(join(fb[t & 3][0], fb[t & 3][1]), join(fa[t >> 2][0], fa[t >> 2][1]));
      __builtin_amdgcn_sched_barrier(0);
    };
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int t = 0; t < kFlight; ++t) multiply(t);
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int i = i0 + (t >> 2), j = t & 3;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[i][j][e] = fmaf(part[t % kFlight][e], ROWS_B ? sa[i] * sb[j][e] : sa[i], acc[i][j][e]);
      __builtin_amdgcn_sched_barrier(0);
      if (t + kFlight < 16) multiply(t + kFlight);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  auto request = [&](int k) {
    issue(A0, k);
    issue(B0, k);
    issue(B1, k);
    issue_scales(k);
  };
  auto step = [&](int k, auto ragged_tag) {
    constexpr bool RAGGED = decltype(ragged_tag)::value;
    // phase 0
    read(fa, k, 64 * wm);
    read(fb, k, 256 + 64 * wn);
    read_scales(k);
    issue(A1, k + 1);
    wait_loads<9>();
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
    wait_loads<9>();
    bare_barrier();
    if constexpr (RAGGED) mask(fa);
    products(4);
    bare_barrier();
  };
  request(0);
  issue(A1, 0);
  request(1);
  wait_loads<9>();  // what phase 0 of step 0 reads
  bare_barrier();
  if (wm == 1) bare_barrier();  // waves 4-7: half a phase behind
#pragma unroll 1
  for (int k = 0; k < n_full; ++k) step(k, std::false_type{});
  if (n_full < n_k) step(n_full, std::true_type{});
  if (wm == 0) bare_barrier();
  wait_loads<0>();  // the last loads have left the LDS alone before the workgroup gives it up

  // lane: row 128 (i / 4) + 64 wm + 16 (i % 4) + s, columns 64 wn + 16 j + 4 q .. + 3
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t m = bm * kBT + 128 * (i >> 2) + 64 * wm + 16 * (i & 3) + s;
    if (m >= a.m) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = bn * kBT + 64 * wn + 16 * j + 4 * q;
      if (n < a.n) store4(static_cast<__bf16*>(a.c) + m * a.ld_c + n, acc[i][j], (int)min(a.n - n, (int64_t)4));
    }
  }
}

// Large float32 products: tiles of 256 x 128 by 8 waves of 64 x 64, with the matrix
// instruction for float16.  As in big_kernel, waves 4-7 run half a step behind waves 0-3: on
// every SIMD one wave reads its operands of a block of columns, and waits for the loads to come, while the other
// multiplies.  Three stages in LDS: block k + 2 is requested in the memory part of block k, into the place of block k -
// 1, which every wave has read by then; before the barrier that ends that part a wave waits until
// only these 7 loads are outstanding, so that block k + 1 is there.
constexpr int kWM = 256, kWN = 128, kWRows = kWM + kWN;
constexpr int kWStage = kWRows * 128 + 8 * 64 * 4;  // codes, then a scale of each row (and room to keep 8 waves alike)

template <int FA, int FB, bool ROWS_B>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) wide_kernel(MatArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t stage[3 * kWStage];
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int per_xcd = gridDim.x / 8;
  const int tile = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (tile >= a.tiles_m * a.tiles_n) return;  // whole workgroup
  int64_t bm, bn;
  place(tile, a.tiles_m, a.tiles_n, bm, bn);

  const int64_t am = bm * kWM + 32 * wv, bnr = bn * kWN + 16 * wv;  // rows this wave stages
  const uint8_t* const pa = a.a + am * a.ld_a;
  const uint8_t* const pb = a.b + bnr * a.ld_b;
  const uint32_t len_a = range_bytes(am, a.m, 32, a.ld_a, a.k), len_b = range_bytes(bnr, a.n, 16, a.ld_b, a.k);
  // scales of 64 rows: of A in waves 0-3, of B in waves 4-5 and, to no use, again in 6-7; rows past the last take the last one's
  const bool sc_a = wv < 4;
  const int64_t sc_row = sc_a ? bm * kWM + 64 * wv + lane : bn * kWN + 64 * (wv & 1) + lane;
  const float* sc_at = (sc_a ? a.sa : a.sb) +
                       (min(sc_row, (sc_a ? a.m : a.n) - 1) >> (sc_a ? a.a_shift : a.b_shift)) * (sc_a ? a.sa_row : a.sb_row);
  const int64_t sc_block = sc_a ? a.sa_block : a.sb_block;
  const int n_kb = (int)((a.k + 127) / 128);
  auto request = [&](int kb, int st) {  // past the last block: an empty range, and its scales again
    uint8_t* dst = stage + st * kWStage;
    const bool in = kb < n_kb;
    stage_issue<32, 0>(make_rsrc(pa, in ? len_a : 0u), dst + 128 * 32 * wv, 128u * (uint32_t)kb, (uint32_t)a.ld_a, lane);
    stage_issue<16, 0>(make_rsrc(pb, in ? len_b : 0u), dst + 128 * (kWM + 16 * wv), 128u * (uint32_t)kb,
                       (uint32_t)a.ld_b, lane, 16 * wv);
    __builtin_amdgcn_global_load_lds(sc_at + (in ? kb : n_kb - 1) * sc_block, (lds_void*)(dst + 128 * kWRows + 256 * wv),
                                     4, 0, 0);
  };

  const int wm = wv >> 1, wn = wv & 1;
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto block = [&](int kb, int st, auto last_tag) {
    constexpr bool LAST = decltype(last_tag)::value;  // columns from k on are whatever the rows hold there
    const uint8_t* ta = stage + st * kWStage;
    const uint8_t* tb = ta + kWM * 128;
    const float* sc = reinterpret_cast<const float*>(ta + 128 * kWRows);
    u32x4 fa[4][2], fb[4][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        fa[r][h] = stage_chunk(ta, 64 * wm + 16 * r + s, 4 * h + q);
        fb[r][h] = stage_chunk(tb, 64 * wn + 16 * r + s, 4 * h + q);
      }
    float sa[4];
    f32x4 sb[ROWS_B ? 4 : 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) sa[i] = sc[64 * wm + 16 * i + s];
    if constexpr (ROWS_B) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sb[j] = *reinterpret_cast<const f32x4*>(sc + kWM + 64 * wn + 16 * j + 4 * q);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) sa[i] *= sc[kWM + 64 * wn];
    }
    request(kb + 2, st == 0 ? 2 : st - 1);
    wait_loads<7>();
    bare_barrier();
    if constexpr (LAST) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int keep = (int)(a.k - (int64_t)kb * 128) - 16 * (4 * h + q);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          keep_chunk(fa[r][h], keep);
          keep_chunk(fb[r][h], keep);
        }
      }
    }
    // The 16 sums of the block stay in registers while its columns are widened and multiplied, 32 after 32.  Between the
    // products of 32 columns go, in this order, the conversions of the next 32 and, in the last, the additions to C.
    f32x4 part[4][4];
    f16x8 ha[2][4], hb[2][4];
    auto convert = [&](int h, int u) {  // one of the eight operands of columns 32 h .. + 31
      const int w = 2 * (h & 1), r = u >> 1;
      if (u & 1)
        hb[h & 1][r] = widen<FB>(fb[r][h >> 1][w], fb[r][h >> 1][w + 1]);
      else
        ha[h & 1][r] = widen<FA>(fa[r][h >> 1][w], fa[r][h >> 1][w + 1]);
    };
    auto add = [&](int i, int j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(part[i][j][e], ROWS_B ? sa[i] * sb[j][e] : sa[i], acc[i][j][e]);
    };
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < 8; ++u) convert(0, u);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int i = t & 3, j = t >> 2;
        part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
            hb[h & 1][j], ha[h & 1][i], h == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (h < 3 && (t & 1)) convert(h + 1, t >> 1);
        if (h == 3 && t >= 4) add(t & 3, (t - 4) >> 2);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) add(i, 3);
    __builtin_amdgcn_s_setprio(0);
    bare_barrier();
  };
  request(0, 0);
  request(1, 1);
  wait_loads<7>();
  bare_barrier();
  if (wv >= 4) bare_barrier();  // half a step behind
  int st = 0;
#pragma unroll 1
  for (int kb = 0; kb + 1 < n_kb; ++kb) {
    block(kb, st, std::false_type{});
    st = st == 2 ? 0 : st + 1;
  }
  block(n_kb - 1, st, std::true_type{});
  if (wv < 4) bare_barrier();
  wait_loads<0>();  // the last loads have left the LDS alone before the workgroup gives it up

#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = bm * kWM + 64 * wm + 16 * i + s;
    if (m >= a.m) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t n = bn * kWN + 64 * wn + 16 * j + 4 * q;
      if (n < a.n) store4(static_cast<float*>(a.c) + m * a.ld_c + n, acc[i][j], (int)min(a.n - n, (int64_t)4));
    }
  }
}

// Few rows of A: every byte of B is used once or a few times, so B's rate from memory
// bounds the call, and B goes straight to registers.  A workgroup takes 16 TN rows of B
// against all rows of A (16 TM), its 8 waves every eighth block of columns each;
// their sums meet in LDS and are added in a fixed order.  A wave requests
// AHEAD blocks before it multiplies them; four waves a SIMD keep memory busy meanwhile.
// The matrix cores are idle enough for the float16 instruction, so every block's sum is
// exact to float32 here whatever C's type.  A plain A (PLAIN 1: bf16, 2: float32) that
// fits LDS is quantised by every workgroup for itself, which saves a launch.
constexpr int kFewWaves = 8;
constexpr int64_t kPlainBytes = 48 << 10;  // LDS for the codes and scales of a plain A

struct Chunks {
  u32x4 c[2];  // 32 codes of one row: columns 16 q .. 16 q + 15 of each half of a block
};

// Reads columns c .. c + 15 and c + 64 .. c + 79 of a row.
__device__ __forceinline__ Chunks load_chunks(const uint8_t* row, int c) {
  return Chunks{{*reinterpret_cast<const u32x4*>(row + c), *reinterpret_cast<const u32x4*>(row + c + 64)}};
}

// The same where the row has k codes: columns from k on are zeros.
__device__ __forceinline__ Chunks load_last(const uint8_t* row, int c, int k) {
  Chunks r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    r.c[h] = u32x4{0, 0, 0, 0};
    if (c + 64 * h < k) {
      r.c[h] = *reinterpret_cast<const u32x4*>(row + c + 64 * h);
      keep_chunk(r.c[h], k - c - 64 * h);
    }
  }
  return r;
}

// Codes 8 h .. 8 h + 7 of them as float16.
template <int F>
__device__ __forceinline__ f16x8 widen(const Chunks& r, int h) {
  return widen<F>(r.c[h >> 1][2 * (h & 1)], r.c[h >> 1][2 * (h & 1) + 1]);
}

// Quantises the rows of a plain A into LDS, as the quantiser does: 16 lanes take a block, 8 values each.
template <typename T>
__device__ __forceinline__ void stage_plain(const MatArgs& a, uint8_t* codes, int n_kb) {
  const int k = (int)a.k, m = (int)a.m;
  float* scale = reinterpret_cast<float*>(codes + m * n_kb * 128);
  const int l = threadIdx.x & 15;
#pragma unroll 2
  for (int b = threadIdx.x >> 4; b < m * n_kb; b += 4 * kFewWaves) {
    const int r = b / n_kb, kb = b % n_kb, c = 128 * kb + 8 * l;
    Eight<T> x;
    x.load(reinterpret_cast<const T*>(a.a) + r * a.ld_a + c, c, k);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, x.magnitude(e));
    float sc, inv;
    block_scale(max16(top), format_top(false), sc, inv);
    uint2 w = make_uint2(encode4<false>(x.value(0) * inv, x.value(1) * inv, x.value(2) * inv, x.value(3) * inv),
                         encode4<false>(x.value(4) * inv, x.value(5) * inv, x.value(6) * inv, x.value(7) * inv));
    // zeros past the last column, also of a block that is not finite
    if (c + 8 > k) w = make_uint2(keep_bytes(w.x, k - c), keep_bytes(w.y, k - c - 4));
    *reinterpret_cast<uint2*>(codes + 128 * b + 8 * l) = w;
    if (l == 0) scale[b] = sc;
  }
}

template <int TM, int TN, int PLAIN, int FA, int FB>
__global__ void __launch_bounds__(64 * kFewWaves, TM * TN == 1 ? 4 : 2) few_rows_kernel(MatArgs a) {
  static_assert(PLAIN == 0 || TM <= 2, "a plain A has 32 rows at most");
  constexpr int AHEAD = PLAIN ? 4 : 2;
  __shared__ f32x4 sums[kFewWaves][TM * TN][64];
  extern __shared__ __attribute__((aligned(16))) uint8_t plain_codes[];  // PLAIN: [m][n_kb][128], then scales [m][n_kb]
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int k = (int)a.k, n_kb = (k + 127) / 128, n_full = k / 128;
  const int64_t n0 = (int64_t)blockIdx.x * 16 * TN;
  using T = typename std::conditional<PLAIN == 1, __bf16, float>::type;
  const float* plain_scale = reinterpret_cast<const float*>(plain_codes + (PLAIN ? a.m * n_kb * 128 : 0));

  // rows past the last read the last one's, their results are dropped
  const uint8_t* pa[TM];
  const float* ps[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = min((int64_t)(16 * i + s), a.m - 1);
    pa[i] = PLAIN ? plain_codes + m * n_kb * 128 : a.a + m * a.ld_a;
    ps[i] = PLAIN ? plain_scale + m * n_kb : a.sa + (m >> a.a_shift) * a.sa_row;
  }
  const uint8_t* pb[TN];
  const float* pt[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t n = min(n0 + 16 * j + s, a.n - 1);
    pb[j] = a.b + n * a.ld_b;
    pt[j] = a.sb + (n >> a.b_shift) * a.sb_row;
  }

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  struct Side {
    Chunks b[TN], a[TM];
    float sb[TN], sa[TM];
  };
  auto load = [&](Side& t, int kb, auto last) {
    constexpr bool LAST = decltype(last)::value;  // the block that column k ends in
    const int c = 128 * kb + 16 * q;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      t.b[j] = LAST ? load_last(pb[j], c, k) : load_chunks(pb[j], c);
      t.sb[j] = pt[j][kb * a.sb_block];
    }
    if constexpr (PLAIN == 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        t.a[i] = LAST ? load_last(pa[i], c, k) : load_chunks(pa[i], c);
        t.sa[i] = ps[i][kb * a.sa_block];
      }
    }
  };
  auto multiply = [&](Side& t, int kb) {
    __builtin_amdgcn_sched_barrier(0);  // one block's codes as float16 at a time
    if constexpr (PLAIN != 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        t.a[i] = load_chunks(pa[i], 128 * kb + 16 * q);
        t.sa[i] = ps[i][kb];
      }
    }
    f32x4 part[TM][TN];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      f16x8 ha[TM], hb[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) ha[i] = widen<FA>(t.a[i], h);
#pragma unroll
      for (int j = 0; j < TN; ++j) hb[j] = widen<FB>(t.b[j], h);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              hb[j], ha[i], h == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float sb = __shfl(t.sb[j], 4 * q + e);
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j][e] = fmaf(part[i][j][e], t.sa[i] * sb, acc[i][j][e]);
      }
  };
  // this wave's full blocks wv, wv + 8, ..: `count` of them, in groups of AHEAD
  const int count = n_full > wv ? (n_full - wv + kFewWaves - 1) / kFewWaves : 0, groups = count / AHEAD;
  if constexpr (PLAIN != 0) {
    stage_plain<T>(a, plain_codes, n_kb);
    __syncthreads();
  }
  int kb = wv;
#pragma unroll 1
  for (int g = 0; g < groups; ++g, kb += kFewWaves * AHEAD) {
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
    f32x4 r = sums[0][t][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) r += sums[w][t][lane];
    const int64_t m = 16 * (t / TN) + s, n = n0 + 16 * (t % TN) + 4 * q;
    if (m >= a.m || n >= a.n) continue;
    const int left = (int)min(a.n - n, (int64_t)4);
    if (a.c_bf16)
      store4(static_cast<__bf16*>(a.c) + m * a.ld_c + n, r, left);
    else
      store4(static_cast<float*>(a.c) + m * a.ld_c + n, r, left);
  }
}

// Adds the parts of C, in order, and rounds once.
template <typename TC>
__global__ void __launch_bounds__(256) join_kernel(MatArgs a) {
  const int64_t per_row = a.ld_parts / 4, all = a.m * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / per_row, n = 4 * (i % per_row);
    const float* p = a.parts + m * a.ld_parts + n;
    f32x4 r = *reinterpret_cast<const f32x4*>(p);
    for (int z = 1; z < a.splits; ++z) r += *reinterpret_cast<const f32x4*>(p + z * a.m * a.ld_parts);
    store4(static_cast<TC*>(a.c) + m * a.ld_c + n, r, (int)min(a.n - n, (int64_t)4));
  }
}

// What a call runs: sn_matmul_kernel, and its workgroups of so many threads.
struct Run {
  int32_t kernel, threads;
  int64_t workgroups;
};

template <int FA, int FB, bool ROWS_B>
void launch2(const MatArgs& a, const Run& run, bool bf16, hipStream_t st) {
  const dim3 g((uint32_t)run.workgroups);
  switch (run.kernel) {
    case SN_MATMUL_BIG: return big_kernel<FA, FB, ROWS_B><<<g, 512, 0, st>>>(a);
    case SN_MATMUL_WIDE: return wide_kernel<FA, FB, ROWS_B><<<g, 512, 0, st>>>(a);
    case SN_MATMUL_TILE_8:
      return bf16 ? tile_kernel<FA, FB, ROWS_B, __bf16, 8><<<g, 512, 0, st>>>(a)
                  : tile_kernel<FA, FB, ROWS_B, float, 8><<<g, 512, 0, st>>>(a);
    default:
      return bf16 ? tile_kernel<FA, FB, ROWS_B, __bf16, 4><<<g, 256, 0, st>>>(a)
                  : tile_kernel<FA, FB, ROWS_B, float, 4><<<g, 256, 0, st>>>(a);
  }
}

template <int FA, int FB>
void launch1(const MatArgs& a, const Run& run, bool bf16, hipStream_t st) {
  a.b_shift ? launch2<FA, FB, false>(a, run, bf16, st) : launch2<FA, FB, true>(a, run, bf16, st);
}

void launch_tiles(const MatArgs& a, const Run& run, bool fa, bool fb, bool bf16, hipStream_t st) {
  if (fa)
    fb ? launch1<1, 1>(a, run, bf16, st) : launch1<1, 0>(a, run, bf16, st);
  else
    fb ? launch1<0, 1>(a, run, bf16, st) : launch1<0, 0>(a, run, bf16, st);
  if (a.splits > 1) {
    const dim3 j((uint32_t)std::min<int64_t>((a.m * (a.ld_parts / 4) + 255) / 256, 4096));
    bf16 ? join_kernel<__bf16><<<j, 256, 0, st>>>(a) : join_kernel<float><<<j, 256, 0, st>>>(a);
  }
}

// ------------------------------------------------------------------ host side

using sn::aligned;
using sn::refuse;

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Rows of A up to which there is a kernel for few rows.
constexpr int64_t kFewRows = 64;

// Its cost in us, as in choose(): 256 workgroups at a time, each wave an eighth of the columns, a block
// at 0.66 and 0.015 a row for one tile of 16 rows of A, 2.0, 2.35 and 2.9 for 2 to 4 (1, 16, 24, 40 and 64 rows
// against 8192 x 8192: 13.8, 17.4, 19.3, 21.9 and 26.3; tiles of 128 x 128 with the sum in parts 17.7 for 16 rows, 18.5,
// 19.8 and 20.7; one row against 256 x 16384 11.4 and 17.3).
double few_cost(int64_t m, int64_t n, int64_t k) {
  const int t = (int)((m + 15) / 16);
  const double block = t == 1 ? 0.66 + 0.015 * (double)m : t == 2 ? 2.0 : t == 3 ? 2.35 : 2.9;
  const double wgs = (double)((n + (t == 1 ? 15 : 31)) / (t == 1 ? 16 : 32));
  return std::max(1.0, wgs / 256.0) * (double)(((k + 127) / 128 + kFewWaves - 1) / kFewWaves) * block;
}

// LDS that the codes and scales of a plain A take.
int64_t plain_bytes(int64_t m, int64_t k) { return m * ((k + 127) / 128) * (128 + 4); }

template <int FA, int FB>
void launch_few(const MatArgs& a, const Run& run, int plain, hipStream_t st) {
  const int t = (int)((a.m + 15) / 16);
  const dim3 g((uint32_t)run.workgroups);
  constexpr int W = 64 * kFewWaves;
  if constexpr (FA == 0) {
    const size_t lds = (size_t)plain_bytes(a.m, a.k);
    if (plain == 1)
      return t == 1 ? few_rows_kernel<1, 1, 1, FA, FB><<<g, W, lds, st>>>(a)
                    : few_rows_kernel<2, 1, 1, FA, FB><<<g, W, lds, st>>>(a);
    if (plain == 2)
      return t == 1 ? few_rows_kernel<1, 1, 2, FA, FB><<<g, W, lds, st>>>(a)
                    : few_rows_kernel<2, 1, 2, FA, FB><<<g, W, lds, st>>>(a);
  }
  switch (t) {
    case 1: return few_rows_kernel<1, 1, 0, FA, FB><<<g, W, 0, st>>>(a);
    case 2: return few_rows_kernel<2, 2, 0, FA, FB><<<g, W, 0, st>>>(a);
    case 3: return few_rows_kernel<3, 2, 0, FA, FB><<<g, W, 0, st>>>(a);
    default: return few_rows_kernel<4, 2, 0, FA, FB><<<g, W, 0, st>>>(a);
  }
}

// The kernel of a product of more than kFewRows rows, and over how many workgroups a tile's sum
// is split: the cheapest by these costs in us, each for a block of 128 columns.  Large tiles,
// one workgroup per compute unit: 256 x 256 to bf16 1.75 (8192^3: 427 us, 4096^3
// 60), 256 x 128 to float32 1.85 (1024 x 8192 x 16384: 239).  A 128 x 128 tile alone on its unit 0.67
// (512 x 8192 x 8192: 45), two of them 1.12 (1024 x 8192 x 8192: 72, by the large
// tiles 105), to float32 1.1 and 2.1 (1024 x 8192 x 16384: 264).  Parts are
// written, read and joined at 5.5 TB/s in a launch more: 512 x 512 x 16384 takes 95 us in
// one part, 53, 31 and 22 in 2, 4 and 8; 512 x 8192 x 8192 45 in one part, 53 in two.
struct Way {
  bool big;
  int splits, blocks_per_split;
  double cost;  // without the launch itself
};

Way choose(int64_t m, int64_t n, int64_t k, bool f32) {
  auto up = [](int64_t x, int64_t t) { return (x + t - 1) / t; };
  const int64_t n_kb = up(k, 128), small = up(m, 128) * up(n, 128);
  Way best{false, 1, (int)n_kb, 0.0};
  double cost = 1e30;
  if (n_kb > 0) {
    best.big = true;
    cost = (f32 ? 1.85 * (double)up(up(m, kWM) * up(n, kWN), 256) : 1.75 * (double)up(up(m, kBT) * up(n, kBT), 256)) *
           (double)n_kb;
    best.cost = cost;
  }
  const double alone = f32 ? 1.1 : 0.67, both = f32 ? 2.1 : 1.12;
  for (int64_t s = 1; s <= 16 && (s == 1 || 2 * s <= n_kb); ++s) {
    const int64_t per = up(n_kb, s), wgs = small * s, rest = wgs % 512;
    if (s > 1 && (s - 1) * per >= n_kb) continue;  // a split without blocks
    double c = (double)per * ((double)(wgs / 512) * both + (rest == 0 ? 0.0 : rest <= 256 ? alone : both));
    if (s > 1) c += 4.0 + (double)(8 * s + (f32 ? 4 : 2)) * (double)m * (double)n / 5.5e6;
    if (c < cost) {
      cost = c;
      best = Way{false, (int)s, (int)per, c};
    }
  }
  return best;
}

struct MatPlan {
  Way way;
  Run run;
  int32_t tiles_m, tiles_n;
  int64_t off_parts, ld_parts;
  bool plain_a;
  bool few;   // the kernel for few rows
  bool fuse;  // ... which quantises a plain A itself
  int64_t ld_codes;  // of a plain A's codes
  int64_t off_scale, bytes;
};

// The launch of the kernel that the plan chose.
void set_run(const sn_matmul& p, MatPlan& pl) {
  if (pl.few) {
    const int64_t cols = p.m <= 16 || pl.fuse ? 16 : 32;  // of C that a workgroup takes
    pl.run = Run{SN_MATMUL_FEW_ROWS, 64 * kFewWaves, (p.n + cols - 1) / cols};
    return;
  }
  const bool f32 = p.c_type == SN_F32;
  const int tm = !pl.way.big ? kT : f32 ? kWM : kBT, tn = !pl.way.big ? kT : f32 ? kWN : kBT;
  pl.tiles_m = (int32_t)((p.m + tm - 1) / tm);
  pl.tiles_n = (int32_t)((p.n + tn - 1) / tn);
  const int64_t units = (int64_t)pl.tiles_m * pl.tiles_n * pl.way.splits;
  // a 128 x 128 tile alone on its compute unit: 8 waves (512 x 8192 x 8192 to bf16 48.6 us with 4, 44.6 with 8); else two
  // of 4 (1024 x 8192 x 8192 71.9 with 4, 74.2 with 8)
  const bool eight = pl.way.big || units <= 256;
  pl.run.kernel = !pl.way.big ? (eight ? SN_MATMUL_TILE_8 : SN_MATMUL_TILE_4) : f32 ? SN_MATMUL_WIDE : SN_MATMUL_BIG;
  pl.run.threads = eight ? 512 : 256;
  pl.run.workgroups = (units + 7) / 8 * 8;  // whole rounds of the XCDs
}

// Checks the description and fills in its defaults.
int resolve(sn_matmul& p, MatPlan& pl) {
  const bool plain = p.a_type == SN_F32 || p.a_type == SN_BF16;
  if (!plain && p.a_type != SN_E4M3 && p.a_type != SN_E5M2)
    return refuse(SN_EDTYPE, "a_type must be SN_E4M3, SN_E5M2, SN_F32 or SN_BF16");
  if (p.b_type != SN_E4M3 && p.b_type != SN_E5M2) return refuse(SN_EDTYPE, "b_type must be SN_E4M3 or SN_E5M2");
  if (p.c_type != SN_F32 && p.c_type != SN_BF16) return refuse(SN_EDTYPE, "c_type must be SN_F32 or SN_BF16");
  if (p.m < 0 || p.n < 0 || p.k < 0) return refuse(SN_EINVAL, "m, n and k must be >= 0");
  if ((p.a_block_rows != 1 && p.a_block_rows != 128) || (p.b_block_rows != 1 && p.b_block_rows != 128))
    return refuse(SN_EINVAL, "a_block_rows and b_block_rows must be 1 or 128");
  if (plain && p.a_block_rows != 1) return refuse(SN_EINVAL, "a plain A is quantised by rows: a_block_rows must be 1");
  constexpr int64_t kMost = int64_t(1) << 40, kMostRows = int64_t(1) << 34, kMostLd = int64_t(1) << 22;
  if (p.m > kMostRows || p.n > kMostRows || p.k > kMostLd || p.ld_a > kMost || p.ld_b > kMost || p.ld_c > kMost)
    return refuse(SN_EINVAL, "m, n or a row stride is too large (k and code rows stay below 2^22)");
  if (p.ld_a == 0) p.ld_a = plain ? p.k : round_up(p.k, 16);
  if (p.ld_b == 0) p.ld_b = round_up(p.k, 16);
  if (p.ld_c == 0) p.ld_c = p.n;
  if (p.ld_a < p.k || p.ld_b < p.k || p.ld_c < p.n)
    return refuse(SN_EINVAL, "ld_a and ld_b must be >= k, ld_c >= n");
  if ((!plain && (p.ld_a % 16 || p.ld_a >= kMostLd)) || p.ld_b % 16 || p.ld_b >= kMostLd || p.k >= kMostLd - 128)
    return refuse(SN_EINVAL, "code rows must be multiples of 16 bytes, below 2^22");
  if (p.sa_block == 0 && p.sa_row == 0) {
    p.sa_row = 1;
    p.sa_block = (p.m + p.a_block_rows - 1) / p.a_block_rows;
  }
  if (p.sb_block == 0 && p.sb_row == 0) {
    p.sb_row = 1;
    p.sb_block = (p.n + p.b_block_rows - 1) / p.b_block_rows;
  }
  for (int64_t* s : {&p.sa_block, &p.sa_row, &p.sb_block, &p.sb_row})
    if (*s == SN_STRIDE_ZERO) *s = 0;
  if (p.sa_block < 0 || p.sa_row < 0 || p.sb_block < 0 || p.sb_row < 0 || p.sa_block > kMost || p.sa_row > kMost ||
      p.sb_block > kMost || p.sb_row > kMost)
    return refuse(SN_EINVAL, "scale strides must be >= 0 and below 2^40");
  if (((p.m + 127) / 128) * ((p.n + 127) / 128) >= (int64_t(1) << 22))
    return refuse(SN_EINVAL, "m x n must stay below 2^22 tiles of 128 x 128");
  if (plain && ((p.m + 127) / 128) * ((p.k + 127) / 128) >= (int64_t(1) << 24))
    return refuse(SN_EINVAL, "a plain A must stay below 2^24 tiles of 128 x 128");
  pl = MatPlan{};
  pl.plain_a = plain;
  pl.way = choose(p.m, p.n, p.k, p.c_type == SN_F32);
  // within 2 us the kernel for few rows: its sums are the more exact ones, and it takes a plain A without a launch more
  // (the choice is the same for codes, so that both give the same bits)
  // 512 lanes for 16 columns of C have to stay below the 2^32 of a launch
  pl.few = p.m <= kFewRows && p.m > 0 && p.n <= (int64_t(1) << 27) - 16 &&
           few_cost(p.m, p.n, p.k) <= pl.way.cost + 2.0;
  pl.fuse = pl.few && plain && p.m <= 32 && plain_bytes(p.m, p.k) <= kPlainBytes;
  if (plain && !pl.fuse && p.m > 0 && p.k > 0) {
    pl.ld_codes = round_up(p.k, 16);
    pl.off_scale = round_up(p.m * pl.ld_codes, 256);
    pl.bytes = pl.off_scale + round_up(p.m * ((p.k + 127) / 128) * 4, 256);
  }
  if (!pl.few) {
    if (pl.way.big && (p.sa_row >= (1 << 20) || p.sb_row >= (1 << 20))) pl.way.big = false;
    if (pl.way.splits > 1) {
      pl.off_parts = pl.bytes;
      pl.ld_parts = round_up(p.n, 4);
      pl.bytes += round_up(pl.way.splits * p.m * pl.ld_parts * 4, 256);
    }
  }
  if (p.m > 0 && p.n > 0) set_run(p, pl);
  return SN_OK;
}

}  // namespace

extern "C" SN_API int spectral_matmul_fp8_workspace_bytes(const sn_matmul* desc, int64_t* bytes) {
  if (!desc || !bytes) return refuse(SN_ENULL, "p and bytes must not be NULL");
  sn_matmul p = *desc;
  MatPlan pl;
  if (int rc = resolve(p, pl)) return rc;
  *bytes = pl.bytes;
  return SN_OK;
}

extern "C" SN_API int spectral_matmul_fp8_kernel(const sn_matmul* desc, int32_t* kernel, int32_t* parts,
                                                 int64_t* workgroups, int32_t* threads) {
  if (!desc || !kernel || !parts || !workgroups || !threads)
    return refuse(SN_ENULL, "p, kernel, parts, workgroups and threads must not be NULL");
  sn_matmul p = *desc;
  MatPlan pl;
  if (int rc = resolve(p, pl)) return rc;
  *kernel = pl.run.kernel;
  *parts = pl.run.kernel == 0 ? 0 : pl.few ? 1 : pl.way.splits;
  *workgroups = pl.run.workgroups;
  *threads = pl.run.threads;
  return SN_OK;
}

extern "C" SN_API int spectral_matmul_fp8(const sn_matmul* desc, const void* a, const float* sa, const void* b,
                                          const float* sb, void* c, void* workspace, int64_t workspace_bytes,
                                          void* hip_stream) {
  if (!desc) return refuse(SN_ENULL, "p must not be NULL");
  sn_matmul p = *desc;
  MatPlan pl;
  if (int rc = resolve(p, pl)) return rc;
  if (p.m == 0 || p.n == 0) return SN_OK;
  if (!c || (p.k > 0 && (!a || !b || !sb || (!pl.plain_a && !sa))))
    return refuse(SN_ENULL, "a, sa (of codes), b, sb and c must not be NULL");
  if (pl.plain_a ? !aligned(a, p.a_type == SN_F32 ? 4 : 2) : !aligned(a, 16) || !aligned(sa, 4))
    return refuse(SN_EINVAL, "codes must be 16-byte aligned, a plain A and scales aligned to their type");
  if (!aligned(b, 16) || !aligned(sb, 4) || !aligned(c, p.c_type == SN_F32 ? 4 : 2))
    return refuse(SN_EINVAL, "codes must be 16-byte aligned, scales and C aligned to their type");
  if (pl.bytes > 0) {
    if (!workspace) return refuse(SN_ENULL, "workspace must not be NULL");
    if (workspace_bytes < pl.bytes) return refuse(SN_EINVAL, "workspace too small (spectral_matmul_fp8_workspace_bytes)");
    if (!aligned(workspace, 256)) return refuse(SN_EINVAL, "workspace must be 256-byte aligned");
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = sn::check_stream(st)) return rc;

  MatArgs g{};
  g.a = static_cast<const uint8_t*>(a);
  g.b = static_cast<const uint8_t*>(b);
  g.sa = sa;
  g.sb = sb;
  g.c = c;
  g.m = p.m;
  g.n = p.n;
  g.k = p.k;
  g.ld_a = p.ld_a;
  g.ld_b = p.ld_b;
  g.ld_c = p.ld_c;
  g.sa_block = p.sa_block;
  g.sa_row = p.sa_row;
  g.sb_block = p.sb_block;
  g.sb_row = p.sb_row;
  g.a_shift = p.a_block_rows == 128 ? 7 : 0;
  g.b_shift = p.b_block_rows == 128 ? 7 : 0;
  const bool fa = p.a_type == SN_E5M2, fb = p.b_type == SN_E5M2;
  g.c_bf16 = p.c_type == SN_BF16;
  if (pl.plain_a && !pl.fuse && p.k > 0) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    sn::QuantArgs qa{};
    qa.x = a;
    qa.rows = p.m;
    qa.cols = p.k;
    qa.ld_x = p.ld_a;
    qa.row_codes = ws;
    qa.ld_row = pl.ld_codes;
    qa.row_scale = reinterpret_cast<float*>(ws + pl.off_scale);
    sn::launch_quantize(qa, p.a_type == SN_BF16, false, false, st);
    if (int rc = sn::launched("quantise")) return rc;
    g.a = ws;
    g.ld_a = pl.ld_codes;
    g.sa = qa.row_scale;
    g.sa_block = p.m;
    g.sa_row = 1;
  }
  g.splits = pl.way.splits;
  g.blocks_per_split = pl.way.blocks_per_split;
  g.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + pl.off_parts);
  g.ld_parts = pl.ld_parts;
  g.tiles_m = pl.tiles_m;
  g.tiles_n = pl.tiles_n;
  if (pl.few) {
    const int plain = !pl.fuse ? 0 : p.a_type == SN_BF16 ? 1 : 2;
    if (fa)
      fb ? launch_few<1, 1>(g, pl.run, plain, st) : launch_few<1, 0>(g, pl.run, plain, st);
    else
      fb ? launch_few<0, 1>(g, pl.run, plain, st) : launch_few<0, 0>(g, pl.run, plain, st);
  } else {
    launch_tiles(g, pl.run, fa, fb, g.c_bf16 != 0, st);
  }
  return sn::launched("product");
}
