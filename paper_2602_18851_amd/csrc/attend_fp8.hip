// Attention of single tokens and of trees of drafted tokens over an 8-bit cache (spectral_cache_attend):
//   S = scale q K^T over the places that a token sees, O = softmax(S) V.
//
// The query heads of a key head and the drafted tokens are rows of one product, so the cache is read once for
// all of them.  Every product is formed transposed: S^T = K Q^T, then O^T = V^T P^T.  The columns, one to each
// lane % 16, are query rows, and the places of S^T that a lane holds are those of P^T that the second product
// asks it for, so that P stays in registers.
//
// Codes become bf16 with their row's scale, a power of two, on the way: exactly (bf16 has float32's range; parts of
// values below 2^-126 are lost).  Products of bf16 are exact and summed in float32.  Queries in float32 are three
// parts of bf16 (2^-24), P, in float32 with its running maximum and sum, two parts (2^-16: nothing beside a bf16
// result) or three.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "cache_fp8.h"
#include "device_util.h"
#include "fp8_device.h"
#include "tile_device.h"

namespace {

using namespace sn_dev;
using sn::CacheView;

constexpr int kStep = 32;   // places that a wave of attend_kernel takes at a time
constexpr int kTreeWaves = 8;

struct AttendArgs {
  CacheView c;
  const void* q;
  void* out;
  int64_t q_batch, q_draft, q_head, out_batch, out_draft, out_head;
  const int32_t* table;
  int64_t table_ld;
  const int32_t* lengths;
  const int64_t* masks;  // or NULL: a drafted token sees those before it and itself
  int64_t mask_batch;
  int32_t batch, drafts, group, rows;  // rows = drafts * group, of a key head
  int32_t max_places, step;  // step: places that go together
  int32_t row_waves, row_blocks;  // waves of a workgroup with rows of their own, and workgroups that share a key head's rows
  int32_t strands;                // key heads times row_blocks
  int32_t target, least;          // workgroups to aim at, and the least steps of one
  float c_log2;                   // scale * log2(e)
  uint32_t* plan;                 // [batch + 1] chunks of the sequences before each one, or NULL: every workgroup finds them
  float* part_out;                // [unit][rows of a workgroup][head_dim], where a sequence is split
  float2* part_stat;              // maximum and sum of each row
};

constexpr float kNone = -__builtin_inff();

// ---- how the places are shared out --------------------------------------
//
// Lengths are known on the device only, and every workgroup derives the same plan from them: all sequences' steps (one
// at least to a sequence), over `target` workgroups, give the steps of one (`least` at least, which hide its start and
// end); a sequence is cut into as many equal chunks as come nearest to that, one at least.  A unit, a chunk of one
// key head's rows, is one workgroup's.  Of more than kScanned sequences plan_kernel forms the same plan once, and every
// workgroup looks its chunk up: workgroups that scan all sequences grow with the square of their number.

__device__ __forceinline__ int length_of(const AttendArgs& a, int b) { return min(max(a.lengths[b], 0), a.max_places); }

// Steps of sequence b, none past the last one.
__device__ __forceinline__ uint32_t steps_of(const AttendArgs& a, int b) {
  return b < a.batch ? max(1u, ((uint32_t)length_of(a, b) + (uint32_t)a.step - 1) / (uint32_t)a.step) : 0u;
}

// Sums over the lanes up to and with each.
__device__ __forceinline__ uint32_t scan64(uint32_t x) {
#define SN_ADD(ctrl, rows) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false)
  SN_ADD(0x111, 0xf);  // from 1, 2, 4 and 8 lanes down in each row of 16
  SN_ADD(0x112, 0xf);
  SN_ADD(0x114, 0xf);
  SN_ADD(0x118, 0xf);
  SN_ADD(0x142, 0xa);  // from the last lane of the row below, and of the lower half
  SN_ADD(0x143, 0xc);
#undef SN_ADD
  return x;
}
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}

// `steps` over chunks of about `per`.
__device__ __forceinline__ uint32_t chunks_of(uint32_t steps, uint32_t per) {
  return steps == 0 ? 0u : max(1u, (steps + per / 2) / per);
}

// Steps that a unit should have, of all sequences'.
__device__ __forceinline__ uint32_t per_of(const AttendArgs& a, uint32_t all) {
  return max((all * (uint32_t)a.strands + (uint32_t)a.target - 1) / (uint32_t)a.target, (uint32_t)a.least);
}

struct Plan {
  uint32_t steps0;  // of sequence `lane`
  uint32_t per;     // steps that a unit should have
};

__device__ __forceinline__ Plan plan_of(const AttendArgs& a, int lane) {
  Plan p;
  p.steps0 = steps_of(a, lane);
  uint32_t all = lane_of(scan64(p.steps0), 63);
  for (int b0 = 64; b0 < a.batch; b0 += 64) all += lane_of(scan64(steps_of(a, b0 + lane)), 63);
  p.per = per_of(a, all);
  return p;
}

// The plan of many sequences, by one workgroup.  8 key heads of 128, 32-256 places each, one token: 512 sequences 70 us, 1024 137
// and 4096 549, by workgroups that scan them all 88, 226 and 1994 (16384 of 256 places: 33.7 ms); 256 sequences 40 and 42, and
// with one key head, where its launch counts, 13 and 10.5.
constexpr int kScanned = 256;
constexpr int kPlanWaves = 16, kPlanEach = 4;  // waves of its workgroup; sequences of a lane at a time

__global__ void __launch_bounds__(64 * kPlanWaves) plan_kernel(AttendArgs a) {
  __shared__ uint32_t sums[kPlanWaves];
  const int t = threadIdx.x, lane = t & 63, wv = t >> 6;
  // sums over the lanes up to and with each, and over all
  auto scan = [&](uint32_t x, uint32_t& all) {
    x = scan64(x);
    __syncthreads();  // the sums before have been read
    if (lane == 63) sums[wv] = x;
    __syncthreads();
    all = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
      x += w < wv ? sums[w] : 0u;
      all += sums[w];
    }
    return x;
  };
  uint32_t steps = 0, all;
  for (int b = t; b < a.batch; b += 64 * kPlanWaves) steps += steps_of(a, b);
  scan(steps, all);
  const uint32_t per = per_of(a, all);
  uint32_t base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64 * kPlanWaves * kPlanEach) {
    const int b = b0 + kPlanEach * t;
    uint32_t n[kPlanEach], mine = 0;
#pragma unroll
    for (int e = 0; e < kPlanEach; ++e) mine += n[e] = chunks_of(steps_of(a, b + e), per);
    uint32_t at = base + scan(mine, all) - mine;
#pragma unroll
    for (int e = 0; e < kPlanEach; ++e) {
      if (b + e < a.batch) a.plan[b + e] = at;
      at += n[e];
    }
    base += all;
  }
  if (t == 0) a.plan[a.batch] = base;
}

// The sequence of chunk n of plan[batch]: each look of the 64 lanes leaves a 64th of the sequences.
__device__ __forceinline__ int sequence_of(const AttendArgs& a, uint32_t n, int lane) {
  int lo = 0, hi = a.batch;  // plan[lo] <= n < plan[hi]
  while (hi - lo > 1) {
    const int apart = (hi - lo + 63) / 64, at = lo + (lane + 1) * apart;
    const uint64_t up_to = __ballot(at < hi && a.plan[min(at, hi)] <= n);
    lo += __builtin_popcountll(up_to) * apart;
    hi = min(hi, lo + apart);
  }
  return lo;
}

// The unit of this workgroup.
struct Unit {
  int b, h, rb, len, n_chunks, step0, step1;  // steps from step0 to step1 - 1
};

__device__ __forceinline__ bool find_unit(const AttendArgs& a, int lane, Unit& u) {
  uint32_t in = 0, steps = 0, n = 0;  // in: units of the sequence before this one; n: its chunks
  int b = -1;
  if (a.plan) {
    const uint32_t at = blockIdx.x / (uint32_t)a.strands;
    if (at >= a.plan[a.batch]) return false;
    b = sequence_of(a, at, lane);
    const uint32_t before = a.plan[b];
    steps = steps_of(a, b);
    n = a.plan[b + 1] - before;
    in = blockIdx.x - before * (uint32_t)a.strands;
  } else {
    const Plan p = plan_of(a, lane);
    uint32_t base = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      const uint32_t s = b0 == 0 ? p.steps0 : steps_of(a, b0 + lane);
      const uint32_t mine = chunks_of(s, p.per) * (uint32_t)a.strands, sum = scan64(mine);
      const uint64_t there = __ballot(blockIdx.x < base + sum);
      if (there) {
        const int at = __builtin_ctzll(there);
        b = b0 + at;
        steps = lane_of(s, at);
        n = chunks_of(steps, p.per);
        in = blockIdx.x - (base + lane_of(sum, at) - lane_of(mine, at));
        break;
      }
      base += lane_of(sum, 63);
    }
    if (b < 0) return false;
  }
  const uint32_t chunk = in / (uint32_t)a.strands, strand = in % (uint32_t)a.strands;
  const uint32_t per = (steps + n - 1) / n;
  u.b = uni(b);
  u.h = uni((int)(strand % (uint32_t)a.c.heads));
  u.rb = uni((int)(strand / (uint32_t)a.c.heads));
  u.len = uni(length_of(a, b));
  u.n_chunks = uni((int)n);
  u.step0 = uni((int)min(steps, chunk * per));
  u.step1 = uni((int)min(steps, chunk * per + per));
  return true;
}

// ---- arithmetic ------------------------------------------------------------

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The bf16 parts of eight values, the nearest first.
template <int PARTS>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&part)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    f32x2 rest = {x[e], x[e + 1]};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const bf16x2 near = __builtin_convertvector(rest, bf16x2);
      part[p][e] = near[0];
      part[p][e + 1] = near[1];
      const uint32_t w = __builtin_bit_cast(uint32_t, near);
      if (p + 1 < PARTS) rest = f32x2{rest[0] - __uint_as_float(w << 16), rest[1] - __uint_as_float(w & 0xffff0000u)};
    }
  }
}

// Codes 0, 1 or 2, 3 of a word, times 2^e of the scale, as bf16.
template <bool E5M2, bool HIGH>
__device__ __forceinline__ uint32_t widen2(uint32_t w, float scale) {
  if constexpr (E5M2)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, HIGH));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}

__device__ __forceinline__ f32x4 multiply(const bf16x8& x, const bf16x8& y, const f32x4& sum) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, sum, 0, 0, 0);
}

// Over the four quarters of a wave, lanes with one lane % 16.
__device__ __forceinline__ float quarters_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quarters_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A row's running maximum is raised, and its sums scaled, only when a logit is above it by a factor of 2^kSlack in weight: until
// then weights are up to 2^kSlack, which float32 and bf16 hold as exactly.
constexpr float kSlack = 8.f;

// exp2 of the distance to a running maximum; a row that has seen nothing has none.
__device__ __forceinline__ float weight_of(float m, float to, float c) {
  return m == kNone ? 0.f : __builtin_amdgcn_exp2f((m - to) * c);
}

// Elements d .. d + 3 of row r of sequence b from their sums.
template <typename T>
__device__ __forceinline__ void store_row4(const AttendArgs& a, int b, int h, int r, int d, const f32x4& x) {
  typedef T vec __attribute__((ext_vector_type(4)));
  typedef vec vec_any __attribute__((aligned(sizeof(T))));
  const int i = r / a.group, g = r % a.group;
  const int64_t at = b * a.out_batch + i * a.out_draft + ((int64_t)h * a.group + g) * a.out_head + d;
  *reinterpret_cast<vec_any*>(static_cast<T*>(a.out) + at) = vec{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
}

// Waves of a workgroup of attend_kernel.
constexpr int kWaves = 4;

// Up to 64 rows of a key head (float32 queries and head_dim above 128: any number): bound by memory, so codes go straight
// to registers.  Four waves of NT blocks of 16 rows; those with the same rows take every so many steps of the chunk, and
// their results meet in LDS.  The keys of the next step are on their way while this one's weights are formed and its values
// multiplied.  One token at the end of 131071 places, 8 key heads of 128 with 8 query heads each: 47-49 us (5.7 TB/s), and 10
// for the join and its launch; with 8 waves to a workgroup, one on a compute unit in place of two, 81 us in all.
// D: head_dim rounded up to 64, 128 or 256.  Lane q * 16 + s of a wave holds
//   of K: places s of each of two groups of 16, bytes 16 q .. + 15 of every 64;
//   of V: places 4 q .. 4 q + 3 of each group, D / 16 bytes from D / 16 s on;
//   of S^T and P^T: those places of V for row s of each block;
//   of O^T: for row s, D / 4 elements from D / 4 q on.
template <int D, bool E5M2, bool F32, int NT>
__global__ void __launch_bounds__(64 * kWaves, D == 256 || NT * D * (F32 ? 2 : 1) > 256 ? 1 : 2)
attend_kernel(AttendArgs a) {
  constexpr int W = kWaves, KC = D / 64, VB = D / 16, QP = F32 ? 3 : 1, PP = F32 ? 3 : 2;
  constexpr int REGS = NT * (D / 4 + 2);  // of a wave's result: O, maximum, sum
  __shared__ float merge[W / 2][REGS][64];
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int q = lane >> 4, s = lane & 15;
  const int dh = a.c.head_dim, T = a.drafts;

  Unit unit;
  if (!find_unit(a, lane, unit)) return;  // whole workgroup: past the last one
  const int b = unit.b, h = unit.h, rb = unit.rb, len = unit.len, n_chunks = unit.n_chunks;
  const int step0 = unit.step0, step1 = unit.step1;

  const int rw = wv % a.row_waves, part = wv / a.row_waves, parts = W / a.row_waves;
  const int row0 = (rb * a.row_waves + rw) * 16 * NT;  // this wave's rows
  const bool rows_there = row0 < a.rows;

  // queries and what each sees of the drafted tokens
  bf16x8 qf[NT][KC][2][QP];
  uint64_t sees[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = row0 + 16 * n + s, i = min(r, a.rows - 1) / a.group, g = min(r, a.rows - 1) % a.group;
    const int64_t at = b * a.q_batch + i * a.q_draft + ((int64_t)h * a.group + g) * a.q_head;
    sees[n] = a.masks ? (uint64_t)a.masks[b * a.mask_batch + i] : ((uint64_t)2 << i) - 1;
    sees[n] &= ~(uint64_t)0 >> (64 - T);
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int d = 64 * c + 16 * q + 8 * u;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (d < dh && r < a.rows) {
          if constexpr (F32) {
            Eight<float> v;
            v.load(static_cast<const float*>(a.q) + at + d, 0, 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = v.value(e);
          } else {
            Eight<__bf16> v;
            v.load(static_cast<const __bf16*>(a.q) + at + d, 0, 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = v.value(e);
          }
        }
        split8<QP>(x, qf[n][c][u]);
      }
  }

  // One step's part of the cache in registers.  Elements from head_dim on are out of range of a load and read zeros, and so
  // does all of a step past the last.
  u32x4 kc[2][KC];
  float ks[2];
  uint32_t vc[2][4][VB / 4];
  f32x4 vs[2];
  constexpr uint32_t kNowhere = 0x80000000u;
  uint32_t k_off[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) k_off[c] = 64 * c + 16 * q < dh ? (uint32_t)(s * dh + 64 * c + 16 * q) : kNowhere;
  const uint32_t v_off = VB * s < dh ? (uint32_t)(4 * q * dh + VB * s) : kNowhere;
  const int count = rows_there && step1 - step0 > part ? (step1 - step0 - part + parts - 1) / parts : 0;
  int page_a = -1, page_b = -1;  // lane l: pages of this wave's step l of the current 64
  int ids[2];                    // of the step whose keys were requested last
  auto place_of = [&](int i) { return (int)((uint32_t)(step0 + part + parts * i) * kStep); };
  auto base_of = [&](int i, int g, int64_t& page) {
    // a group without a page reads page 0, to no use
    const int id = ids[g];
    page = id >= 0 ? id : 0;
    return (h << a.c.page_shift) + (id >= 0 ? (place_of(i) + 16 * g) & (a.c.page - 1) : 0);
  };
  auto load_k = [&](int i) {  // this wave's step i, in order
    if ((i & 63) == 0) {
      auto page_of = [&](int64_t place) {
        int id = -1;
        if (place >= 0 && place < len) id = a.table[b * a.table_ld + (place >> a.c.page_shift)];
        return id >= 0 && id < a.c.pages ? id : -1;
      };
      const int64_t mine = (int64_t)(step0 + part) + (int64_t)parts * (i + lane);
      page_a = page_of(mine < step1 ? mine * kStep : -1);
      page_b = page_of(mine < step1 ? mine * kStep + 16 : -1);
    }
    const uint32_t bytes = i < count ? 0x7fffffffu : 0u;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      ids[g] = __builtin_amdgcn_readlane(g ? page_b : page_a, i & 63);
      int64_t page;
      const int in = base_of(i, g, page);
      const __amdgpu_buffer_rsrc_t r = make_rsrc(a.c.k + page * a.c.code_page + (int64_t)in * dh, bytes);
#pragma unroll
      for (int c = 0; c < KC; ++c)
        kc[g][c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, k_off[c], 0, 0));
      ks[g] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
          make_rsrc(a.c.k_scale + page * a.c.scale_page + in, bytes), 4u * (uint32_t)s, 0, 0));
    }
  };
  auto load_v = [&](int i) {  // after load_k(i)
    const uint32_t bytes = i < count ? 0x7fffffffu : 0u;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      int64_t page;
      const int in = base_of(i, g, page);
      const __amdgpu_buffer_rsrc_t r = make_rsrc(a.c.v + page * a.c.code_page + (int64_t)in * dh, bytes);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (VB == 4) {
          vc[g][e][0] = __builtin_amdgcn_raw_buffer_load_b32(r, v_off, (uint32_t)(e * dh), 0);
        } else if constexpr (VB == 8) {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, v_off, (uint32_t)(e * dh), 0));
          vc[g][e][0] = x[0], vc[g][e][1] = x[1];
        } else {
          const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, v_off, (uint32_t)(e * dh), 0));
#pragma unroll
          for (int w = 0; w < 4; ++w) vc[g][e][w] = x[w];
        }
      }
      vs[g] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                            make_rsrc(a.c.v_scale + page * a.c.scale_page + in, bytes),
                                            16u * (uint32_t)q, 0, 0));
    }
  };

  f32x4 acc[NT][VB];
  float top[NT], total[NT];  // total: of the places that this lane holds
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    top[n] = kNone;
    total[n] = 0.f;
#pragma unroll
    for (int j = 0; j < VB; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c_log2 = a.c_log2;
  f32x4 st[NT][2];
  bf16x8 pf[NT][PP];
  uint32_t seen[NT];  // bit 4 g + e

  auto scores = [&]() {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
#pragma unroll
      for (int n = 0; n < NT; ++n) st[n][g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if constexpr (NT > 1) __builtin_amdgcn_sched_barrier(0);  // a few converted values at a time
          const uint32_t w0 = kc[g][c][2 * u], w1 = kc[g][c][2 * u + 1];
          const u32x4 wide = {widen2<E5M2, false>(w0, ks[g]), widen2<E5M2, true>(w0, ks[g]),
                              widen2<E5M2, false>(w1, ks[g]), widen2<E5M2, true>(w1, ks[g])};
          const bf16x8 kf = __builtin_bit_cast(bf16x8, wide);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int p = QP - 1; p >= 0; --p) st[n][g] = multiply(kf, qf[n][c][u][p], st[n][g]);
        }
    }
  };
  auto hide = [&](int place, bool there0, bool there1) {  // what a row does not see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      seen[n] = 0;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        // four places from drafted token j on: ones before the first, zeros past the last
        const int j = place + 16 * g + 4 * q - (len - T);
        const int before = min(max(-j, 0), 4);
        const uint32_t of_tree = (uint32_t)(sees[n] >> min(max(j, 0), 63)) << before | ((1u << before) - 1u);
        const uint32_t four = (g ? there1 : there0) & (j < 64) ? of_tree & 15u : 0u;
        seen[n] |= four << (4 * g);
        f32x4 of_seen;
#pragma unroll
        for (int e = 0; e < 4; ++e) of_seen[e] = four >> e & 1u ? st[n][g][e] : kNone;
        st[n][g] = of_seen;
      }
    }
  };
  auto weights = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float m = fmaxf(fmaxf(fmaxf(st[n][0][0], st[n][0][1]), fmaxf(st[n][0][2], st[n][0][3])),
                      fmaxf(fmaxf(st[n][1][0], st[n][1][1]), fmaxf(st[n][1][2], st[n][1][3])));
      m = quarters_max(m);
      if (__ballot((m - top[n]) * c_log2 > kSlack)) {
        m = fmaxf(m, top[n]);
        const float w = weight_of(top[n], m, c_log2);
        total[n] *= w;
#pragma unroll
        for (int j = 0; j < VB; ++j) acc[n][j] *= w;
        top[n] = m;
      }
      const float base = top[n] == kNone ? 0.f : top[n] * c_log2;
      // Weights join the lane's sum in eights, as the matrix cores add their products to the result: one by one, thousands of
      // small ones are lost beside a large one (140 steps, a weight of 1 and others just below 2^-24: 7.1e-5 off, now 4.9e-6).
      float p[8], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(st[n][e >> 2][e & 3], c_log2, -base));
        sum += p[e];
      }
      total[n] += sum;
      split8<PP>(p, pf[n]);
    }
  };
  // V, place by place, to pairs of places of one element each: place pairs 01 and 23 of both groups, of elements 4 w .. + 3
  auto widen = [&](int w, u32x4 (&vt)[4]) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        uint32_t x[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[e][0] = widen2<E5M2, false>(vc[g][2 * h2 + e][w], vs[g][2 * h2 + e]);
          x[e][1] = widen2<E5M2, true>(vc[g][2 * h2 + e][w], vs[g][2 * h2 + e]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          vt[2 * u][2 * g + h2] = __builtin_amdgcn_perm(x[1][u], x[0][u], 0x05040100u);
          vt[2 * u + 1][2 * g + h2] = __builtin_amdgcn_perm(x[1][u], x[0][u], 0x07060302u);
        }
      }
  };
  // Values that are not finite reach only the rows that see them: in steps that not all rows see they count as zeros,
  // and whoever sees one gets NaN afterwards.
  auto bad_of = [](uint32_t v) {
    return ((v & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((v & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
  };
  auto values = [&](bool edge) {
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < VB / 4; ++w) {
      if constexpr (NT > 1) __builtin_amdgcn_sched_barrier(0);  // a few converted values at a time
      u32x4 vt[4];
      widen(w, vt);
      if (edge) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t bad = bad_of(vt[j][x]);
            any |= bad;
            vt[j][x] &= ~bad;
          }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int p = PP - 1; p >= 0; --p)
            acc[n][4 * w + j] = multiply(__builtin_bit_cast(bf16x8, vt[j]), pf[n][p], acc[n][4 * w + j]);
    }
    if (edge && __ballot(any != 0)) {
#pragma unroll
      for (int w = 0; w < VB / 4; ++w) {
        u32x4 vt[4];
        widen(w, vt);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u32x4 ones;
#pragma unroll
          for (int x = 0; x < 4; ++x) ones[x] = bad_of(vt[j][x]) & 0x3f803f80u;  // 1 in bf16
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            u32x4 who;
#pragma unroll
            for (int x = 0; x < 4; ++x)
              who[x] = (seen[n] >> (2 * x) & 1 ? 0x3f80u : 0u) | (seen[n] >> (2 * x + 1) & 1 ? 0x3f800000u : 0u);
            const f32x4 n_bad = multiply(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, who),
                                         f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[n][4 * w + j][e] = n_bad[e] > 0.f ? __uint_as_float(0x7fc00000u) : acc[n][4 * w + j][e];
          }
        }
      }
    }
  };

  // The keys of the next step are on their way while this one's weights are formed and its values multiplied, the next values
  // while the next scores are.
  if (count > 0) {
    load_k(0);
    __builtin_amdgcn_sched_barrier(0);  // requested in the order of the loop, or this would wait for all of them
    load_v(0);
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const bool there0 = ids[0] >= 0, there1 = ids[1] >= 0;
      const int place = place_of(i);
      scores();
      load_k(i + 1);
      // all places of the step are seen by every row, unless it holds drafted tokens, the end, or lacks a page
      const bool edge = !there0 || !there1 || (int64_t)place + kStep > len - T;
      if (edge) hide(place, there0, there1);
      weights();
      values(edge);
      __builtin_amdgcn_sched_barrier(0);
      load_v(i + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // the parts' results meet in LDS, half of them at a time, lane for lane
#pragma unroll 1
  for (int half = parts / 2; half >= 1; half /= 2) {
    float(*at)[64] = merge[(part - (part >= half ? half : 0)) * a.row_waves + rw];
    if (part >= half && part < 2 * half) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        at[n * (D / 4 + 2)][lane] = top[n];
        at[n * (D / 4 + 2) + 1][lane] = total[n];
#pragma unroll
        for (int j = 0; j < VB; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) at[n * (D / 4 + 2) + 2 + 4 * j + e][lane] = acc[n][j][e];
      }
    }
    __syncthreads();
    if (part < half) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float other = at[n * (D / 4 + 2)][lane], m = fmaxf(top[n], other);
        const float w0 = weight_of(top[n], m, c_log2), w1 = weight_of(other, m, c_log2);
        top[n] = m;
        total[n] = total[n] * w0 + at[n * (D / 4 + 2) + 1][lane] * w1;
#pragma unroll
        for (int j = 0; j < VB; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[n][j][e] = acc[n][j][e] * w0 + at[n * (D / 4 + 2) + 2 + 4 * j + e][lane] * w1;
      }
    }
    __syncthreads();
  }
  if (part != 0 || !rows_there) return;

#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = row0 + 16 * n + s;
    const float sum = quarters_sum(total[n]);
    if (r >= a.rows) continue;
    if (n_chunks > 1) {
      const int64_t at = (int64_t)blockIdx.x * (16 * NT * a.row_waves) + 16 * NT * rw + 16 * n + s;
      if (q == 0) a.part_stat[at] = make_float2(top[n], sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (VB * (4 * q + e) < dh)
#pragma unroll
          for (int j = 0; j < VB; j += 4)
            *reinterpret_cast<f32x4*>(a.part_out + at * dh + VB * (4 * q + e) + j) =
                f32x4{acc[n][j][e], acc[n][j + 1][e], acc[n][j + 2][e], acc[n][j + 3][e]};
      }
      continue;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (VB * (4 * q + e) < dh)
#pragma unroll
        for (int j = 0; j < VB; j += 4)
          store_row4<typename std::conditional<F32, float, __bf16>::type>(
              a, b, h, r, VB * (4 * q + e) + j,
              f32x4{acc[n][j][e], acc[n][j + 1][e], acc[n][j + 2][e], acc[n][j + 3][e]} * inv);
    }
  }
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 multiply32(const bf16x8& x, const bf16x8& y, const f32x16& sum) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, sum, 0, 0, 0);
}

// Many rows of bf16 (trees of drafted tokens): the matrix cores and the exponentials bound the call.  8 waves of 32 rows share
// tiles of 8192 / D places, which they widen to bf16 together, once: K to LDS place by place, V turned, so that a lane's eight
// places of P^T are 16 bytes of a row of V^T.  With 128 rows or less, PARTS 2: pairs of waves have the same rows and half
// of a tile's places each.  Products of 32 x 32: lane 32 hi + s holds
//   of K and Q: row s, elements 8 hi .. + 7 of every 16;
//   of S^T and O^T: for row s of Q, rows 8 i + 4 hi .. + 3, i < 4, of every 32.
// A wave takes half a tile at a time, a step: with PARTS 1 one half after the other, with PARTS 2 its own.  A step falls into
// a part on the matrix cores, O += P V of step k - 1 and S of step k, and one on the vector units, P of step k, with a bare
// barrier after each, and waves 4-7 run one part behind waves 0-3: on every SIMD one wave multiplies while the other
// exponentiates.  With the vector part goes a share of a tile to LDS, where K and V have two places each.  Counting
// parts, waves 0-3 multiply step k in part 2 k, waves 4-7 in part 2 k + 1.
//   PARTS 1: K of tile i + 1 is first read in part 4 i + 4, K of i - 1 last in 4 i - 1; V of i + 1 first at the end of 4 i
//   + 5, V of i - 1 last in 4 i + 1.  All waves write K of i + 1 with step 2 i, in parts 4 i + 1 and 4 i + 2, and V of i + 1 with
//   step 2 i + 1, in 4 i + 3 and 4 i + 4.
//   PARTS 2, both with each step: K of i + 1 and V of i are first read in 2 i + 2, K of i - 1 and V of i - 2 last in 2 i - 1;
//   waves 0-3 write them in 2 i + 1, waves 4-7, a tile ahead, in 2 i.
// Tiles past the last are loaded and written too, to no use, so that no load in flight meets a branch: the compiler would
// wait for all of them there (with branches 677 us in the case below, without 483).
// 16 sequences of 64 tokens, 8 key heads of 128 with 8 query heads each, over 8000-8192 places: 381-412 us by the chip.  The matrix
// products alone take 263 (1.55 PFLOP/s with P in two parts, at the clock that power leaves, the rate of a large bf16
// product); one part of P 335, with twice the rounding error of the result's type.  Addresses are scalar work that
// goes beside the matrix products (420 us with the vector part), whose waves have the lower priority.
constexpr int tile_of(int d) { return 8192 / d; }

template <int D, bool E5M2, int PARTS>
__global__ void __launch_bounds__(64 * kTreeWaves, 2) tree_kernel(AttendArgs a) {
  constexpr int kTile = tile_of(D), kGroups = kTile / 16;
  constexpr int KS = D / 16, DB = D / 32, NB = kTile / 64;
  constexpr int kBytes = kTile * D * 2;  // of K or of V in LDS
  constexpr int REGS = 16 * DB + 2;      // of a wave's result
  constexpr int kMerge = PARTS == 1 ? 0 : kTreeWaves / 2 * REGS * 256;
  __shared__ __attribute__((aligned(16))) uint8_t tiles[4 * kBytes > kMerge ? 4 * kBytes : kMerge];  // K, K, V, V
  // which values of a tile that not all rows see are not finite (in LDS they are zeros): of places 4 f .. + 3 and elements
  // 4 g .. + 3, bit 4 place + element of word [f][g]; looked through two words at a time
  __shared__ __attribute__((aligned(4))) uint16_t bad[2][kTile * D / 16];
  const int lane = threadIdx.x & 63;
  const int wv = uni((int)(threadIdx.x >> 6));
  const int hi = lane >> 5, s = lane & 31;
  const int dh = a.c.head_dim, T = a.drafts;
  Unit unit;
  if (!find_unit(a, lane, unit)) return;  // whole workgroup: past the last one
  const int b = unit.b, h = unit.h, len = unit.len;
  const int rw = wv % (kTreeWaves / PARTS), part = PARTS == 1 ? 0 : wv / (kTreeWaves / PARTS);
  const int row = (unit.rb * (kTreeWaves / PARTS) + rw) * 32 + s;  // this lane's

  bf16x8 qf[KS];
  const int draft = min(row, a.rows - 1) / a.group, in_group = min(row, a.rows - 1) % a.group;
  uint64_t sees = a.masks ? (uint64_t)a.masks[b * a.mask_batch + draft] : ((uint64_t)2 << draft) - 1;
  sees &= ~(uint64_t)0 >> (64 - T);
  {
    const __bf16* q = static_cast<const __bf16*>(a.q) + b * a.q_batch + draft * a.q_draft +
                      ((int64_t)h * a.group + in_group) * a.q_head;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      Eight<__bf16> v;
      v.clear();
      const int d = 16 * k + 8 * hi;
      if (d < dh && row < a.rows) v.load(q + d, 0, 8);
      qf[k] = __builtin_bit_cast(bf16x8, v.w[0]);
    }
  }

  // Pages: lane l holds that of group l % kGroups of tile l / kGroups of a window of tiles, the current one, the one
  // before (of which V and P are still to come) and the next.
  constexpr int kWindow = 64 / kGroups;
  const int count = unit.step1 - unit.step0;
  auto pages_of = [&](int window) {
    const int64_t place = ((int64_t)unit.step0 + window * kWindow) * kTile + 16 * lane;
    int id = -1;
    if (place < len) id = a.table[b * a.table_ld + (place >> a.c.page_shift)];
    return id >= 0 && id < a.c.pages ? id : -1;
  };
  int window = 0, ids_before = -1, ids = pages_of(0), ids_next = pages_of(1);
  // this wave's share of a tile: kTile / 8 places, in one group
  constexpr int kShare = kTile / 8;
  auto locate = [&](int i, int64_t& page, int& in) {
    const int at = kGroups * (i % kWindow) + wv * kShare / 16;
    const int id = i / kWindow == window ? __builtin_amdgcn_readlane(ids, at) : __builtin_amdgcn_readlane(ids_before, at);
    // a group without a page reads page 0, to no use
    const int place = (int)((uint32_t)(unit.step0 + i) * kTile) + kShare * wv;
    in = (h << a.c.page_shift) + (id >= 0 ? place & (a.c.page - 1) : kShare * wv & 15);
    page = id >= 0 ? id : 0;
  };
  auto there_of = [&](int i) {  // bit g: group g of tile i has a page
    const uint64_t all = i / kWindow == window ? __ballot(ids >= 0) : __ballot(ids_before >= 0);
    return (uint32_t)(all >> (kGroups * (i % kWindow))) & ((1u << kGroups) - 1u);
  };
  auto edge_of = [&](int i) {  // whether not all rows see all of tile i
    return there_of(i) != (1u << kGroups) - 1u || (int64_t)(unit.step0 + i + 1) * kTile > len - T;
  };
  // 16 codes of K of one place, 4 of V of each of 4 places, on their way to LDS
  u32x4 kc;
  uint32_t vc[4];
  float ks;
  f32x4 vs;
  constexpr int KL = D / 16, VL = D / 4;  // lanes of a place, of four places
  const int k_place = lane / KL, k_at = 16 * (lane % KL), v_four = lane / VL, v_at = 4 * (lane % VL);
  // byte offsets from the share's first place; elements from head_dim on are out of range and read zeros
  constexpr uint32_t kNowhere = 0x80000000u;
  const uint32_t k_off = k_at < dh ? (uint32_t)(k_place * dh + k_at) : kNowhere;
  const uint32_t v_off = v_at < dh ? (uint32_t)(4 * v_four * dh + v_at) : kNowhere;
  auto from = [](const void* p) { return make_rsrc(p, 0x7fffffffu); };
  // Where tile i's keys (in order) and values are: scalar work, which goes with the matrix cores'.
  const uint8_t *k_from, *v_from;
  const float *ks_from, *vs_from;
  auto find_k = [&](int i) {
    if (i / kWindow != window) {
      ++window;
      ids_before = ids;
      ids = ids_next;
      ids_next = pages_of(window + 1);
    }
    int64_t page;
    int in;
    locate(i, page, in);
    k_from = a.c.k + page * a.c.code_page + (int64_t)in * dh;
    ks_from = a.c.k_scale + page * a.c.scale_page + in;
  };
  auto find_v = [&](int i) {
    int64_t page;
    int in;
    locate(i, page, in);
    v_from = a.c.v + page * a.c.code_page + (int64_t)in * dh;
    vs_from = a.c.v_scale + page * a.c.scale_page + in;
  };
  auto load_k = [&]() {
    kc = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from(k_from), k_off, 0, 0));
    ks = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from(ks_from), 4u * (uint32_t)k_place, 0, 0));
  };
  auto load_v = [&]() {
    const __amdgpu_buffer_rsrc_t r = from(v_from);
#pragma unroll
    for (int e = 0; e < 4; ++e) vc[e] = __builtin_amdgcn_raw_buffer_load_b32(r, v_off, (uint32_t)(e * dh), 0);
    vs = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from(vs_from), 16u * (uint32_t)v_four, 0, 0));
  };
  // In LDS, rows of 128 bytes with their chunks of 16 swapped as staged tiles have them: K in parts of 64 elements, V^T in
  // parts of 64 places.
  auto k_chunk = [&](int i, int place, int chunk) {
    return tiles + (i & 1) * kBytes + (chunk >> 3) * kTile * 128 + 128 * place + 16 * ((chunk & 7) ^ stage_swz(place));
  };
  auto v_chunk = [&](int i, int d, int chunk) {
    return tiles + (2 + (i & 1)) * kBytes + (chunk >> 3) * D * 128 + 128 * d + 16 * ((chunk & 7) ^ stage_swz(d));
  };
  // Where this lane reads chunk 2 c + hi of 8 of row s of a block of 32 rows (the swaps repeat every 32 rows)
  int at_chunk[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) at_chunk[c] = 128 * s + 16 * ((2 * c + hi) ^ stage_swz(s));
  auto widen_k = [&](int i) {
#pragma unroll
    for (int w = 0; w < 4; w += 2)
      *reinterpret_cast<u32x4*>(k_chunk(i, kShare * wv + k_place, k_at / 8 + w / 2)) =
          u32x4{widen2<E5M2, false>(kc[w], ks), widen2<E5M2, true>(kc[w], ks), widen2<E5M2, false>(kc[w + 1], ks),
                widen2<E5M2, true>(kc[w + 1], ks)};
  };
  auto widen_v = [&](int i) {
    uint32_t x[4][2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e][0] = widen2<E5M2, false>(vc[e], vs[e]);
      x[e][1] = widen2<E5M2, true>(vc[e], vs[e]);
    }
    if (edge_of(i)) {
      uint32_t word = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t lo = (x[e][y] & 0x7f80u) == 0x7f80u, up = (x[e][y] & 0x7f800000u) == 0x7f800000u;
          word |= (lo | up << 1) << (4 * e + 2 * y);
          x[e][y] &= (lo ? 0u : 0xffffu) | (up ? 0u : 0xffff0000u);
        }
      bad[i & 1][(kShare / 4 * wv + v_four) * (D / 4) + v_at / 4] = (uint16_t)word;
    }
    // places 16 g + 4 y .. + 3 go to half y / 2 of chunk 2 g + y % 2: a lane's eight places of P^T
    const int four = kShare / 4 * wv + v_four;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
      *reinterpret_cast<uint2*>(v_chunk(i, v_at + j, 2 * (four >> 2) + (four & 1)) + 8 * (four >> 1 & 1)) =
          make_uint2(__builtin_amdgcn_perm(x[1][j >> 1], x[0][j >> 1], sel),
                     __builtin_amdgcn_perm(x[3][j >> 1], x[2][j >> 1], sel));
    }
  };
  // Tile i to LDS, and the tile that was found last on its way
  auto fill_k = [&](int i) {
    widen_k(i);
    load_k();
  };
  auto fill_v = [&](int i) {
    widen_v(i);
    load_v();
  };

  f32x16 acc[DB], zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
  for (int j = 0; j < DB; ++j) acc[j] = zero;
  float top = kNone, total = 0.f;  // total: of the places that this lane holds
  const float c_log2 = a.c_log2;
  f32x16 st[NB];
  bf16x8 pf[2 * NB][2];
  uint32_t seen[NB];  // bit 4 i + e: row 8 i + 4 hi + e
  bool edge = false;  // of the tile whose P this wave holds

  auto tile = [](int k) { return PARTS == 1 ? k >> 1 : k; };
  auto half = [&](int k) { return PARTS == 1 ? k & 1 : part; };
  // Operands from LDS: of V for eight products with each part of P, of K for eight
  bf16x8 vf[8], kf[8];
  auto read_values = [&](int k) {
    const int u = half(k);
    const uint8_t* v = tiles + (2 + (tile(k) & 1)) * kBytes + (NB == 2 ? u * D * 128 : 0);
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
      const int at = at_chunk[g] ^ (NB == 1 ? 64 * u : 0);  // chunk 4 u + 2 g + hi
#pragma unroll
      for (int j = 0; j < DB; ++j) vf[g * DB + j] = *reinterpret_cast<const bf16x8*>(v + 32 * j * 128 + at);
    }
  };
  auto read_keys = [&](int k, int x) {  // four of them
    const uint8_t* kt = tiles + (tile(k) & 1) * kBytes + half(k) * 32 * NB * 128;
#pragma unroll
    for (int y = x; y < x + 4; ++y) {
      const int c = y / NB, n = y % NB;
      kf[y] = *reinterpret_cast<const bf16x8*>(kt + ((c >> 2) * kTile + 32 * n) * 128 + at_chunk[c & 3]);
    }
  };
  auto multiply_values = [&](int x) {
#pragma unroll
    for (int y = x; y < x + 4; ++y) acc[y % DB] = multiply32(vf[y], pf[y / DB][1], acc[y % DB]);
#pragma unroll
    for (int y = x; y < x + 4; ++y) acc[y % DB] = multiply32(vf[y], pf[y / DB][0], acc[y % DB]);
  };
  auto multiply_keys = [&](int x) {
#pragma unroll
    for (int y = x; y < x + 4; ++y) st[y % NB] = multiply32(kf[y], qf[y / NB], y < NB ? zero : st[y % NB]);
  };
  auto weights = [&](int k) {
    const int i = tile(k), first = half(k) * 32 * NB, place = (unit.step0 + i) * kTile;
    const uint32_t there = there_of(i);
    edge = edge_of(i);
    if (edge) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        seen[n] = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          // four places from drafted token j on: ones before the first, zeros past the last
          const int at = first + 32 * n + 8 * x + 4 * hi, j = place + at - (len - T);
          const int before = min(max(-j, 0), 4);
          const uint32_t of_tree = (uint32_t)(sees >> min(max(j, 0), 63)) << before | ((1u << before) - 1u);
          const uint32_t four = (there >> (at >> 4) & 1u) & (uint32_t)(j < 64) ? of_tree & 15u : 0u;
          seen[n] |= four << (4 * x);
        }
        f32x16 of_seen;
#pragma unroll
        for (int e = 0; e < 16; ++e) of_seen[e] = seen[n] >> e & 1u ? st[n][e] : kNone;
        st[n] = of_seen;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    float m = st[0][0];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, st[n][e]);
    {
      // the other half's maximum
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
      m = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
    }
    if (__ballot((m - top) * c_log2 > kSlack)) {
      m = fmaxf(m, top);
      const float w = weight_of(top, m, c_log2);
      total *= w;
#pragma unroll
      for (int j = 0; j < DB; ++j) acc[j] *= w;
      top = m;
    }
    const float base = top == kNone ? 0.f : top * c_log2;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float p[8], sum = 0.f;  // in eights, as in attend_kernel
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(st[n][8 * g + e], c_log2, -base));
          sum += p[e];
        }
        total += sum;
        split8<2>(p, pf[2 * n + g]);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  // Whoever sees a value that is not finite gets NaN (tiles that not all rows see; hardly ever any).
  auto poison = [&](int k) {
    const int i = tile(k), first = half(k) * 32 * NB;
    uint32_t any = 0;
    for (int n = lane; n < kTile * D / 32; n += 64) any |= reinterpret_cast<const uint32_t*>(bad[i & 1])[n];
    if (__ballot(any != 0) == 0) return;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const uint32_t other = (uint32_t)__shfl_xor((int)seen[n], 32);  // the other places of the row
#pragma unroll 1
      for (int y = 0; y < 8; ++y) {  // places 4 y .. + 3 of the 32
        const uint32_t four = ((y & 1) == hi ? seen[n] : other) >> (4 * (y >> 1)) & 15u;
        const uint32_t mask = (four & 1u ? 0x000fu : 0u) | (four & 2u ? 0x00f0u : 0u) | (four & 4u ? 0x0f00u : 0u) |
                              (four & 8u ? 0xf000u : 0u);
        const uint16_t* at = bad[i & 1] + (first / 4 + 8 * n + y) * (D / 4) + hi;
#pragma unroll
        for (int j = 0; j < DB; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t hit = at[8 * j + 2 * x] & mask;
            hit |= hit >> 8;
            hit |= hit >> 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[j][4 * x + e] = hit >> e & 1u ? __uint_as_float(0x7fc00000u) : acc[j][4 * x + e];
          }
      }
    }
  };
  auto meet = [&]() {
    wait_loads<63>();  // what this wave has written to LDS
    bare_barrier();
  };

  if (count > 0) {
    const int behind = wv >> 2;
    find_k(0);
    load_k();
    find_v(0);
    load_v();
    widen_k(0);
    find_k(1);
    load_k();
    if constexpr (PARTS == 1) {
      widen_v(0);
      find_v(1);
      load_v();
    }
    meet();
    if (behind) {
      if constexpr (PARTS == 2) {
        find_v(1);
        fill_v(0);
        find_k(2);
        fill_k(1);
      }
      meet();
    }
    if constexpr (PARTS == 2) find_v(1 + behind);
    find_k(2 + (PARTS == 2 ? behind : 0));
    read_keys(0, 0);
    read_keys(0, 4);
    multiply_keys(0);
    multiply_keys(4);
    meet();
    auto multiply_part = [&](int k, auto find) {
      __builtin_amdgcn_s_setprio(0);
      if constexpr (PARTS == 2) read_values(k);
      multiply_values(0);
      find();
      __builtin_amdgcn_sched_barrier(0);
      read_keys(k + 1, 0);
      multiply_values(4);
      __builtin_amdgcn_sched_barrier(0);
      read_keys(k + 1, 4);
      if (edge) poison(k);
      multiply_keys(0);
      multiply_keys(4);
      __builtin_amdgcn_s_setprio(1);  // of the vector part: few of its instructions are ready at a time
      meet();
    };
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      if constexpr (PARTS == 1) {
        fill_k(i + 1);
        weights(2 * i);
        read_values(2 * i);
        meet();
        multiply_part(2 * i, [&]() { find_v(i + 2); });
        fill_v(i + 1);
        weights(2 * i + 1);
        read_values(2 * i + 1);
        meet();
        multiply_part(2 * i + 1, [&]() { find_k(i + 3); });
      } else {
        fill_v(i + behind);
        fill_k(i + 1 + behind);
        weights(i);
        meet();
        multiply_part(i, [&]() {
          find_k(i + 3 + behind);
          find_v(i + 2 + behind);
        });
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (!behind) meet();
  }

  if constexpr (PARTS == 2) {
    float(*at)[64] = reinterpret_cast<float(*)[64]>(tiles) + rw * REGS;
    __syncthreads();  // all tiles read
    if (part == 1) {
      at[0][lane] = top;
      at[1][lane] = total;
#pragma unroll
      for (int j = 0; j < DB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) at[2 + 16 * j + e][lane] = acc[j][e];
    }
    __syncthreads();
    if (part == 1) return;
    const float other = at[0][lane], m = fmaxf(top, other);
    const float w0 = weight_of(top, m, c_log2), w1 = weight_of(other, m, c_log2);
    top = m;
    total = total * w0 + at[1][lane] * w1;
#pragma unroll
    for (int j = 0; j < DB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][e] = acc[j][e] * w0 + at[2 + 16 * j + e][lane] * w1;
  }
  const float sum = total + __shfl_xor(total, 32);
  if (row >= a.rows) return;
  const float inv = unit.n_chunks > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
  const int64_t at = (int64_t)blockIdx.x * (32 * (kTreeWaves / PARTS)) + 32 * rw + s;
  if (unit.n_chunks > 1 && hi == 0) a.part_stat[at] = make_float2(top, sum);
#pragma unroll
  for (int j = 0; j < DB; ++j)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int d = 32 * j + 8 * x + 4 * hi;
      if (d >= dh) continue;
      const f32x4 o = f32x4{acc[j][4 * x], acc[j][4 * x + 1], acc[j][4 * x + 2], acc[j][4 * x + 3]} * inv;
      if (unit.n_chunks > 1)
        *reinterpret_cast<f32x4*>(a.part_out + at * dh + d) = o;
      else
        store_row4<__bf16>(a, b, h, row, d, o);
    }
}

// Joins the chunks of rows.  Groups of lanes, 4 elements a lane, take every so many chunks, eight at a time, whose loads are
// all on their way at once; the groups' results meet in LDS.  A workgroup takes some rows of a key head, so that the
// workgroups of many rows that were not cut, which have nothing to do, are few (65536 rows: 43 us with one to
// a workgroup, 4.7 with 64).
constexpr int kAtOnce = 8;

template <bool F32>
__global__ void __launch_bounds__(256) join_kernel(AttendArgs a, int unit_rows, int rows_each) {
  __shared__ f32x4 sums[256];
  __shared__ float2 stats[16];
  const int t = threadIdx.x, lane = t & 63;
  const int per_head = (a.rows + rows_each - 1) / rows_each;
  const int part = blockIdx.x % per_head, h = blockIdx.x / per_head % a.c.heads, b = blockIdx.x / per_head / a.c.heads;
  uint32_t n_chunks, before = 0;  // before: units of the sequences before
  if (a.plan) {
    n_chunks = a.plan[b + 1] - a.plan[b];
    if (n_chunks <= 1) return;  // whole workgroup: written already
    before = a.plan[b] * (uint32_t)a.strands;
  } else {
    const Plan p = plan_of(a, lane);
    const uint32_t steps = b < 64 ? lane_of(p.steps0, b) : (uint32_t)uni((int)steps_of(a, b));
    n_chunks = chunks_of(steps, p.per);
    if (n_chunks <= 1) return;  // whole workgroup: written already
    for (int b0 = 0; b0 < b; b0 += 64) {
      const uint32_t n = b0 == 0 ? p.steps0 : steps_of(a, b0 + lane);
      before += lane_of(scan64(b0 + lane < b ? chunks_of(n, p.per) * (uint32_t)a.strands : 0u), 63);
    }
  }
  const int dh = a.c.head_dim, lanes = dh <= 64 ? 16 : dh <= 128 ? 32 : 64, groups = 256 / lanes;
  const int l = t % lanes, g = t / lanes, d = min(4 * l, dh - 4);
  const auto put = [&](int r, const f32x4& sum, float total) {
    if (4 * l < dh)
      store_row4<typename std::conditional<F32, float, __bf16>::type>(a, b, h, r, 4 * l,
                                                                      sum * (total == 0.f ? 0.f : 1.f / total));
  };
  // One row: the chunks from c0 on, `step` apart.
  float top, total;
  f32x4 sum;
  const auto add = [&](int r, uint32_t c0, uint32_t step) {
    const int rb = r / unit_rows, in = r % unit_rows;
    const int64_t first = ((int64_t)before + rb * a.c.heads + h) * unit_rows + in, apart = (int64_t)a.strands * unit_rows;
    top = kNone;
    total = 0.f;
    sum = f32x4{0.f, 0.f, 0.f, 0.f};
    for (; c0 < n_chunks; c0 += kAtOnce * step) {
      float2 st[kAtOnce];
      f32x4 x[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int64_t at = first + (int64_t)min(c0 + u * step, n_chunks - 1) * apart;
        st[u] = a.part_stat[at];
        x[u] = *reinterpret_cast<const f32x4*>(a.part_out + at * dh + d);
      }
      float m = top;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) m = fmaxf(m, st[u].x);
      const float w0 = weight_of(top, m, a.c_log2);
      total *= w0;
      sum *= w0;
      top = m;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (c0 + u * step >= n_chunks) continue;
        const float w = weight_of(st[u].x, m, a.c_log2);
        total += st[u].y * w;
        sum += x[u] * w;
      }
    }
  };
  if (n_chunks <= kAtOnce) {
    // few chunks: a row to each group, and the rows of as many workgroups to the first of them
    if (part % groups) return;
    for (int r = part * rows_each + g; r < min(a.rows, (part + groups) * rows_each); r += groups) {
      add(r, 0, 1);
      put(r, sum, total);
    }
    return;
  }
  const int end = min(a.rows, (part + 1) * rows_each);
  for (int r = part * rows_each; r < end; ++r) {
    add(r, g, groups);
    sums[t] = sum;
    if (l == 0) stats[g] = make_float2(top, total);
    __syncthreads();
    if (g == 0) {
      float m = top;
      for (int o = 1; o < groups; ++o) m = fmaxf(m, stats[o].x);
      float w = weight_of(top, m, a.c_log2);
      total *= w;
      sum *= w;
      for (int o = 1; o < groups; ++o) {
        w = weight_of(stats[o].x, m, a.c_log2);
        total += stats[o].y * w;
        sum += sums[o * lanes + l] * w;
      }
      put(r, sum, total);
    }
    if (r + 1 < end) __syncthreads();  // before the next row's
  }
}

// ------------------------------------------------------------------ host side

using namespace sn;

constexpr float kLog2E = 1.44269504088896340736f;

struct Way {
  bool tree;      // tree_kernel
  int nt;         // blocks of 16 rows in a wave of attend_kernel
  int unit_rows;  // rows of a workgroup
  int64_t units;  // at most
  bool cut;       // whether a sequence may have several chunks
  int64_t off_stat, off_plan, bytes;
};

template <int D, bool E5M2, bool F32>
void launch2(const AttendArgs& a, const Way& w, hipStream_t st) {
  const dim3 g((uint32_t)w.units);
  if constexpr (!F32 && D != 256) {
    if (w.tree)
      return a.row_waves == kTreeWaves ? tree_kernel<D, E5M2, 1><<<g, 64 * kTreeWaves, 0, st>>>(a)
                                       : tree_kernel<D, E5M2, 2><<<g, 64 * kTreeWaves, 0, st>>>(a);
  }
  if constexpr (D != 256)
    if (w.nt == 2) return attend_kernel<D, E5M2, F32, 2><<<g, 64 * kWaves, 0, st>>>(a);
  attend_kernel<D, E5M2, F32, 1><<<g, 64 * kWaves, 0, st>>>(a);
}

template <int D>
void launch1(const AttendArgs& a, const Way& w, bool e5m2, bool f32, hipStream_t st) {
  if (f32)
    e5m2 ? launch2<D, true, true>(a, w, st) : launch2<D, false, true>(a, w, st);
  else
    e5m2 ? launch2<D, true, false>(a, w, st) : launch2<D, false, false>(a, w, st);
}

// Checks the description and fills in the kernel's arguments.
int resolve(const sn_cache* cache, const sn_attend* p, AttendArgs& a, Way& w, bool need_memory) {
  if (!p) return refuse(SN_ENULL, "p must not be NULL");
  if (int rc = view_cache(cache, a.c, need_memory)) return rc;
  if (p->dtype != SN_F32 && p->dtype != SN_BF16) return refuse(SN_EDTYPE, "queries must be SN_F32 or SN_BF16");
  if (p->batch < 0 || p->batch > (1 << 20)) return refuse(SN_EINVAL, "batch must be in [0, 2^20]");
  if (p->drafts < 1 || p->drafts > 64) return refuse(SN_EINVAL, "drafts must be in [1, 64]");
  if (p->q_heads < 1 || p->q_heads > 65536 || p->q_heads % a.c.heads)
    return refuse(SN_EINVAL, "q_heads must be a multiple of the cache's heads, 65536 at most");
  if (p->table_cols < 0 || (int64_t)p->table_cols * a.c.page >= (int64_t(1) << 31) - 128)
    return refuse(SN_EINVAL, "table_cols must be >= 0, and table_cols * page below 2^31 - 128");
  if (!(p->scale > 0.f) || !std::isfinite(p->scale * kLog2E)) return refuse(SN_EINVAL, "scale must be positive and below 2e38");
  constexpr int64_t kMost = int64_t(1) << 40;
  for (int64_t s : {p->q_batch, p->q_draft, p->q_head, p->out_batch, p->out_draft, p->out_head})
    if (s < 0 || s > kMost) return refuse(SN_EINVAL, "strides must be >= 0 and below 2^40");
  // rows of out must not overlap: each dimension steps over what those of smaller strides span
  struct Dim {
    int64_t stride, size;
  } dims[3] = {{p->out_batch, p->batch}, {p->out_draft, p->drafts}, {p->out_head, p->q_heads}};
  std::sort(dims, dims + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  int64_t span = a.c.head_dim;
  for (const Dim& d : dims) {
    if (d.size <= 1) continue;
    if (d.stride < span) return refuse(SN_EINVAL, "rows of out must not overlap");
    span += (d.size - 1) * d.stride;
  }
  if (p->table_ld < 0 || p->table_ld > kMost || p->mask_batch < 0 || p->mask_batch > kMost)
    return refuse(SN_EINVAL, "table_ld and mask_batch must be >= 0 and below 2^40");
  a.q_batch = p->q_batch;
  a.q_draft = p->q_draft;
  a.q_head = p->q_head;
  a.out_batch = p->out_batch;
  a.out_draft = p->out_draft;
  a.out_head = p->out_head;
  a.table_ld = p->table_ld ? p->table_ld : p->table_cols;
  a.mask_batch = p->mask_batch;
  a.batch = p->batch;
  a.drafts = p->drafts;
  a.group = p->q_heads / a.c.heads;
  a.rows = a.drafts * a.group;
  a.max_places = p->table_cols * a.c.page;
  a.c_log2 = p->scale * kLog2E;

  const bool f32 = p->dtype == SN_F32;
  const int wide = a.c.head_dim <= 64 ? 64 : a.c.head_dim <= 128 ? 128 : 256;
  w.tree = !f32 && wide <= 128 && a.rows > 64;
  if (w.tree) {
    a.step = tile_of(wide);
    a.row_waves = a.rows > 128 ? kTreeWaves : kTreeWaves / 2;
    w.unit_rows = 32 * a.row_waves;
    a.row_blocks = (a.rows + w.unit_rows - 1) / w.unit_rows;
    // A chunk to each compute unit.  With pairs of waves and strands of many sequences, whose chunks differ, shorter ones even out
    // (16 trees of 9 tokens, 72 rows, over 2000-8192 places 93 us, 100.5 with 256; 3 of 12 over 2000-20000 53 and 47; of 64
    // tokens, without pairs, 480 and 412).
    a.target = a.row_waves == kTreeWaves || (int64_t)a.batch * a.c.heads * a.row_blocks <= 64 ? 256 : 512;
    a.least = 4;
  } else {
    // Sums of 256 elements fill the registers of a whole SIMD with 16 rows (8 sequences of 100-1500 places, 8 heads: 19.9 us;
    // with two workgroups on a compute unit, half the registers and loads that wait, 23.0; 4 tokens each of 16 over
    // 3500-4000: 54.7, with 32 rows a wave 61.8).
    w.nt = a.rows <= 16 || wide == 256 ? 1 : 2;
    const int waves = kWaves, blocks = (a.rows + 16 * w.nt - 1) / (16 * w.nt);
    a.step = kStep;
    a.row_waves = 1;
    while (a.row_waves < waves && a.row_waves < blocks) a.row_waves *= 2;
    w.unit_rows = 16 * w.nt * a.row_waves;
    a.row_blocks = (a.rows + w.unit_rows - 1) / w.unit_rows;
    // Strands of few sequences have equal chunks: as many workgroups as run at once (131071 places: 59 us, with twice as many
    // 63.7).  Chunks of many sequences' differ: twice as many even out (64 sequences of 200-8192 places: 73 us, 78.5).
    // Kernels of which one workgroup fits a compute unit: half as many for a single sequence (65536 places, 4 heads of 256:
    // 43.5 us with 512, 33.9 with 256; f32, 4 tokens over 65536 places, 8 heads of 128: 58 and 49), the same for more, whose
    // chunks differ (8 sequences of 500-4000 places, 8 tokens, 8 heads of 256: 64.4 us with 512, 75 with 256).
    const bool alone = wide == 256 || (f32 && wide == 128 && w.nt == 2);
    a.target = a.batch == 1 && alone ? 256 : (int64_t)a.batch * a.c.heads * a.row_blocks <= 256 ? 512 : 1024;
    a.least = 8;
  }
  const int waves = w.tree ? kTreeWaves : kWaves;
  const int64_t strands = (int64_t)a.c.heads * a.row_blocks;
  const int64_t steps = std::max<int64_t>(1, ((int64_t)a.max_places + a.step - 1) / a.step);
  if (a.batch * steps * strands >= (int64_t(1) << 31))
    return refuse(SN_EINVAL, "batch * table_cols * page * heads is too large");
  a.strands = (int32_t)strands;
  // a sequence has a chunk for every `per` of its steps and one more at most, and `per` is `least` at least
  const int64_t longest = std::max<int64_t>(1, (steps + a.least / 2) / a.least);
  w.units = std::min((int64_t)a.batch * longest * strands, a.target + (int64_t)a.batch * strands);
  if (w.units * 64 * waves >= (int64_t(1) << 32) ||
      (int64_t)a.batch * a.drafts * p->q_heads * 256 >= (int64_t(1) << 32))
    return refuse(SN_EINVAL, "batch * drafts * q_heads is too large");
  w.off_stat = w.off_plan = w.bytes = 0;
  w.cut = longest > 1;
  if (w.cut) {
    w.off_stat = (w.units * w.unit_rows * a.c.head_dim * 4 + 255) / 256 * 256;
    w.bytes = w.off_stat + (w.units * w.unit_rows * 8 + 255) / 256 * 256;
  }
  if (a.batch > kScanned) {
    w.off_plan = w.bytes;
    w.bytes += (((int64_t)a.batch + 1) * 4 + 255) / 256 * 256;
  }
  return SN_OK;
}

}  // namespace

extern "C" SN_API int spectral_cache_attend_workspace_bytes(const sn_cache* cache, const sn_attend* p, int64_t* bytes) {
  if (!bytes) return refuse(SN_ENULL, "bytes must not be NULL");
  AttendArgs a{};
  Way w{};
  if (int rc = resolve(cache, p, a, w, false)) return rc;
  *bytes = w.bytes;
  return SN_OK;
}

extern "C" SN_API int spectral_cache_attend(const sn_cache* cache, const sn_attend* p, const void* q,
                                            const int32_t* table, const int32_t* lengths, const int64_t* masks,
                                            void* out, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  AttendArgs a{};
  Way w{};
  if (int rc = resolve(cache, p, a, w, p && p->batch > 0)) return rc;
  if (a.batch == 0) return SN_OK;
  if (a.c.pages == 0) return refuse(SN_EINVAL, "the cache has no pages");
  if (!q || !lengths || !out || (p->table_cols > 0 && !table))
    return refuse(SN_ENULL, "q, table, lengths and out must not be NULL");
  const int type = p->dtype == SN_F32 ? 4 : 2;
  if (!aligned(q, type) || !aligned(out, type) || !aligned(table, 4) || !aligned(lengths, 4) || !aligned(masks, 8))
    return refuse(SN_EINVAL, "q, out, table, lengths and masks must be aligned to their type");
  if (w.bytes > 0) {
    if (!workspace) return refuse(SN_ENULL, "workspace must not be NULL");
    if (workspace_bytes < w.bytes)
      return refuse(SN_EINVAL, "workspace too small (spectral_cache_attend_workspace_bytes)");
    if (!aligned(workspace, 256)) return refuse(SN_EINVAL, "workspace must be 256-byte aligned");
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = check_stream(st)) return rc;
  a.q = q;
  a.out = out;
  a.table = table;
  a.lengths = lengths;
  a.masks = masks;
  a.part_out = static_cast<float*>(workspace);
  a.part_stat = reinterpret_cast<float2*>(static_cast<char*>(workspace) + w.off_stat);
  if (a.batch > kScanned) {
    a.plan = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + w.off_plan);
    plan_kernel<<<1, 64 * kPlanWaves, 0, st>>>(a);
    if (int rc = sn::launched("plan")) return rc;
  }
  const bool f32 = p->dtype == SN_F32, e5m2 = cache->format == SN_E5M2;
  if (a.c.head_dim <= 64)
    launch1<64>(a, w, e5m2, f32, st);
  else if (a.c.head_dim <= 128)
    launch1<128>(a, w, e5m2, f32, st);
  else
    launch1<256>(a, w, e5m2, f32, st);
  if (int rc = sn::launched("attention")) return rc;
  if (w.cut) {
    // about 512 workgroups
    const int64_t all = (int64_t)a.batch * a.c.heads * a.rows;
    const int rows_each = (int)std::min<int64_t>(a.rows, std::max<int64_t>(1, all / 512));
    const dim3 g((uint32_t)((int64_t)a.batch * a.c.heads * ((a.rows + rows_each - 1) / rows_each)));
    f32 ? join_kernel<true><<<g, 256, 0, st>>>(a, w.unit_rows, rows_each)
        : join_kernel<false><<<g, 256, 0, st>>>(a, w.unit_rows, rows_each);
    return sn::launched("join");
  }
  return SN_OK;
}
