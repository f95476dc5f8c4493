// Rotary positions of queries and keys (spectral_rotary; Sec. 3.3 of the paper): pairs (x0, x1) of a head turn by
// p f_i, the token's position times the pair's frequency, or back.
//
// A far position's angle is many turns: p f_i is formed in turns in double and its
// whole part taken off exactly (one fused multiply-add).  The sine and cosine of the rest,
// at most half a turn, are formed in double too, and rounded to float once, with the amplitude.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "device_util.h"
#include "entry_util.h"
#include "rotary.h"

namespace {

using namespace sn_dev;
using sn::kMaxPairs;
using sn::RotaryTable;

// Element types: V values at offset `at` of a tensor to and from float.
template <typename T>
struct Plain {
  const T* x;
  T* out;
  template <int V>
  __device__ __forceinline__ void load(int64_t at, float (&f)[V]) const {
    if constexpr (V * sizeof(T) >= 4) {
      typedef T vec __attribute__((ext_vector_type(V)));
      typedef vec vec_any __attribute__((aligned(sizeof(T))));  // wide accesses need no more
      const vec w = *reinterpret_cast<const vec_any*>(x + at);
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] = (float)w[e];
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] = (float)x[at + e];
    }
  }
  template <int V>
  __device__ __forceinline__ void store(int64_t at, const float (&f)[V]) const {
    if constexpr (V * sizeof(T) >= 4) {
      typedef T vec __attribute__((ext_vector_type(V)));
      typedef vec vec_any __attribute__((aligned(sizeof(T))));
      vec w;
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = (T)f[e];
      *reinterpret_cast<vec_any*>(out + at) = w;
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) out[at + e] = (T)f[e];
    }
  }
};

// Values as bf16 hi + lo planes (the logit consumer's projections), 2^-17 of the value each time they are split.
struct Planes {
  uint16_t* hi;
  uint16_t* lo;
  template <int V>
  __device__ __forceinline__ void load(int64_t at, float (&f)[V]) const {
    typedef __bf16 vec __attribute__((ext_vector_type(V)));
    const vec h = *reinterpret_cast<const vec*>(hi + at), l = *reinterpret_cast<const vec*>(lo + at);
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = (float)h[e] + (float)l[e];
  }
  template <int V>
  __device__ __forceinline__ void store(int64_t at, const float (&f)[V]) const {
    typedef __bf16 vec __attribute__((ext_vector_type(V)));
    vec h, l;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[e] = (__bf16)f[e];
      l[e] = (__bf16)(f[e] - (float)h[e]);
    }
    *reinterpret_cast<vec*>(hi + at) = h;
    *reinterpret_cast<vec*>(lo + at) = l;
  }
};

template <typename IO>
struct HeadsArg {
  IO io;
  int32_t heads;
  int32_t copy_rest;     // out is not x: the elements past rot_dim are copied
  int32_t copy_padding;  // ... and so are whole rows of padding (else they are left as out holds them)
  int64_t x_token, x_head, out_token, out_head;
};

template <typename IO>
struct RotaryArgs {
  RotaryTable table;
  HeadsArg<IO> t[2];
  const int64_t* positions;
  int64_t first, n_tokens;
  int64_t group0;      // groups of tokens that earlier launches of the call turn
  int64_t period;      // tokens after which positions repeat (the layers of the consumer), or n_tokens
  float sign;          // -1 turns back
  int32_t n_tensors, tokens_per_group, splits;
  int32_t zero_stays;  // in place without amplitude: rows at position zero are not read and split again
};

// One pair, the same operations in every variant, so that they give the same bits.
__device__ __forceinline__ void turn(float x0, float x1, float c, float s, float& y0, float& y1) {
  y0 = fmaf(x0, c, -(x1 * s));
  y1 = fmaf(x0, s, x1 * c);
}

// Sine and cosine of r turns, |r| <= 1/2, to 2^-34 of themselves: the quarter turns off, then the Taylor series of the rest, at
// most an eighth of a turn.
__device__ __forceinline__ void sine_cosine(double r, double& sn, double& cn) {
  const double quarters = rint(4.0 * r);
  const double x = fma(quarters, -0.25, r) * 6.283185307179586476925, x2 = x * x;
  double s = -1.0 / 39916800.0, c = 1.0 / 479001600.0;
  s = fma(s, x2, 1.0 / 362880.0);
  c = fma(c, x2, -1.0 / 3628800.0);
  s = fma(s, x2, -1.0 / 5040.0);
  c = fma(c, x2, 1.0 / 40320.0);
  s = fma(s, x2, 1.0 / 120.0);
  c = fma(c, x2, -1.0 / 720.0);
  s = fma(s, x2, -1.0 / 6.0);
  c = fma(c, x2, 1.0 / 24.0);
  s = fma(s * x2, x, x);
  c = fma(c, x2, -0.5);
  c = fma(c, x2, 1.0);
  const int q = (int)quarters;  // -2 .. 2
  const double a = q & 1 ? c : s, b = q & 1 ? s : c;
  sn = q & 2 ? -a : a;
  cn = (q + 1) & 2 ? -b : b;
}

constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;  // tokens of one workgroup

// A workgroup forms the cosines and sines of its tokens once, in LDS, and then
// turns all heads of them; V neighbouring pairs a thread.  With few tokens the
// heads of one are split over `splits` workgroups.  Bound by memory: 8191 tokens of 72 heads of 128 bf16 56 us
// (5.4 TB/s), 4096 of 64 interleaved 27 (5.0; 29 with pairs of 16-byte accesses 32 bytes apart); one token
// 3.2 us.
template <typename IO, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs<IO> a) {
  __shared__ __attribute__((aligned(16))) float cs[kMaxTokens * 2 * kMaxPairs];  // cosines, then sines, of a token
  __shared__ int skip[kMaxTokens];
  const int t = threadIdx.x;
  const int pairs = a.table.pairs, rest = a.table.head_dim - 2 * pairs;
  const int64_t token0 = (a.group0 + blockIdx.x / a.splits) * a.tokens_per_group;
  const int split = blockIdx.x % a.splits;
  const int n = (int)(a.n_tokens - token0 < a.tokens_per_group ? a.n_tokens - token0 : a.tokens_per_group);
  for (int i = t; i < n * pairs; i += kThreads) {
    const int k = i / pairs, j = i % pairs;
    const int64_t row = a.n_tokens == a.period ? token0 + k : (token0 + k) % a.period;
    const int64_t p = a.positions ? a.positions[row] : a.first + row;
    const double f = a.table.turns[j], pd = (double)p;
    const double r = fma(pd, f, -rint(pd * f));  // what whole turns leave
    double sn, cn;
    sine_cosine(r, sn, cn);
    cs[k * 2 * pairs + j] = (float)(cn * a.table.amplitude);
    cs[k * 2 * pairs + pairs + j] = (float)(sn * a.table.amplitude) * a.sign;
    if (j == 0) skip[k] = a.zero_stays ? p <= 0 : p < 0;
  }
  __syncthreads();
  const int chunks = pairs / V;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    if (w >= a.n_tensors) break;
    const HeadsArg<IO>& h = a.t[w];
    const int items = n * h.heads * chunks;
    bool padded = false;  // this thread met a row of padding
    for (int i = split * kThreads + t; i < items; i += a.splits * kThreads) {
      const int c = i % chunks, th = i / chunks, hd = th % h.heads, k = th / h.heads;
      if (skip[k]) {
        padded = true;
        continue;
      }
      const int64_t xi = (token0 + k) * h.x_token + hd * h.x_head, oi = (token0 + k) * h.out_token + hd * h.out_head;
      float cn[V], sn[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        cn[e] = cs[k * 2 * pairs + c * V + e];
        sn[e] = cs[k * 2 * pairs + pairs + c * V + e];
      }
      if constexpr (INTERLEAVED) {
        float x[2 * V], y[2 * V];
        h.io.load(xi + 2 * V * c, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          turn(x[2 * e], x[2 * e + 1], cn[e], sn[e], y[2 * e], y[2 * e + 1]);
        }
        h.io.store(oi + 2 * V * c, y);
      } else {
        float x0[V], x1[V], y0[V], y1[V];
        h.io.load(xi + V * c, x0);
        h.io.load(xi + pairs + V * c, x1);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          turn(x0[e], x1[e], cn[e], sn[e], y0[e], y1[e]);
        }
        h.io.store(oi + V * c, y0);
        h.io.store(oi + pairs + V * c, y1);
      }
    }
    // apart from the loop above, which a branch there would slow down (5 heads of 8191 tokens: 6.65 us, with it 6.9)
    if (padded && h.copy_padding) {
      for (int i = split * kThreads + t; i < items; i += a.splits * kThreads) {
        const int c = i % chunks, th = i / chunks, hd = th % h.heads, k = th / h.heads;
        if (!skip[k]) continue;
        const int64_t xi = (token0 + k) * h.x_token + hd * h.x_head, oi = (token0 + k) * h.out_token + hd * h.out_head;
        float x[V];
        for (int at = V * c; at < 2 * pairs; at += pairs) {
          h.io.load(xi + at, x);
          h.io.store(oi + at, x);
        }
      }
    }
    if (h.copy_rest && rest > 0) {
      const int per = (rest + V - 1) / V, todo = n * h.heads * per;
      for (int i = split * kThreads + t; i < todo; i += a.splits * kThreads) {
        const int c = i % per, th = i / per, hd = th % h.heads, k = th / h.heads;
        if (skip[k] && !h.copy_padding) continue;
        const int64_t xi = (token0 + k) * h.x_token + hd * h.x_head + 2 * pairs + V * c;
        const int64_t oi = (token0 + k) * h.out_token + hd * h.out_head + 2 * pairs + V * c;
        float x[V];
        h.io.load(xi, x);
        h.io.store(oi, x);
      }
    }
  }
}

template <typename IO, int V, bool INTERLEAVED>
void launch_pairs(RotaryArgs<IO> a, hipStream_t st) {
  const int64_t heads = (int64_t)a.t[0].heads + (a.n_tensors > 1 ? a.t[1].heads : 0);
  const int64_t per_token = std::max<int64_t>(1, heads * (a.table.pairs / V));  // items
  a.tokens_per_group = (int32_t)std::min<int64_t>(kMaxTokens, std::max<int64_t>(1, 4 * kThreads / per_token));
  const int64_t groups = (a.n_tokens + a.tokens_per_group - 1) / a.tokens_per_group;
  a.splits = groups >= 512 ? 1 : (int32_t)std::min<int64_t>((per_token + kThreads - 1) / kThreads, 64);
  constexpr int64_t kMost = int64_t(1) << 20;  // groups of a launch, whose lanes are counted in 32 bits
  for (; a.group0 < groups; a.group0 += kMost)
    rotary_kernel<IO, V, INTERLEAVED>
        <<<dim3((uint32_t)(std::min(kMost, groups - a.group0) * a.splits)), kThreads, 0, st>>>(a);
}

// Pairs a thread takes: as many as make 16-byte accesses (W elements, half as many
// neighbouring pairs), where rot_dim and the rest of the head are multiples of that, else
// half as many, else one.
template <typename IO, int W>
void launch_layout(const RotaryArgs<IO>& a, hipStream_t st) {
  const int rest = a.table.head_dim - 2 * a.table.pairs;
  auto fits = [&](int v) { return a.table.pairs % v == 0 && rest % v == 0; };
  if (a.table.interleaved) {
    if (fits(W / 2)) return launch_pairs<IO, W / 2, true>(a, st);
    if (fits(W / 4)) return launch_pairs<IO, W / 4, true>(a, st);
    return launch_pairs<IO, 1, true>(a, st);
  }
  if (fits(W)) return launch_pairs<IO, W, false>(a, st);
  if (fits(W / 2)) return launch_pairs<IO, W / 2, false>(a, st);
  launch_pairs<IO, 1, false>(a, st);
}

}  // namespace

namespace sn {

namespace {
// The table of this thread's last good plan: a program turns every layer by one plan, and forming 64
// powers takes as long as the launch.
struct Formed {
  sn_rotary plan;
  RotaryTable table;
  bool any;
};
thread_local Formed t_formed{};
int form_table(const sn_rotary* p, RotaryTable& t);
}  // namespace

int rotary_table(const sn_rotary* p, RotaryTable& t) {
  if (p && t_formed.any && std::memcmp(&t_formed.plan, p, sizeof *p) == 0) {
    t = t_formed.table;
    return SN_OK;
  }
  const int rc = form_table(p, t);
  if (rc == SN_OK) t_formed = Formed{*p, t, true};
  return rc;
}

namespace {
int form_table(const sn_rotary* p, RotaryTable& t) {
  if (!p) return refuse(SN_ENULL, "the rotary plan must not be NULL");
  if (p->head_dim < 2 || p->head_dim > 1024) return refuse(SN_EINVAL, "head_dim must be in [2, 1024]");
  if (p->rot_dim < 2 || p->rot_dim % 2 || p->rot_dim > p->head_dim || p->rot_dim > 2 * kMaxPairs)
    return refuse(SN_EINVAL, "rot_dim must be even, in [2, min(head_dim, 256)]");
  if (p->layout != SN_ROTARY_HALF && p->layout != SN_ROTARY_INTERLEAVED)
    return refuse(SN_EINVAL, "layout must be SN_ROTARY_HALF or SN_ROTARY_INTERLEAVED");
  if (p->scaling < SN_ROTARY_NONE || p->scaling > SN_ROTARY_TURNS) return refuse(SN_EINVAL, "unknown scaling");
  if (!(p->base > 1.0) || !std::isfinite(p->base)) return refuse(SN_EINVAL, "base must be finite and > 1");
  const double rot = p->rot_dim, tau = 6.283185307179586476925;
  double base = p->base;
  const bool by_parts = p->scaling == SN_ROTARY_INDEX || p->scaling == SN_ROTARY_TURNS;
  if (p->scaling != SN_ROTARY_NONE && (!(p->factor >= 1.0) || !std::isfinite(p->factor)))
    return refuse(SN_EINVAL, "factor must be finite and >= 1");
  if (by_parts && (!(p->low > 0.0) || !(p->high > p->low) || !std::isfinite(p->high) || p->trained < 1))
    return refuse(SN_EINVAL, "scaling by parts needs 0 < low < high and trained >= 1");
  if (p->scaling == SN_ROTARY_BASE) {
    if (p->rot_dim < 4) return refuse(SN_EINVAL, "an enlarged base needs rot_dim >= 4");
    base *= std::pow(p->factor, rot / (rot - 2.0));
    if (!std::isfinite(base)) return refuse(SN_EINVAL, "the enlarged base must be finite");
  }
  double first = 0.0, last = 0.0;
  if (p->scaling == SN_ROTARY_INDEX) {
    auto index = [&](double turns) { return rot * std::log((double)p->trained / (turns * tau)) / (2.0 * std::log(base)); };
    first = std::max(std::floor(index(p->high)), 0.0);
    last = std::min(std::ceil(index(p->low)), rot - 1.0);
  }
  t.pairs = p->rot_dim / 2;
  t.head_dim = p->head_dim;
  t.interleaved = p->layout == SN_ROTARY_INTERLEAVED;
  t.amplitude = p->scaling == SN_ROTARY_INDEX ? 1.0 + 0.1 * std::log(p->factor) : 1.0;
  for (int i = 0; i < kMaxPairs; ++i) {
    double f = i < t.pairs ? std::pow(base, -2.0 * i / rot) : 0.0;
    double mix = 0.0;  // share of the divided frequency
    if (p->scaling == SN_ROTARY_LINEAR) mix = 1.0;
    if (p->scaling == SN_ROTARY_INDEX) mix = std::min(std::max((i - first) / std::max(last - first, 1e-3), 0.0), 1.0);
    if (p->scaling == SN_ROTARY_TURNS)
      mix = 1.0 - std::min(std::max(((double)p->trained * f / tau - p->low) / (p->high - p->low), 0.0), 1.0);
    t.turns[i] = (mix == 1.0 ? f / p->factor : mix == 0.0 ? f : f * (1.0 - mix) + f / p->factor * mix) / tau;
  }
  return SN_OK;
}
}  // namespace

int launch_rotary_planes(const RotaryTable& t, int64_t layers, int64_t seq, const int64_t* positions, int64_t q_heads,
                         int64_t k_heads, uint16_t* qh, uint16_t* ql, uint16_t* kh, uint16_t* kl, hipStream_t st) {
  RotaryArgs<Planes> a{};
  a.table = t;
  a.positions = positions;
  a.n_tokens = layers * seq;
  a.period = seq;
  a.zero_stays = t.amplitude == 1.0;
  a.sign = 1.f;
  a.n_tensors = 2;
  const int64_t heads[2] = {q_heads, k_heads};
  uint16_t* const hi[2] = {qh, kh};
  uint16_t* const lo[2] = {ql, kl};
  for (int w = 0; w < 2; ++w) {
    HeadsArg<Planes>& h = a.t[w];
    h.io = Planes{hi[w], lo[w]};
    h.heads = (int32_t)heads[w];
    h.x_head = h.out_head = t.head_dim;
    h.x_token = h.out_token = heads[w] * t.head_dim;
  }
  launch_layout<Planes, 8>(a, st);
  return launched("rotary");
}

}  // namespace sn

using namespace sn;

extern "C" SN_API int spectral_rotary_frequencies(const sn_rotary* p, double* freq, double* amplitude) {
  if (!freq || !amplitude) return refuse(SN_ENULL, "freq and amplitude must not be NULL");
  RotaryTable t{};
  if (int rc = rotary_table(p, t)) return rc;
  for (int i = 0; i < t.pairs; ++i) freq[i] = t.turns[i] * 6.283185307179586476925;
  *amplitude = (float)t.amplitude;
  return SN_OK;
}

namespace {

template <typename T>
int run_rotary(const RotaryTable& table, int64_t n_tokens, const int64_t* positions, int64_t first, int inverse,
               const sn_heads* heads, int n_heads, hipStream_t st) {
  RotaryArgs<Plain<T>> a{};
  a.table = table;
  a.positions = positions;
  a.first = first;
  a.n_tokens = a.period = n_tokens;
  a.sign = inverse & ~SN_ROTARY_COPY_PADDING ? -1.f : 1.f;
  a.n_tensors = n_heads;
  for (int w = 0; w < n_heads; ++w) {
    const sn_heads& s = heads[w];
    HeadsArg<Plain<T>>& h = a.t[w];
    h.io = Plain<T>{static_cast<const T*>(s.x), static_cast<T*>(s.out)};
    h.heads = (int32_t)s.heads;
    h.copy_rest = s.x != s.out;
    h.copy_padding = h.copy_rest && (inverse & SN_ROTARY_COPY_PADDING);
    h.x_token = s.x_token;
    h.x_head = s.x_head;
    h.out_token = s.out_token;
    h.out_head = s.out_head;
  }
  launch_layout<Plain<T>, 16 / (int)sizeof(T)>(a, st);
  return launched("rotary");
}

}  // namespace

extern "C" SN_API int spectral_rotary(const sn_rotary* p, int32_t dtype, int64_t n_tokens, const int64_t* positions,
                                      int64_t first, int32_t inverse, const sn_heads* heads, int32_t n_heads,
                                      void* hip_stream) {
  if (dtype != SN_F32 && dtype != SN_BF16) return refuse(SN_EDTYPE, "dtype must be SN_F32 or SN_BF16");
  RotaryTable table{};
  if (int rc = rotary_table(p, table)) return rc;
  if (!heads) return refuse(SN_ENULL, "heads must not be NULL");
  if (n_heads < 1 || n_heads > 2) return refuse(SN_EINVAL, "n_heads must be 1 or 2");
  if (n_tokens < 0 || n_tokens >= (int64_t(1) << 30)) return refuse(SN_EINVAL, "n_tokens must be in [0, 2^30)");
  if (!positions && (first < -(int64_t(1) << 40) || first > (int64_t(1) << 40)))
    return refuse(SN_EINVAL, "first must be within 2^40");
  const uintptr_t es = dtype == SN_F32 ? 4 : 2;
  if (!aligned(positions, 8)) return refuse(SN_EINVAL, "positions must be 8-byte aligned");
  for (int w = 0; w < n_heads; ++w) {
    const sn_heads& h = heads[w];
    constexpr int64_t kMost = int64_t(1) << 40;
    if (h.heads < 0 || h.heads > 65536) return refuse(SN_EINVAL, "heads must be in [0, 65536]");
    if (h.x_token < 0 || h.x_head < 0 || h.out_token < 0 || h.out_head < 0 || h.x_token > kMost || h.x_head > kMost ||
        h.out_token > kMost || h.out_head > kMost)
      return refuse(SN_EINVAL, "strides must be in [0, 2^40]");
    if (n_tokens > 0 && h.heads > 0 && (!h.x || !h.out)) return refuse(SN_ENULL, "x and out must not be NULL");
    if (!aligned(h.x, es) || !aligned(h.out, es)) return refuse(SN_EINVAL, "x and out must be aligned to their type");
    if (n_tokens == 0 || h.heads == 0) continue;
    const bool heads_apart = h.heads <= 1 || h.out_head >= p->head_dim;
    const bool tokens_apart = n_tokens <= 1 || h.out_token >= p->head_dim;
    const bool nested = n_tokens <= 1 || h.heads <= 1 || h.out_token / h.heads >= h.out_head ||
                        h.out_head / n_tokens >= h.out_token;
    if (!heads_apart || !tokens_apart || !nested) return refuse(SN_EINVAL, "the heads of out must not overlap");
    if (h.x == h.out && h.x && (h.x_token != h.out_token || h.x_head != h.out_head))
      return refuse(SN_EINVAL, "out may be x only with the same strides");
  }
  if (n_tokens == 0 || (heads[0].heads == 0 && (n_heads == 1 || heads[1].heads == 0))) return SN_OK;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = check_stream(st)) return rc;
  return dtype == SN_F32 ? run_rotary<float>(table, n_tokens, positions, first, inverse, heads, n_heads, st)
                         : run_rotary<__bf16>(table, n_tokens, positions, first, inverse, heads, n_heads, st);
}
