// A paged cache of keys and values in 8 bits, written and read back (spectral_cache_write, spectral_cache_read).
// A row, the head_dim elements of one token and head, has one power-of-two scale, formed as the block
// quantiser does; its codes lie together.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cache_fp8.h"
#include "fp8_device.h"

namespace {

using namespace sn_dev;
using sn::CacheView;

struct RowsArgs {
  CacheView c;
  const int64_t* slots;
  void* x[2];  // keys and values
  int64_t token[2], head[2];
  uint32_t rows;  // tokens * heads
};

// Row `row` of tokens * heads: its token, head, and place in the cache; false where the slot is outside.
__device__ __forceinline__ bool locate(const RowsArgs& a, uint32_t row, uint32_t& token, uint32_t& head, int64_t& codes,
                                       int64_t& scale) {
  token = row / (uint32_t)a.c.heads;
  head = row - token * (uint32_t)a.c.heads;
  const int64_t slot = a.slots[token];
  if (slot < 0 || slot >= a.c.pages << a.c.page_shift) return false;
  const int64_t page = slot >> a.c.page_shift, in = ((int64_t)head << a.c.page_shift) + (slot & (a.c.page - 1));
  codes = page * a.c.code_page + in * a.c.head_dim;
  scale = page * a.c.scale_page + in;
  return true;
}

// LANES lanes of 16 elements take a row of keys and that of values together, so that enough is on its way: 8191
// tokens of 8 heads of 128 in bf16 take 9.9 us (11.5 with 8 elements of one of the two a lane) again and again, when the
// 256 MB cache holds them, and 13.9 (3.7 TB/s) when it does not; in float32 10.8 again and again.
template <typename T, bool E5M2, int LANES>
__global__ void __launch_bounds__(256) write_kernel(RowsArgs a) {
  const int t = threadIdx.x, c = 16 * (t % LANES);
  for (uint32_t row = blockIdx.x * (256u / LANES) + t / LANES; row < a.rows; row += gridDim.x * (256u / LANES)) {
    uint32_t token, head;
    int64_t codes, scale;
    if (!locate(a, row, token, head, codes, scale)) continue;  // all lanes of the row
    Eight<T> x[2][2];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[which][i].clear();
        if (c < a.c.head_dim)
          x[which][i].load(static_cast<const T*>(a.x[which]) + token * a.token[which] + head * a.head[which] + c + 8 * i, 0, 8);
      }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max(top, x[which][e >> 3].magnitude(e & 7));
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      float s, inv;
      block_scale(top, format_top(E5M2), s, inv);
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Eight<T>& v = x[which][i >> 1];
        const int e = 4 * (i & 1);
        w[i] = encode4<E5M2>(v.value(e) * inv, v.value(e + 1) * inv, v.value(e + 2) * inv, v.value(e + 3) * inv);
      }
      if (c < a.c.head_dim) *reinterpret_cast<u32x4*>((which ? a.c.v : a.c.k) + codes + c) = w;
      if (c == 0) (which ? a.c.v_scale : a.c.k_scale)[scale] = s;
    }
  }
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

template <bool E5M2>
__device__ __forceinline__ void decode4(uint32_t w, float (&f)[4]) {
  f32x2 lo, hi;
  if constexpr (E5M2) {
    lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  }
  f[0] = lo[0], f[1] = lo[1], f[2] = hi[0], f[3] = hi[1];
}

// A lane takes the elements of one 16-byte store of keys and of values, and two rows at a time.  The results are more
// than the caches hold where it counts, so their stores pass them by: 32768 tokens of 8 heads of 128 to bf16 33.6 us, 41.5 with
// ordinary stores, 47.5 with 8 elements of one of the two a lane, all again and again; 41.6 (4.9 TB/s) of inputs that no
// cache holds.
template <typename T, bool E5M2, int LANES>
__global__ void __launch_bounds__(256) read_kernel(RowsArgs a) {
  constexpr int PER = 16 / sizeof(T), WORDS = PER / 4, ROWS = 2;
  typedef T out_vec __attribute__((ext_vector_type(PER)));
  typedef out_vec out_any __attribute__((aligned(sizeof(T))));
  const int t = threadIdx.x, c = PER * (t % LANES);
  if (c >= a.c.head_dim) return;
  constexpr uint32_t kApart = 256 / LANES;
  for (uint32_t row0 = blockIdx.x * (ROWS * kApart) + t / LANES; row0 < a.rows; row0 += gridDim.x * (ROWS * kApart)) {
    uint32_t token[ROWS], head[ROWS], w[ROWS][2][WORDS];
    float s[ROWS][2];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      int64_t codes, scale;
      const bool there = locate(a, min(row0 + r * kApart, a.rows - 1), token[r], head[r], codes, scale);
#pragma unroll
      for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[r][which][i] = 0;
        s[r][which] = 0.f;
        if (!there) continue;
        const uint32_t* p = reinterpret_cast<const uint32_t*>((which ? a.c.v : a.c.k) + codes + c);
        if constexpr (WORDS == 2) {
          const uint2 x = *reinterpret_cast<const uint2*>(p);
          w[r][which][0] = x.x, w[r][which][1] = x.y;
        } else {
          w[r][which][0] = *p;
        }
        s[r][which] = (which ? a.c.v_scale : a.c.k_scale)[scale];
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (row0 + r * kApart >= a.rows) continue;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        out_vec o;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
          float f[4];
          decode4<E5M2>(w[r][which][i], f);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[4 * i + e] = (T)(f[e] * s[r][which]);
        }
        __builtin_nontemporal_store(o, reinterpret_cast<out_any*>(static_cast<T*>(a.x[which]) + token[r] * a.token[which] +
                                                                  head[r] * a.head[which] + c));
      }
    }
  }
}

template <typename T, bool E5M2, bool WRITE>
void launch2(const RowsArgs& a, hipStream_t st) {
  const int size = a.c.head_dim <= 64 ? 64 : a.c.head_dim <= 128 ? 128 : 256;
  constexpr int PER = WRITE ? 16 : 16 / (int)sizeof(T);
  const uint32_t per = 256 / (size / PER) * (WRITE ? 1 : 2);  // rows of a workgroup
  const dim3 grid(std::min<uint32_t>((a.rows - 1) / per + 1, 1u << 20));
#define SN_GO(D)                                                     \
  do {                                                               \
    if constexpr (WRITE)                                             \
      write_kernel<T, E5M2, D / PER><<<grid, 256, 0, st>>>(a);       \
    else                                                             \
      read_kernel<T, E5M2, D / PER><<<grid, 256, 0, st>>>(a);        \
  } while (0)
  if (size == 64)
    SN_GO(64);
  else if (size == 128)
    SN_GO(128);
  else
    SN_GO(256);
#undef SN_GO
}

template <bool WRITE>
void launch1(const RowsArgs& a, bool bf16, bool e5m2, hipStream_t st) {
  if (bf16)
    e5m2 ? launch2<__bf16, true, WRITE>(a, st) : launch2<__bf16, false, WRITE>(a, st);
  else
    e5m2 ? launch2<float, true, WRITE>(a, st) : launch2<float, false, WRITE>(a, st);
}

using namespace sn;

// Either call: rows of x to the cache, or of the cache to x.
int rows_call(bool write, const sn_cache* cache, int32_t dtype, int64_t tokens, const int64_t* slots, void* const x[2],
              const int64_t token[2], const int64_t head[2], void* hip_stream) {
  RowsArgs a{};
  if (int rc = view_cache(cache, a.c, tokens > 0)) return rc;
  if (dtype != SN_F32 && dtype != SN_BF16) return refuse(SN_EDTYPE, "keys and values must be SN_F32 or SN_BF16");
  if (tokens < 0 || tokens >= (int64_t(1) << 31) || tokens * a.c.heads >= (int64_t(1) << 31))
    return refuse(SN_EINVAL, "tokens must be >= 0, and tokens * heads below 2^31");
  for (int i = 0; i < 2; ++i) {
    constexpr int64_t kMost = int64_t(1) << 40;
    if (token[i] < 0 || head[i] < 0 || token[i] > kMost || head[i] > kMost)
      return refuse(SN_EINVAL, "token and head strides must be >= 0 and below 2^40");
    if (!aligned(x[i], dtype == SN_F32 ? 4 : 2)) return refuse(SN_EINVAL, "keys and values must be aligned to their type");
    // rows of a result must not overlap: heads within tokens or tokens within heads
    const int64_t dh = a.c.head_dim, n = tokens, h = a.c.heads;
    if (!write && !((h == 1 || head[i] >= dh) && (n <= 1 || token[i] >= (h == 1 ? dh : (h - 1) * head[i] + dh))) &&
        !((n <= 1 || token[i] >= dh) && (h == 1 || head[i] >= (n <= 1 ? dh : (n - 1) * token[i] + dh))))
      return refuse(SN_EINVAL, "rows of the results must not overlap");
  }
  if (!aligned(slots, 8)) return refuse(SN_EINVAL, "slots must be 8-byte aligned");
  if (tokens == 0) return SN_OK;
  if (!slots || !x[0] || !x[1]) return refuse(SN_ENULL, "keys, values and slots must not be NULL");
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (int rc = check_stream(st)) return rc;
  a.slots = slots;
  for (int i = 0; i < 2; ++i) {
    a.x[i] = x[i];
    a.token[i] = token[i];
    a.head[i] = head[i];
  }
  a.rows = (uint32_t)(tokens * a.c.heads);
  const bool bf16 = dtype == SN_BF16, e5m2 = cache->format == SN_E5M2;
  write ? launch1<true>(a, bf16, e5m2, st) : launch1<false>(a, bf16, e5m2, st);
  return sn::launched(write ? "cache write" : "cache read");
}

}  // namespace

namespace sn {

int view_cache(const sn_cache* c, CacheView& view, bool need_memory) {
  if (!c) return refuse(SN_ENULL, "cache must not be NULL");
  if (c->format != SN_E4M3 && c->format != SN_E5M2) return refuse(SN_EDTYPE, "format must be SN_E4M3 or SN_E5M2");
  if (c->pages < 0 || c->pages >= (int64_t(1) << 31)) return refuse(SN_EINVAL, "pages must be in [0, 2^31)");
  if (c->heads < 1 || c->heads > 65536) return refuse(SN_EINVAL, "heads must be in [1, 65536]");
  if (c->page < 16 || c->page > 65536 || (c->page & (c->page - 1)))
    return refuse(SN_EINVAL, "page must be a power of two in [16, 65536]");
  if ((int64_t)c->heads * c->page >= (int64_t(1) << 31)) return refuse(SN_EINVAL, "heads * page must stay below 2^31");
  if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16)
    return refuse(SN_EINVAL, "head_dim must be a multiple of 16 in [16, 256]");
  const int64_t scales = (int64_t)c->heads * c->page, codes = scales * c->head_dim;
  const int64_t code_page = c->code_page ? c->code_page : codes, scale_page = c->scale_page ? c->scale_page : scales;
  constexpr int64_t kMost = int64_t(1) << 40;
  if (code_page < codes || code_page % 16 || code_page > kMost || scale_page < scales || scale_page % 4 || scale_page > kMost)
    return refuse(SN_EINVAL, "pages must not overlap; code_page a multiple of 16, scale_page of 4");
  if (need_memory && c->pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale))
    return refuse(SN_ENULL, "codes and scales of the cache must not be NULL");
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))
    return refuse(SN_EINVAL, "codes and scales of the cache must be 16-byte aligned");
  int shift = 0;
  while ((1 << shift) < c->page) ++shift;
  view = CacheView{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, c->pages,
                   code_page, scale_page, c->heads, c->page, shift, c->head_dim};
  return SN_OK;
}

}  // namespace sn

extern "C" SN_API int spectral_cache_write(const sn_cache* cache, int32_t dtype, int64_t tokens, const void* k,
                                           int64_t k_token, int64_t k_head, const void* v, int64_t v_token,
                                           int64_t v_head, const int64_t* slots, void* hip_stream) {
  void* const x[2] = {const_cast<void*>(k), const_cast<void*>(v)};
  const int64_t token[2] = {k_token, v_token}, head[2] = {k_head, v_head};
  return rows_call(true, cache, dtype, tokens, slots, x, token, head, hip_stream);
}

extern "C" SN_API int spectral_cache_read(const sn_cache* cache, int32_t dtype, int64_t tokens, const int64_t* slots,
                                          void* k, int64_t k_token, int64_t k_head, void* v, int64_t v_token,
                                          int64_t v_head, void* hip_stream) {
  void* const x[2] = {k, v};
  const int64_t token[2] = {k_token, v_token}, head[2] = {k_head, v_head};
  return rows_call(false, cache, dtype, tokens, slots, x, token, head, hip_stream);
}
