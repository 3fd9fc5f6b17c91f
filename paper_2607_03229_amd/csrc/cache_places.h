// Where a token's heads lie in a paged cache, and its 8-bit values.
#pragma once
#include <hip/hip_runtime.h>

#include "attn_kernels.h"
#include "common.h"

namespace mpipe {

constexpr int64_t kCacheNone = -1;   // a row that is left out
constexpr int64_t kCacheBad = -2;    // a place outside the tables or the pool

// n / d for n below 2^32 (d at most 2^17) by a product: n (2^49 / d rounded up) / 2^49, off by less
// than n / 2^49 < 1 / d.  (A launch's lanes end at 2^31, and a last block's beyond are some hundreds.)
struct Divide {
  uint64_t mul;
  __device__ __forceinline__ int64_t quotient(int64_t n) const {
    return (int64_t)__umul64hi((uint64_t)n << 15, mul);
  }
};
inline Divide divide_by(uint32_t d) { return {((uint64_t(1) << 49) + d - 1) / d}; }

struct CachePlaces {
  const int32_t *table, *seq, *pos;
  int64_t ld_table, first;   // first: added to the row, for its seq and pos
  int32_t n_seq, width, n_pages, heads, d, shift;   // a page has 2^shift tokens

  // The row of d values of (token, head): the index into scales, and d times it into pages.
  __device__ __forceinline__ int64_t in_page(int32_t page, int32_t token, int head) const {
    return (((int64_t)page * heads + head) << shift) + (token & ((1 << shift) - 1));
  }
  // Of U rows at once.
  template <int U>
  __device__ __forceinline__ void of(const int64_t (&row)[U], const int (&head)[U], int64_t (&place)[U]) const {
    int32_t t[U], page[U];
    int64_t s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      t[u] = pos[row[u] + first];
      s[u] = seq ? (int64_t)seq[row[u] + first] : row[u] + first;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      place[u] = t[u] < 0 || s[u] < 0 ? kCacheNone : s[u] >= n_seq || (t[u] >> shift) >= width ? kCacheBad : 0;
      page[u] = place[u] == 0 ? table[s[u] * ld_table + (t[u] >> shift)] : 0;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (place[u] == 0) place[u] = page[u] < 0 || page[u] >= n_pages ? kCacheBad : in_page(page[u], t[u], head[u]);
    }
  }
};

inline CachePlaces cache_places(const mpipe_kv_cache& c, const int32_t* table, int64_t ld_table,
                                int32_t n_seq, int32_t width, const int32_t* seq,
                                const int32_t* pos) {
  CachePlaces p;
  p.table = table;
  p.seq = seq;
  p.pos = pos;
  p.ld_table = ld_table;
  p.first = 0;
  p.n_seq = n_seq;
  p.width = width;
  p.n_pages = (int32_t)c.n_pages;
  p.heads = c.heads;
  p.d = c.head_dim;
  p.shift = __builtin_ctz((unsigned)c.page);
  return p;
}

// 2^(b - 127)
__device__ __forceinline__ float e8m0(uint8_t b) {
  return b ? __uint_as_float((uint32_t)b << 23) : 0x1p-127f;
}
// Eight e4m3 values (8-byte aligned) times a power of two.
__device__ __forceinline__ void load8_e4m3(const uint8_t* p, float scale, float (&x)[8]) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, true);
  x[0] = a[0] * scale; x[1] = a[1] * scale; x[2] = b[0] * scale; x[3] = b[1] * scale;
  x[4] = c[0] * scale; x[5] = c[1] * scale; x[6] = d[0] * scale; x[7] = d[1] * scale;
}
// Values times a power of two, in fp32 and (exact there too) in bf16.
__device__ __forceinline__ f32x4 f32_of_e4m3(uint32_t w, float scale) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return f32x4{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
}
__device__ __forceinline__ bf16x8 bf16_of_e4m3(uint2 w, float scale) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace mpipe
