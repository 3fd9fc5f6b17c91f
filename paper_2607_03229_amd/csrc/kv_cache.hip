// Keys and values into and out of the pages of a cache (mpipe_op_cache_write / _read).
//
// A token's head is a unit of work: LPU lanes (the power of two that holds head_dim / 8) move
// eight values each, so that the largest magnitude of a head is a few lane exchanges away when it
// is quantised.  A power of two as its scale makes every step exact but the one rounding to
// e4m3, and what is read back is exact in bf16.  Bound by HBM for prompts, by one chain of loads
// (position, page, row) for single tokens.
#include "attn_kernels.h"
#include "common.h"
#include "cache_places.h"

namespace mpipe {
namespace {

typedef __attribute__((ext_vector_type(8), aligned(2))) bf16 bf16x8_any;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;

struct RowArgs {
  void *ck, *cv;
  uint8_t *sk, *sv;
  AttnView k, v;
  CachePlaces at;
  int64_t rows;
  int32_t* status;
};

__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const bf16x8_any v = *reinterpret_cast<const bf16x8_any*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4_any a = *reinterpret_cast<const f32x4_any*>(p);
  const f32x4_any b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  bf16x8_any v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (bf16)x[e];
  *reinterpret_cast<bf16x8_any*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<f32x4_any*>(p) = f32x4_any{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4_any*>(p + 4) = f32x4_any{x[4], x[5], x[6], x[7]};
}

// Least whole e of [-120, 120] with top <= 448 * 2^e; top >= 0 and finite.
__device__ __forceinline__ int scale_exponent(float top) {
  int e;
  const float m = frexpf(top, &e);   // top = m * 2^e, m in [1/2, 1); 448 = 0.875 * 2^9
  e = e - 9 + (m > 0.875f ? 1 : 0);
  return top == 0.f ? -120 : min(max(e, -120), 120);
}

// Eight values of a unit; `lane` counts within it.  Every lane of a unit calls this.
template <int LPU>
__device__ __forceinline__ void store_e4m3(uint8_t* p, uint8_t* scale, float (&x)[8], int lane,
                                           bool real) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]);
    if (!(a < INFINITY)) x[i] = NAN;   // an infinity has no e4m3 value either
    else top = fmaxf(top, a);
  }
#pragma unroll
  for (int o = LPU / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const int e = scale_exponent(top);
  if (!real) return;
  const float f = __uint_as_float((uint32_t)(127 - e) << 23);
  uint2 out;
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, w, false);
  out.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, w, true);
  w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * f, x[5] * f, w, false);
  out.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[6] * f, x[7] * f, w, true);
  *reinterpret_cast<uint2*>(p + 8 * lane) = out;
  if (lane == 0) *scale = (uint8_t)(e + 127);
}

// A unit: (row, key or value, head), heads fastest, so that neighbours read one row of a product.
template <class T, class C, int LPU, bool WRITE>
__global__ __launch_bounds__(256) void rows_kernel(RowArgs a) {
  const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPU;
  const int lane = threadIdx.x % LPU, heads = a.at.heads, d = a.at.d;
  int64_t row = unit / (2 * heads);
  const bool in = row < a.rows;
  row = in ? row : a.rows - 1;
  const int rest = (int)(unit % (2 * heads)), side = rest / heads, head = rest % heads;
  const int64_t place = in ? a.at.of(row, head) : kCacheNone;
  const bool real = place >= 0 && 8 * lane < d;
  if (in && place == kCacheBad && rest == 0 && lane == 0 && a.status) *a.status = 1;
  const AttnView& v = side ? a.v : a.k;
  T* x = reinterpret_cast<T*>(const_cast<void*>(v.p)) + v.row * row + v.head * head + 8 * lane;
  C* c = reinterpret_cast<C*>(side ? a.cv : a.ck) + (place >= 0 ? place : 0) * d;
  uint8_t* s = (side ? a.sv : a.sk) + (place >= 0 ? place : 0);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = 0.f;
  if constexpr (WRITE) {
    if (real) load8(x, y);
    if constexpr (sizeof(C) == 1) store_e4m3<LPU>(reinterpret_cast<uint8_t*>(c), s, y, lane, real);
    else if (real) store8(c + 8 * lane, y);
  } else {
    if (place == kCacheNone || 8 * lane >= d) return;
    if (place == kCacheBad) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = NAN;
    } else if constexpr (sizeof(C) == 1) {
      load8_e4m3(reinterpret_cast<const uint8_t*>(c) + 8 * lane, e8m0(*s), y);
    } else {
      load8(c + 8 * lane, y);
    }
    store8(x, y);
  }
}

template <class T, class C, bool WRITE>
hipError_t launch(const RowArgs& a, hipStream_t s) {
  int lpu = 1;
  while (8 * lpu < a.at.d) lpu *= 2;
  // units of a launch: 2^23 blocks at most
  RowArgs b = a;
  const int64_t step = ((int64_t(1) << 31) / lpu) / (2 * a.at.heads);
  for (int64_t r = 0; r < a.rows; r += step) {
    b.rows = a.rows - r < step ? a.rows - r : step;
    b.at.first = r;
    const int esz = sizeof(T);
    b.k.p = (const char*)a.k.p + r * a.k.row * esz;
    b.v.p = (const char*)a.v.p + r * a.v.row * esz;
    const int64_t blocks = (b.rows * 2 * a.at.heads * lpu + 255) / 256;
    const dim3 grid((unsigned)blocks), block(256);
    switch (lpu) {
      case 1: hipLaunchKernelGGL((rows_kernel<T, C, 1, WRITE>), grid, block, 0, s, b); break;
      case 2: hipLaunchKernelGGL((rows_kernel<T, C, 2, WRITE>), grid, block, 0, s, b); break;
      case 4: hipLaunchKernelGGL((rows_kernel<T, C, 4, WRITE>), grid, block, 0, s, b); break;
      case 8: hipLaunchKernelGGL((rows_kernel<T, C, 8, WRITE>), grid, block, 0, s, b); break;
      case 16: hipLaunchKernelGGL((rows_kernel<T, C, 16, WRITE>), grid, block, 0, s, b); break;
      default: hipLaunchKernelGGL((rows_kernel<T, C, 32, WRITE>), grid, block, 0, s, b); break;
    }
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

template <bool WRITE>
hipError_t rows(const CacheRows& p, hipStream_t s) {
  RowArgs a;
  a.ck = p.cache.k;
  a.cv = p.cache.v;
  a.sk = p.cache.k_scale;
  a.sv = p.cache.v_scale;
  a.k = {p.k.p, p.k.row, p.k.head};
  a.v = {p.v.p, p.v.row, p.v.head};
  a.at = cache_places(p.cache, p.table, p.ld_table, p.n_seq, p.width, p.seq, p.pos);
  a.rows = p.rows;
  a.status = p.status;
  if (p.dtype == DT_BF16) {
    switch (p.cache.dtype) {
      case MPIPE_F32: return launch<bf16, float, WRITE>(a, s);
      case MPIPE_BF16: return launch<bf16, bf16, WRITE>(a, s);
      default: return launch<bf16, uint8_t, WRITE>(a, s);
    }
  }
  switch (p.cache.dtype) {
    case MPIPE_F32: return launch<float, float, WRITE>(a, s);
    case MPIPE_BF16: return launch<float, bf16, WRITE>(a, s);
    default: return launch<float, uint8_t, WRITE>(a, s);
  }
}

}  // namespace

hipError_t cache_write(const CacheRows& p, hipStream_t s) { return rows<true>(p, s); }
hipError_t cache_read(const CacheRows& p, hipStream_t s) { return rows<false>(p, s); }

}  // namespace mpipe
