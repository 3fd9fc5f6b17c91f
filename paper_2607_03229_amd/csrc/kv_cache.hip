// Keys and values into and out of the pages of a cache (mpipe_op_cache_write / _read).
//
// A token's head, its key and its value, is a unit of work: LPU lanes (the power of two that holds
// head_dim / 8) move eight values of each, so that the largest magnitude of a head is a few lane
// exchanges away when it is quantised.  A power of two as its scale makes every step exact but the one rounding to
// e4m3, and what is read back is exact in bf16.  Bound by HBM for prompts, by one chain of loads
// (position, page, row) for single tokens: 64 tokens of 8 heads of 128 into 8 bits take 4 us, 3,001
// rows of 6 fp32 heads of 40 7.5 us each way, and four prompts of up to 32768, 4 heads of 128, are
// read in 89 us (5.3 TB/s).
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
  Divide by_heads;
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

// Eight values of a head, and its scale; `lane` counts within it.  Every lane of a unit calls this.
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
  *reinterpret_cast<uint2*>(p) = out;
  if (lane == 0) *scale = (uint8_t)(e + 127);
}

// A unit: (row, head), its key and its value; heads fastest, so that neighbours read one row of a
// product.  A thread takes U units, so that their chains of loads (position, page, values) run
// beside each other.
template <class T, class C, int LPU, int U, bool WRITE>
__global__ __launch_bounds__(256) void rows_kernel(RowArgs a) {
  const int lane = threadIdx.x % LPU, heads = a.at.heads, d = a.at.d;
  const int64_t unit0 = ((int64_t)blockIdx.x * 256 * U + threadIdx.x) / LPU;
  bool in[U];
  int64_t row[U], place[U];
  int head[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t unit = unit0 + u * (256 / LPU);
    row[u] = a.by_heads.quotient(unit);
    head[u] = (int)(unit - row[u] * heads);
    in[u] = row[u] < a.rows;
    row[u] = in[u] ? row[u] : a.rows - 1;
  }
  a.at.template of<U>(row, head, place);
  float y[U][2][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!in[u]) place[u] = kCacheNone;
    if (place[u] == kCacheBad && head[u] == 0 && lane == 0 && a.status) *a.status = 1;
    const float none = WRITE || place[u] != kCacheBad ? 0.f : NAN;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[u][i / 8][i % 8] = none;
    if (place[u] >= 0 && 8 * lane < d) {
      if constexpr (WRITE) {
        load8(reinterpret_cast<const T*>(a.k.p) + a.k.row * row[u] + a.k.head * head[u] + 8 * lane, y[u][0]);
        load8(reinterpret_cast<const T*>(a.v.p) + a.v.row * row[u] + a.v.head * head[u] + 8 * lane, y[u][1]);
      } else if constexpr (sizeof(C) == 1) {
        const int64_t at = place[u] * d + 8 * lane;
        load8_e4m3(reinterpret_cast<const uint8_t*>(a.ck) + at, e8m0(a.sk[place[u]]), y[u][0]);
        load8_e4m3(reinterpret_cast<const uint8_t*>(a.cv) + at, e8m0(a.sv[place[u]]), y[u][1]);
      } else {
        const int64_t at = place[u] * d + 8 * lane;
        load8(reinterpret_cast<const C*>(a.ck) + at, y[u][0]);
        load8(reinterpret_cast<const C*>(a.cv) + at, y[u][1]);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool real = place[u] >= 0 && 8 * lane < d;
    if constexpr (WRITE) {
      const int64_t safe = place[u] >= 0 ? place[u] : 0, at = safe * d + 8 * lane;
      if constexpr (sizeof(C) == 1) {
        store_e4m3<LPU>(reinterpret_cast<uint8_t*>(a.ck) + at, a.sk + safe, y[u][0], lane, real);
        store_e4m3<LPU>(reinterpret_cast<uint8_t*>(a.cv) + at, a.sv + safe, y[u][1], lane, real);
      } else if (real) {
        store8(reinterpret_cast<C*>(a.ck) + at, y[u][0]);
        store8(reinterpret_cast<C*>(a.cv) + at, y[u][1]);
      }
    } else if (place[u] != kCacheNone && 8 * lane < d) {
      store8(static_cast<T*>(const_cast<void*>(a.k.p)) + a.k.row * row[u] + a.k.head * head[u] + 8 * lane, y[u][0]);
      store8(static_cast<T*>(const_cast<void*>(a.v.p)) + a.v.row * row[u] + a.v.head * head[u] + 8 * lane, y[u][1]);
    }
  }
}

// From eight blocks a CU on, a thread takes two units of an 8-bit cache, whose loads are short.
// Measured on MI355X, us of write / read at one, two and four units a thread, 65,536 bf16 rows of
// 8 heads of 128: 8 bits 103 / 93, 91 / 90, 102 / 102 (4.5 TB/s); bf16 95 / 94 (5.7 TB/s),
// 100 / 100, 106 / 111.  A key and its value in units of their own, each with a chain of its own:
// 141 / 148 and 118 / 123.
constexpr int64_t MANY_BLOCKS = 2048;

template <class T, class C, int LPU, bool WRITE>
hipError_t launch_units(const RowArgs& a, hipStream_t s) {
  constexpr int MANY = sizeof(C) == 1 ? 2 : 1;
  const int64_t blocks = (a.rows * a.at.heads * LPU + 255) / 256;
  if (MANY == 1 || blocks < MANY_BLOCKS)
    hipLaunchKernelGGL((rows_kernel<T, C, LPU, 1, WRITE>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((rows_kernel<T, C, LPU, MANY, WRITE>), dim3((unsigned)((blocks + MANY - 1) / MANY)),
                       dim3(256), 0, s, a);
  return hipGetLastError();
}

template <class T, class C, bool WRITE>
hipError_t launch(const RowArgs& a, hipStream_t s) {
  int lpu = 1;
  while (8 * lpu < a.at.d) lpu *= 2;
  // lanes of a launch: 2^31 at most
  RowArgs b = a;
  const int64_t step = ((int64_t(1) << 31) / lpu) / a.at.heads;
  for (int64_t r = 0; r < a.rows; r += step) {
    b.rows = a.rows - r < step ? a.rows - r : step;
    b.at.first = r;
    const int esz = sizeof(T);
    b.k.p = (const char*)a.k.p + r * a.k.row * esz;
    b.v.p = (const char*)a.v.p + r * a.v.row * esz;
    hipError_t e;
    switch (lpu) {
      case 1: e = launch_units<T, C, 1, WRITE>(b, s); break;
      case 2: e = launch_units<T, C, 2, WRITE>(b, s); break;
      case 4: e = launch_units<T, C, 4, WRITE>(b, s); break;
      case 8: e = launch_units<T, C, 8, WRITE>(b, s); break;
      case 16: e = launch_units<T, C, 16, WRITE>(b, s); break;
      default: e = launch_units<T, C, 32, WRITE>(b, s); break;
    }
    if (e) return e;
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
  a.by_heads = divide_by(p.cache.heads);
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
