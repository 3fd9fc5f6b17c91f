// The L2 norm of a gradient of several tensors and its scaling to a largest norm
// (mpipe_op_grad_norm, mpipe_op_grad_clip).
//
//   S = sum g^2 (fp64), norm = sqrt(S), out = g * (norm > max ? max / norm : 1)
// Tensors are cut into chunks; their addresses travel in the kernels' arguments, a hundred or
// two tensors a launch.  Every chunk's sum goes to its own place and the places are added in
// order, so the result has the same bits every time.  fp64, because an fp32 square overflows at
// 1.8e19 and a sum of 10^8 of them needs more than 24 bits; it costs nothing.
//
// Bound by HBM: MI355X, 675.8 M fp32 elements in 392 tensors: norm 440 us (6.1 TB/s), clip into
// other buffers 1009 us (5.4); 32 tensors of 0.9 M bf16 elements 12 us in three launches.
#include <algorithm>

#include "common.h"
#include "layer_kernels.h"

namespace mpipe {
namespace {

constexpr int kNormTensors = 248, kClipTensors = 164;   // arguments below 4 KB

// A tensor in 16 bytes (24 with an output): its address, below 2^48, under the upper bits of
// its size; the size is elements * 4 + 1 where it is bf16, + 2 where its output is.
struct NormArgs {
  uint64_t at[kNormTensors];
  uint32_t size[kNormTensors];
  int32_t first[kNormTensors];   // first chunk, from chunk0
};
__host__ __device__ __forceinline__ uint64_t upper(uint64_t at, int64_t size) {
  return at | ((uint64_t)size >> 32) << 48;
}
struct Tensor {
  const char* p;
  int64_t n;
  bool in16, out16;
  __device__ __forceinline__ Tensor(uint64_t at, uint32_t size) {
    const uint64_t whole = (at >> 48) << 32 | size;
    p = reinterpret_cast<const char*>(at & 0xFFFFFFFFFFFFull);
    n = (int64_t)(whole >> 2);
    in16 = whole & 1;
    out16 = whole & 2;
  }
};

// The tensor of chunk c: how many first chunks are not behind it, less one.  All of them are
// compared at once, 64 a step.
template <int N>
__device__ __forceinline__ int tensor_of(const int32_t (&first)[N], int n, int c) {
  const int lane = threadIdx.x & 63;
  int t = -1;
#pragma unroll
  for (int k = 0; k < N; k += 64) {
    const bool before = k + lane < n && first[min(k + lane, N - 1)] <= c;
    t += __popcll(__ballot(before));
  }
  return __builtin_amdgcn_readfirstlane(t);
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += lds[w];
  __syncthreads();
  return s;
}

// E elements in words, aligned to one element: wide accesses take any alignment.
template <class T, int E> struct Group {
  static constexpr int kWords = E * sizeof(T) / 4;
  typedef uint32_t W __attribute__((ext_vector_type(kWords)));
  typedef W At __attribute__((aligned(sizeof(T))));
  W w;
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const At*>(p); }
  template <bool PAST> __device__ __forceinline__ void store(T* p) const {
    if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<At*>(p));
    else *reinterpret_cast<At*>(p) = w;
  }
  __device__ __forceinline__ float get(int i) const {
    if (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};
template <class T, int E>
__device__ __forceinline__ Group<T, E> pack(const float (&v)[E]) {
  Group<T, E> g;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; ++i) g.w[i] = __float_as_uint(v[i]);
  } else {
    typedef __bf16 Two __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const Two t = {(bf16)v[i], (bf16)v[i + 1]};
      g.w[i / 2] = __builtin_bit_cast(uint32_t, t);
    }
  }
  return g;
}

constexpr int kAhead = 8;   // 16-byte loads of a thread in flight

template <class T>
__device__ __forceinline__ double chunk_sum(const T* p, int n) {
  constexpr int E = 16 / sizeof(T);
  double s[2] = {0.0, 0.0};
  const int groups = n / E;
  int i = threadIdx.x;
  for (; i + (kAhead - 1) * 256 < groups; i += kAhead * 256) {
    Group<T, E> g[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) g[u].load(p + (int64_t)(i + u * 256) * E);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double v = (double)g[u].get(e);
        s[e % 2] = fma(v, v, s[e % 2]);
      }
  }
  for (; i < groups; i += 256) {
    Group<T, E> g;
    g.load(p + (int64_t)i * E);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double v = (double)g.get(e);
      s[e % 2] = fma(v, v, s[e % 2]);
    }
  }
  if (groups * E + (int)threadIdx.x < n) {
    const double v = (double)(float)p[groups * E + threadIdx.x];
    s[0] = fma(v, v, s[0]);
  }
  return s[0] + s[1];
}

// partial[chunk0 + block] = sum of squares of one chunk; starts[tensor] = its first chunk
__global__ __launch_bounds__(256) void sumsq_kernel(NormArgs a, int n, int tensor0, int chunk0,
                                                    int64_t chunk, double* partial,
                                                    int32_t* starts) {
  __shared__ double lds[4];
  const int c = blockIdx.x, t = tensor_of(a.first, n, c), nth = c - a.first[t];
  const Tensor x(a.at[t], a.size[t]);
  const int64_t at = nth * chunk;
  const int m = (int)(x.n - at < chunk ? x.n - at : chunk);
  const double s = block_sum(x.in16 ? chunk_sum((const bf16*)x.p + at, m)
                                    : chunk_sum((const float*)x.p + at, m), lds);
  if (threadIdx.x == 0) {
    partial[chunk0 + c] = s;
    if (nth == 0) starts[tensor0 + t] = chunk0 + c;
  }
}

// the thread's share of p[begin .. end): eight loads at once (those past the end repeat the last)
__device__ __forceinline__ double strided_sum(const double* p, int begin, int end) {
  double s = 0.0;
  for (int c = begin + threadIdx.x; c < end; c += 8 * 256) {
    double v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = p[min(c + u * 256, end - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += c + u * 256 < end ? v[u] : 0.0;
  }
  return s;
}

// block t: the sum of tensor t's chunks, its norm
__global__ __launch_bounds__(256) void tensor_sum_kernel(const double* partial,
                                                         const int32_t* starts, int n, int chunks,
                                                         double* sums, float* norms) {
  __shared__ double lds[4];
  const int t = blockIdx.x;
  const double s = block_sum(strided_sum(partial, starts[t], t + 1 < n ? starts[t + 1] : chunks), lds);
  if (threadIdx.x == 0) {
    sums[t] = s;
    if (norms) norms[t] = (float)sqrt(s);
  }
}

__global__ __launch_bounds__(256) void total_kernel(const double* sums, int n, double* sumsq) {
  __shared__ double lds[4];
  const double s = block_sum(strided_sum(sums, 0, n), lds);
  if (threadIdx.x == 0) *sumsq = s;
}

// Both steps in one block, where there are few tensors and chunks: the chunks' sums to LDS at
// once, then a wave a tensor.
constexpr int kFewTensors = 64, kFewChunks = 4096;
__global__ __launch_bounds__(1024) void few_sums_kernel(const double* partial,
                                                        const int32_t* starts, int n, int chunks,
                                                        float* norms, double* sumsq) {
  __shared__ double part[kFewChunks], sums[kFewTensors];
  __shared__ int32_t first[kFewTensors + 1];
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < kFewChunks; k += 1024)
    if (k + (int)threadIdx.x < chunks) part[k + threadIdx.x] = partial[k + threadIdx.x];
  if ((int)threadIdx.x <= n) first[threadIdx.x] = (int)threadIdx.x < n ? starts[threadIdx.x] : chunks;
  __syncthreads();
  for (int t = threadIdx.x >> 6; t < n; t += 16) {
    double s = 0.0;
#pragma unroll 8
    for (int c = first[t] + lane; c < first[t + 1]; c += 64) s += part[c];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) {
      sums[t] = s;
      if (norms) norms[t] = (float)sqrt(s);
    }
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    double s = lane < n ? sums[lane] : 0.0;
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) *sumsq = s;
  }
}

struct ClipArgs {
  uint64_t at[kClipTensors];
  void* out[kClipTensors];
  uint32_t size[kClipTensors];
  int32_t first[kClipTensors];
};

template <bool PAST, class A, class B>
__device__ __forceinline__ void chunk_scale(const A* p, B* o, int n, float f) {
  constexpr int E = sizeof(A) + sizeof(B) == 4 ? 8 : 4, U = 4;
  const int groups = n / E;
  int i = threadIdx.x;
  for (; i + (U - 1) * 256 < groups; i += U * 256) {
    Group<A, E> g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) g[u].load(p + (int64_t)(i + u * 256) * E);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = g[u].get(e) * f;
      pack<B, E>(v).template store<PAST>(o + (int64_t)(i + u * 256) * E);
    }
  }
  for (; i < groups; i += 256) {
    Group<A, E> g;
    g.load(p + (int64_t)i * E);
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = g.get(e) * f;
    pack<B, E>(v).template store<PAST>(o + (int64_t)i * E);
  }
  i = groups * E + threadIdx.x;
  if (i < n) o[i] = (B)((float)p[i] * f);
}

// The same by a factor that fp32 holds as a subnormal, or as zero: one fp64 product, rounded
// to fp32 once.  Such norms are beyond 1e35 times max_norm, so its time does not matter.
template <class A, class B>
__device__ __forceinline__ void chunk_scale_far(const A* p, B* o, int n, double f) {
  for (int i = threadIdx.x; i < n; i += 256) o[i] = (B)(float)((double)(float)p[i] * f);
}

template <bool PAST>
__global__ __launch_bounds__(256) void clip_kernel(ClipArgs a, int n, int64_t chunk,
                                                   const double* sumsq, double max_norm,
                                                   float* norm) {
  const double len2 = sqrt(*sumsq);
  const bool scales = len2 > max_norm && len2 <= 1.7976931348623157e308;
  const double f64 = scales ? max_norm / len2 : 1.0;
  const float f = (float)f64;
  // from the last chunk back: what the norm read last is cached still (1517 -> 1500 us)
  const int c = gridDim.x - 1 - blockIdx.x;
  if (norm && c == 0 && threadIdx.x == 0) *norm = (float)len2;
  if (n == 0) return;
  const int t = tensor_of(a.first, n, c);
  const Tensor x(a.at[t], a.size[t]);
  void* out = a.out[t];
  if (x.p == out && !scales) return;
  const int64_t at = (c - a.first[t]) * chunk;
  const int m = (int)(x.n - at < chunk ? x.n - at : chunk);
  if (f64 > 0.0 && f64 < 0x1p-126) {
    if (x.in16 && x.out16) chunk_scale_far((const bf16*)x.p + at, (bf16*)out + at, m, f64);
    else if (x.in16) chunk_scale_far((const bf16*)x.p + at, (float*)out + at, m, f64);
    else if (x.out16) chunk_scale_far((const float*)x.p + at, (bf16*)out + at, m, f64);
    else chunk_scale_far((const float*)x.p + at, (float*)out + at, m, f64);
    return;
  }
  if (x.in16 && x.out16) chunk_scale<PAST>((const bf16*)x.p + at, (bf16*)out + at, m, f);
  else if (x.in16) chunk_scale<PAST>((const bf16*)x.p + at, (float*)out + at, m, f);
  else if (x.out16) chunk_scale<PAST>((const float*)x.p + at, (bf16*)out + at, m, f);
  else chunk_scale<PAST>((const float*)x.p + at, (float*)out + at, m, f);
}

int chunks_of(int64_t n, int64_t chunk) { return (int)std::max<int64_t>(1, (n + chunk - 1) / chunk); }

}  // namespace

size_t grad_norm_scratch(int n, const GradPlan& p) {   // partials, tensor sums, first chunks
  return (size_t)p.chunks * 8 + (size_t)n * 8 + (size_t)n * 4 + 256;
}

hipError_t grad_norm(const mpipe_grad_tensor* t, int n, const GradPlan& p, double* sumsq,
                     float* norms, char* scratch, hipStream_t s) {
  double* partial = reinterpret_cast<double*>(scratch);
  double* sums = partial + p.chunks;
  int32_t* starts = reinterpret_cast<int32_t*>(sums + n);
  int chunk0 = 0;
  for (int i = 0; i < n;) {
    NormArgs a;
    const int tensor0 = i;
    int k = 0, c = 0;
    for (; i < n && k < kNormTensors; ++i, ++k) {
      const int64_t size = t[i].n * 4 + (t[i].dtype == DT_BF16);
      a.at[k] = upper((uintptr_t)t[i].data, size);
      a.size[k] = (uint32_t)size;
      a.first[k] = c;
      c += chunks_of(t[i].n, p.chunk);
    }
    hipLaunchKernelGGL(sumsq_kernel, dim3(c), dim3(256), 0, s, a, k, tensor0, chunk0, p.chunk,
                       partial, starts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    chunk0 += c;
  }
  if (n <= kFewTensors && p.chunks <= kFewChunks) {
    hipLaunchKernelGGL(few_sums_kernel, dim3(1), dim3(1024), 0, s, partial, starts, n,
                       (int)p.chunks, norms, sumsq);
    return hipGetLastError();
  }
  if (n > 0) {
    hipLaunchKernelGGL(tensor_sum_kernel, dim3(n), dim3(256), 0, s, partial, starts, n,
                       (int)p.chunks, sums, norms);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(total_kernel, dim3(1), dim3(256), 0, s, sums, n, sumsq);
  return hipGetLastError();
}

hipError_t grad_clip(const mpipe_grad_tensor* in, const mpipe_grad_tensor* out, int n,
                     const GradPlan& p, const double* sumsq, double max_norm, float* norm,
                     hipStream_t s) {
  // Outputs of more than the 256 MB of last-level cache are stored past it: the Qwen2-VL
  // shape's fp32 gradient 1500 -> 1459 us.
  int64_t bytes = 0;
  for (int i = 0; i < n; ++i) bytes += out[i].n * (out[i].dtype == DT_BF16 ? 2 : 4);
  const bool past_caches = bytes > int64_t(256) << 20;
  // from the last tensors to the first, as within a launch
  int end = n;
  do {
    ClipArgs a;
    const int begin = std::max(0, end - kClipTensors);
    int c = 0;
    for (int i = begin; i < end; ++i) {
      const int k = i - begin;
      const int64_t size = in[i].n * 4 + (in[i].dtype == DT_BF16) + 2 * (out[i].dtype == DT_BF16);
      a.at[k] = upper((uintptr_t)in[i].data, size);
      a.out[k] = out[i].data;
      a.size[k] = (uint32_t)size;
      a.first[k] = c;
      c += chunks_of(in[i].n, p.chunk);
    }
    hipLaunchKernelGGL(past_caches ? clip_kernel<true> : clip_kernel<false>, dim3(std::max(c, 1)),
                       dim3(256), 0, s, a, end - begin, p.chunk, sumsq, max_norm, norm);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    norm = nullptr;
    end = begin;
  } while (end > 0);
  return hipSuccess;
}

}  // namespace mpipe
