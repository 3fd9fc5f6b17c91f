// Rotary positions with several axes on q and k heads, alone or behind a root-mean-square
// norm of every head with a gain, and that norm's backward (mpipe_ops.h).
//
//   u = R^T dy, r = (mean x^2 + eps)^(-1/2):  y = R (g x r),  dg = sum u x r,
//   dx = r (g u - x r^2 mean(g u x))
// R turns the pair (a, b) by the angle of its axis' position: (a c - b s, b c + a s).
#include <algorithm>

#include "common.h"
#include "layer_kernels.h"

namespace mpipe {
namespace {

struct SideArgs {
  const char* x;
  const char* dy;
  char* y;
  int64_t x_row, x_head, dy_row, dy_head, y_row, y_head;   // elements
  const void* gain;
  float* part;   // backward: [blocks][head_dim]
  int heads, blocks;
  // heads a wave holds at once (log2), its walks over a row's heads, waves per row group,
  // row groups times those
  int log_h, iters, head_groups, items;
};

struct QkArgs {
  SideArgs side[2];
  const int32_t* pos;
  int64_t ld_pos, rows;
  float eps, inv_d;
  int d, half, inverse;
  int log_c;   // lanes of a head (log2)
  RopeTable table;
};

// cos and sin of p * f / 2^64 turns.  The product modulo 2^64 is the angle modulo one turn,
// exactly; what is left to the nearest quarter turn, |x| <= pi / 4, goes through the Taylor
// series (to x^9 and x^10: below 4e-9 of truncation).
__device__ __forceinline__ void turn_cos_sin(uint64_t f, int32_t p, float& c, float& s) {
  const uint64_t t = f * (uint64_t)(int64_t)p;
  const uint32_t q = ((uint32_t)(t >> 32) + 0x20000000u) >> 30;
  const int64_t rem = (int64_t)(t - ((uint64_t)q << 62));   // [-2^61, 2^61)
  // the top 24 bits and the 32 below them, each times 2 pi / 2^32 in two fp32 parts
  const int32_t top = (int32_t)(rem >> 32) & ~0x3F;
  const float rest = (float)(uint32_t)(rem >> 6) * 0x1.921fb6p-56f;
  const float x = fmaf((float)top, 0x1.921fb6p-30f, fmaf((float)top, -0x1.777a5cp-55f, rest));
  const float z = x * x;
  const float ps = fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
  const float sn = fmaf(x * z, ps, x);
  const float pc = fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f);
  const float h = 0.5f * z, w = 1.f - h;
  const float cn = w + fmaf(z * z, pc, (1.f - w) - h);
  const float a = (q & 1) ? sn : cn, b = (q & 1) ? cn : sn;
  c = (q == 1 || q == 2) ? -a : a;
  s = (q >= 2) ? -b : b;
}

// V elements as words, aligned to one element: global accesses of 16 bytes take any alignment.
template <class T, int V> struct Vec;
template <> struct Vec<float, 4> {
  typedef uint32_t W __attribute__((ext_vector_type(4)));
  typedef W At __attribute__((aligned(4)));
};
template <> struct Vec<bf16, 8> {
  typedef uint32_t W __attribute__((ext_vector_type(4)));
  typedef W At __attribute__((aligned(2)));
};
template <> struct Vec<bf16, 4> {
  typedef uint32_t W __attribute__((ext_vector_type(2)));
  typedef W At __attribute__((aligned(2)));
};
template <class T, int V> using Words = typename Vec<T, V>::W;

// What a lane does in every head it takes: V pairs (2 V columns) or, behind the rotated
// columns, 2 V columns that pass through.  col[0] and col[1] each start V adjacent columns;
// with halves they are rot / 2 apart.
template <int V, bool ADJ> struct Lane {
  int col[2];
  bool on[2], turns;
  __device__ __forceinline__ Lane(int c, int half, int d) {
    turns = c * V < half;
    if (turns && !ADJ) {
      col[0] = c * V;
      col[1] = half + c * V;
    } else {
      col[0] = 2 * c * V;
      col[1] = 2 * c * V + V;
    }
    on[0] = col[0] < d;
    on[1] = col[1] < d;
  }
  static __device__ __forceinline__ constexpr int first(int i) { return ADJ ? 2 * i : i; }
  static __device__ __forceinline__ constexpr int second(int i) { return ADJ ? 2 * i + 1 : V + i; }
};

// Lanes that are off keep whatever their registers held: what they compute is not stored, and
// columns past the head are set to zero before a sum.  (Zeroing the registers first would
// make every load wait for the one before.)
template <class T, int V>
__device__ __forceinline__ void load_head(const T* p, const int64_t (&off)[2], const bool (&on)[2],
                                          bool head, Words<T, V> (&r)[2]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    r[k] = __builtin_nondeterministic_value(r[k]);
    if (head && on[k]) r[k] = *reinterpret_cast<const typename Vec<T, V>::At*>(p + off[k]);
  }
}
template <class T, int V>
__device__ __forceinline__ void widen(const Words<T, V> (&r)[2], const bool (&on)[2],
                                      float (&v)[2 * V]) {
  constexpr int E = 4 / sizeof(T);   // elements of a word
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    const uint32_t w = r[i / V][i % V / E];
    v[i] = on[i / V] ? __uint_as_float(E == 1 ? w : i % 2 ? w & 0xFFFF0000u : w << 16) : 0.f;
  }
}
template <class T, int V>
__device__ __forceinline__ void store_head(T* p, const int64_t (&off)[2], const bool (&on)[2],
                                           bool head, const float (&v)[2 * V]) {
  constexpr int E = 4 / sizeof(T);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    Words<T, V> r;
#pragma unroll
    for (int i = 0; i < V / E; ++i) {
      if constexpr (E == 1) {
        r[i] = __float_as_uint(v[k * V + i]);
      } else {
        typedef __bf16 Two __attribute__((ext_vector_type(2)));
        const Two t = {(bf16)v[k * V + 2 * i], (bf16)v[k * V + 2 * i + 1]};
        r[i] = __builtin_bit_cast(uint32_t, t);
      }
    }
    if (head && on[k]) *reinterpret_cast<typename Vec<T, V>::At*>(p + off[k]) = r;
  }
}

// sum over the 1 << log_c adjacent lanes that hold one head
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float head_sum(float v, int log_c) {
  if (log_c > 0) v = dpp_add<0xB1>(v);    // lane ^ 1
  if (log_c > 1) v = dpp_add<0x4E>(v);    // lane ^ 2
  if (log_c > 2) v = dpp_add<0x141>(v);   // mirrored within 8
  if (log_c > 3) v = dpp_add<0x140>(v);   // mirrored within 16
  if (log_c > 4) v += __shfl_xor(v, 16);
  return v;
}
__device__ __forceinline__ float inv_rms(float ss, float inv_d, float eps) {
  const float m = fmaf(ss, inv_d, eps), r = __builtin_amdgcn_rsqf(m);
  return fmaf(0.5f * r, fmaf(-m * r, r, 1.f), r);   // one Newton step: the root to half a step
}

// cos and sin of a wave's rows: each row's lanes share its rot / 2 pairs and meet in LDS
__device__ __forceinline__ void wave_trig(const QkArgs& a, float* cs, float* sn, int64_t row,
                                          int rs, int sub, int width) {
  if (row < a.rows)
    for (int j = sub; j < a.half; j += width) {
      float c, s;
      turn_cos_sin(a.table.turn[j], a.pos[a.table.axis[j] * a.ld_pos + row], c, s);
      cs[rs * a.half + j] = c;
      sn[rs * a.half + j] = a.inverse ? -s : s;
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int V, bool ADJ>
__device__ __forceinline__ void turn(const Lane<V, ADJ>& l, const float (&c)[V], const float (&s)[V],
                                     float (&v)[2 * V]) {
  if (!l.turns) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int p = l.first(i), q = l.second(i);
    const float x = v[p], y = v[q], xs = x * s[i], ys = y * s[i];
    v[p] = fmaf(x, c[i], -ys);
    v[q] = fmaf(y, c[i], xs);
  }
}

// A wave is (rows) x (heads) x (lanes of a head), powers of two: 64 >> (log_c + log_h) rows,
// 1 << log_h heads, walked `iters` times over a row's heads.
struct Place {
  int c, hs, rs, sub;
  __device__ __forceinline__ Place(int lane, int log_c, int log_h) {
    c = lane & ((1 << log_c) - 1);
    hs = (lane >> log_c) & ((1 << log_h) - 1);
    rs = lane >> (log_c + log_h);
    sub = lane & ((1 << (log_c + log_h)) - 1);
  }
};
constexpr int kTrig = 512;   // pairs of a wave's rows: at most 64 lanes * 8

// A view as a wave walks it: the lane's offsets from the wave's first row and head, and the
// (scalar) way to those.
template <class T> struct Walk {
  const T* base;
  int64_t row, head, off[2];
  __device__ __forceinline__ Walk(const void* p, int64_t row_stride, int64_t head_stride,
                                  const Place& at, const int (&col)[2])
      : base(reinterpret_cast<const T*>(p)), row(row_stride), head(head_stride) {
    for (int k = 0; k < 2; ++k) off[k] = at.rs * row + at.hs * head + col[k];
  }
  __device__ __forceinline__ const T* at(int64_t r, int h) const { return base + r * row + h * head; }
};

template <class T, int V, bool ADJ, bool NORM>
__global__ __launch_bounds__(256, 4) void qk_fwd_kernel(QkArgs a) {
  constexpr int U = 2;   // heads loaded ahead
  __shared__ float trig[4][2][kTrig];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int z = (int)blockIdx.x >= a.side[0].blocks;
  const SideArgs& sd = a.side[z];
  const int log_c = a.log_c, log_h = sd.log_h, block = blockIdx.x - (z ? a.side[0].blocks : 0);
  const Place at(lane, log_c, log_h);
  const Lane<V, ADJ> l(at.c, a.half, a.d);
  const Walk<T> x(sd.x, sd.x_row, sd.x_head, at, l.col), y(sd.y, sd.y_row, sd.y_head, at, l.col);
  float* cs = trig[wave][0];
  float* sn = trig[wave][1];
  float g[2 * V];
  if (NORM) {
    Words<T, V> r[2];
    const int64_t off[2] = {l.col[0], l.col[1]};
    load_head<T, V>(reinterpret_cast<const T*>(sd.gain), off, l.on, true, r);
    widen<T, V>(r, l.on, g);
  }
  for (int item = block * 4 + wave; item < sd.items; item += sd.blocks * 4) {
    const int rg = item / sd.head_groups, hg = item - rg * sd.head_groups;
    const int64_t row0 = (int64_t)rg << (6 - log_c - log_h);
    const int head0 = (hg * sd.iters) << log_h, n = min(sd.iters << log_h, sd.heads - head0);
    const int left = row0 + at.rs < a.rows ? n - at.hs : 0;   // heads from the lane's first on
    Words<T, V> r[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
      load_head<T, V>(x.at(row0, head0 + (u << log_h)), x.off, l.on, (u << log_h) < left, r[u]);
    wave_trig(a, cs, sn, row0 + at.rs, at.rs, at.sub, 1 << (log_c + log_h));
    float c[V], s[V];
    if (l.turns) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        c[i] = cs[at.rs * a.half + at.c * V + i];
        s[i] = sn[at.rs * a.half + at.c * V + i];
      }
    }
    __builtin_amdgcn_wave_barrier();
    for (int h = 0;;) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + (u << log_h) >= n) break;
        __builtin_amdgcn_sched_barrier(0);   // one head at a time, or registers run out
        float v[2 * V];
        widen<T, V>(r[u], l.on, v);
        if (NORM) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) ss = fmaf(v[i], v[i], ss);
          const float k = inv_rms(head_sum(ss, log_c), a.inv_d, a.eps);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) v[i] = v[i] * k * g[i];
        }
        turn<V, ADJ>(l, c, s, v);
        store_head<T, V>(const_cast<T*>(y.at(row0, head0 + h + (u << log_h))), y.off, l.on,
                         h + (u << log_h) < left, v);
      }
      h += U << log_h;
      if (h >= n) break;
#pragma unroll
      for (int u = 0; u < U; ++u)
        load_head<T, V>(x.at(row0, head0 + h + (u << log_h)), x.off, l.on,
                        h + (u << log_h) < left, r[u]);
    }
  }
}

template <class T, int V, bool ADJ>
__global__ __launch_bounds__(256, 3) void qk_bwd_kernel(QkArgs a) {
  constexpr int U = 2;
  __shared__ float trig[4][2][kTrig];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int z = (int)blockIdx.x >= a.side[0].blocks;
  const SideArgs& sd = a.side[z];
  const int log_c = a.log_c, log_h = sd.log_h, block = blockIdx.x - (z ? a.side[0].blocks : 0);
  const Place at(lane, log_c, log_h);
  const Lane<V, ADJ> l(at.c, a.half, a.d);
  const Walk<T> x(sd.x, sd.x_row, sd.x_head, at, l.col), dy(sd.dy, sd.dy_row, sd.dy_head, at, l.col),
      y(sd.y, sd.y_row, sd.y_head, at, l.col);
  float* cs = trig[wave][0];
  float* sn = trig[wave][1];
  float g[2 * V], dg[2 * V];
  {
    Words<T, V> r[2];
    const int64_t off[2] = {l.col[0], l.col[1]};
    load_head<T, V>(reinterpret_cast<const T*>(sd.gain), off, l.on, true, r);
    widen<T, V>(r, l.on, g);
  }
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) dg[i] = 0.f;
  for (int item = block * 4 + wave; item < sd.items; item += sd.blocks * 4) {
    const int rg = item / sd.head_groups, hg = item - rg * sd.head_groups;
    const int64_t row0 = (int64_t)rg << (6 - log_c - log_h);
    const int head0 = (hg * sd.iters) << log_h, n = min(sd.iters << log_h, sd.heads - head0);
    const int left = row0 + at.rs < a.rows ? n - at.hs : 0;
    Words<T, V> rx[U][2], rd[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      load_head<T, V>(x.at(row0, head0 + (u << log_h)), x.off, l.on, (u << log_h) < left, rx[u]);
      load_head<T, V>(dy.at(row0, head0 + (u << log_h)), dy.off, l.on, (u << log_h) < left, rd[u]);
    }
    wave_trig(a, cs, sn, row0 + at.rs, at.rs, at.sub, 1 << (log_c + log_h));
    float c[V], s[V];
    if (l.turns) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        c[i] = cs[at.rs * a.half + at.c * V + i];
        s[i] = sn[at.rs * a.half + at.c * V + i];
      }
    }
    __builtin_amdgcn_wave_barrier();
    for (int h = 0;;) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + (u << log_h) >= n) break;
        __builtin_amdgcn_sched_barrier(0);   // one head at a time, or registers run out
        const bool head = h + (u << log_h) < left, on[2] = {head && l.on[0], head && l.on[1]};
        float v[2 * V], w[2 * V];
        widen<T, V>(rx[u], on, v);
        widen<T, V>(rd[u], on, w);
        turn<V, ADJ>(l, c, s, w);
        float ss = 0.f, sw = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
          ss = fmaf(v[i], v[i], ss);
          sw = fmaf(w[i] * g[i], v[i], sw);
        }
        const float k = inv_rms(head_sum(ss, log_c), a.inv_d, a.eps);
        const float m = k * k * head_sum(sw, log_c) * a.inv_d;
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
          dg[i] = fmaf(w[i], v[i] * k, dg[i]);
          w[i] = k * fmaf(w[i], g[i], -v[i] * m);
        }
        store_head<T, V>(const_cast<T*>(y.at(row0, head0 + h + (u << log_h))), y.off, l.on, head, w);
      }
      h += U << log_h;
      if (h >= n) break;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        load_head<T, V>(x.at(row0, head0 + h + (u << log_h)), x.off, l.on,
                        h + (u << log_h) < left, rx[u]);
        load_head<T, V>(dy.at(row0, head0 + h + (u << log_h)), dy.off, l.on,
                        h + (u << log_h) < left, rd[u]);
      }
    }
  }
  if (!sd.part) return;
  // the lanes of one column: over the wave, then over the block's waves through LDS
  __syncthreads();
  float* cols = &trig[0][0][0];
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    for (int o = 1 << log_c; o < 64; o <<= 1) dg[i] += __shfl_xor(dg[i], o);
    if (lane < (1 << log_c) && l.on[i / V]) cols[wave * kMaxHeadDim + l.col[i / V] + i % V] = dg[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.d; i += 256)
    sd.part[(int64_t)block * a.d + i] = (cols[i] + cols[kMaxHeadDim + i]) +
                                        (cols[2 * kMaxHeadDim + i] + cols[3 * kMaxHeadDim + i]);
}

// grad[z][c] (+)= sum of part[z][b][c] over the blocks, in order
struct GainArgs {
  const float* part[2];
  float* grad[2];
  int blocks[2];
  int d, accumulate;
};
// 8 columns x 32 lanes of blocks; blocks of a lane in order, then the lanes
__global__ __launch_bounds__(256) void gain_reduce_kernel(GainArgs a) {
  __shared__ float lds[32][9];
  const int z = blockIdx.y, cl = threadIdx.x & 7, bl = threadIdx.x >> 3, c = blockIdx.x * 8 + cl;
  if (!a.grad[z]) return;
  float s = 0.f;
#pragma unroll 4
  for (int b = bl; b < a.blocks[z]; b += 32) s += a.part[z][(int64_t)b * a.d + c];
  lds[bl][cl] = s;
  __syncthreads();
  for (int o = 16; o > 0; o >>= 1) {
    if (bl < o) lds[bl][cl] += lds[bl + o][cl];
    __syncthreads();
  }
  if (bl == 0) a.grad[z][c] = a.accumulate ? a.grad[z][c] + lds[0][cl] : lds[0][cl];
}

int log2_up(int n) {
  int l = 0;
  while ((1 << l) < n) ++l;
  return l;
}

// Eight columns a vector (16 bytes of bf16) where pairs and tail divide by it, else four.
int vector_of(int dtype, int half, int d) {
  return dtype == DT_BF16 && half % 8 == 0 && (d - 2 * half) % 8 == 0 ? 8 : 4;
}
int lanes_log2(int v, int half, int d) {   // lanes of a head
  return log2_up(half / v + (d - 2 * half + 2 * v - 1) / (2 * v));
}

constexpr int kWaves = 4096;    // enough waves for 256 compute units
constexpr int kFwdBlocks = 4096;

// Heads a wave holds at once: as few idle slots over a row's heads as can be, then as many
// heads as can be (a row's angles are worked out once per wave).  Few rows are spread over
// the heads too.
void divide(SideArgs& s, int64_t rows, int log_c, int max_blocks) {
  if (s.heads == 0 || rows == 0) return;   // no items, no blocks
  int best = 0, idle = 1 << 30;
  for (int h = 0; h <= 6 - log_c; ++h) {
    const int n = (s.heads + (1 << h) - 1) >> h, waste = (n << h) - s.heads;
    if (waste <= idle) {
      idle = waste;
      best = h;
    }
  }
  const int rs = 6 - log_c - best;
  const int64_t groups = (rows + (1 << rs) - 1) >> rs;
  const int iters = (s.heads + (1 << best) - 1) >> best;
  s.log_h = best;
  s.head_groups = (int)std::max<int64_t>(1, std::min<int64_t>(iters, kWaves / groups));
  s.iters = (iters + s.head_groups - 1) / s.head_groups;
  s.head_groups = (iters + s.iters - 1) / s.iters;
  s.items = (int)(groups * s.head_groups);
  s.blocks = std::min((s.items + 3) / 4, max_blocks);
}

constexpr int kBwdBlocks = 512;

QkArgs device_args(const QkProblem& p, int v) {
  QkArgs a;
  for (int z = 0; z < 2; ++z) {
    const QkSide& s = p.side[z];
    a.side[z] = {(const char*)s.x.p, (const char*)s.dy.p, (char*)s.y.p, s.x.row, s.x.head,
                 s.dy.row, s.dy.head, s.y.row, s.y.head, s.gain, nullptr, s.x.heads, 0, 0, 0, 0, 0};
  }
  a.pos = p.pos;
  a.ld_pos = p.ld_pos;
  a.rows = p.rows;
  a.eps = p.eps;
  a.inv_d = 1.f / (float)p.head_dim;
  a.d = p.head_dim;
  a.half = p.rot_dim / 2;
  a.inverse = p.inverse;
  a.log_c = lanes_log2(v, a.half, a.d);
  a.table = p.table;
  return a;
}

}  // namespace

hipError_t qk_rope_fwd(const QkProblem& p, hipStream_t s) {
  if (p.rows == 0) return hipSuccess;
  const int v = vector_of(p.dtype, p.rot_dim / 2, p.head_dim);
  QkArgs a = device_args(p, v);
  for (SideArgs& sd : a.side) divide(sd, p.rows, a.log_c, kFwdBlocks);
  const dim3 grid(a.side[0].blocks + a.side[1].blocks);
  if (grid.x == 0) return hipSuccess;
#define MPIPE_QK(T, V)                                                                            \
  do {                                                                                            \
    if (p.adjacent) {                                                                             \
      if (p.norm) hipLaunchKernelGGL((qk_fwd_kernel<T, V, true, true>), grid, dim3(256), 0, s, a); \
      else hipLaunchKernelGGL((qk_fwd_kernel<T, V, true, false>), grid, dim3(256), 0, s, a);      \
    } else {                                                                                      \
      if (p.norm) hipLaunchKernelGGL((qk_fwd_kernel<T, V, false, true>), grid, dim3(256), 0, s, a); \
      else hipLaunchKernelGGL((qk_fwd_kernel<T, V, false, false>), grid, dim3(256), 0, s, a);     \
    }                                                                                             \
  } while (0)
  if (p.dtype == DT_F32) MPIPE_QK(float, 4);
  else if (v == 8) MPIPE_QK(bf16, 8);
  else MPIPE_QK(bf16, 4);
#undef MPIPE_QK
  return hipGetLastError();
}

size_t qk_norm_rope_bwd_scratch(int64_t rows, int heads_q, int heads_k, int head_dim) {
  const auto blocks = [&](int heads) { return (size_t)std::min<int64_t>(rows * heads, kBwdBlocks); };
  return (blocks(heads_q) + blocks(heads_k)) * head_dim * 4 + 256;
}

hipError_t qk_norm_rope_bwd(const QkProblem& p, bool accumulate, float* scratch, hipStream_t s) {
  const int v = vector_of(p.dtype, p.rot_dim / 2, p.head_dim);
  QkArgs a = device_args(p, v);
  GainArgs r;
  bool any = false;
  for (int z = 0; z < 2; ++z) {
    SideArgs& sd = a.side[z];
    divide(sd, p.rows, a.log_c, kBwdBlocks);
    sd.part = p.side[z].grad ? scratch : nullptr;
    r.part[z] = scratch;
    r.grad[z] = p.side[z].grad;
    r.blocks[z] = sd.blocks;
    scratch += (int64_t)sd.blocks * p.head_dim;
    any |= p.side[z].grad != nullptr;
  }
  const dim3 grid(a.side[0].blocks + a.side[1].blocks);
  if (grid.x > 0) {
#define MPIPE_QK(T, V)                                                                            \
  do {                                                                                            \
    if (p.adjacent) hipLaunchKernelGGL((qk_bwd_kernel<T, V, true>), grid, dim3(256), 0, s, a);    \
    else hipLaunchKernelGGL((qk_bwd_kernel<T, V, false>), grid, dim3(256), 0, s, a);              \
  } while (0)
    if (p.dtype == DT_F32) MPIPE_QK(float, 4);
    else if (v == 8) MPIPE_QK(bf16, 8);
    else MPIPE_QK(bf16, 4);
#undef MPIPE_QK
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!any) return hipSuccess;
  r.d = p.head_dim;
  r.accumulate = accumulate;
  hipLaunchKernelGGL(gain_reduce_kernel, dim3(p.head_dim / 8, 2), dim3(256), 0, s, r);
  return hipGetLastError();
}

}  // namespace mpipe
