// Rotary positions with several axes on q and k heads, alone or behind a root-mean-square
// norm of every head with a gain, and that norm's backward (mpipe_ops.h).
//
//   u = R^T dy, r = (mean x^2 + eps)^(-1/2):  y = R (g x r),  dg = sum u x r,
//   dx = r (g u - x r^2 mean(g u x))
// R turns the pair (a, b) by the angle of its axis' position: (a c - b s, b c + a s).
//
// Bound by HBM: q and k are read and written once (the backward reads their output gradients
// too).  MI355X, 65536 rows, 28 + 4 heads of 128, bf16: rotation 192 us (5.6 TB/s), norm
// backward 308 us (5.2); 42940 rows, 16 + 16 heads of 80, norm forward 93 us (4.7; five of eight
// lanes hold a head); a copy of 4 GiB runs at 4.8.  Few rows take 4.5 us, one chain of loads.
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
  // heads a wave holds at once (log2), its steps over a row's heads, waves that share a row,
  // groups of as many rows as a wave holds
  int log_h, iters, head_groups, groups;
};

struct QkArgs {
  SideArgs side[2];
  const int32_t* pos;
  int64_t ld_pos, rows;
  float eps, inv_d;
  int d, half, inverse;
  int lanes, log_c;   // lanes of a head that hold columns; the power of two above (log2)
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

// Pointers that came through a table of views: known to be global memory, so that loads are
// counted apart from LDS accesses.
#define MPIPE_GLOBAL __attribute__((address_space(1)))

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
// columns, 2 V columns that pass through (V where `two` is off: the second V repeat them).
// col[0] and col[1] each start V adjacent columns; with halves they are rot / 2 apart.
template <int V, bool ADJ> struct Lane {
  int col[2];
  bool two, turns;
  __device__ __forceinline__ Lane(int c, int half, int d) {
    turns = c * V < half;
    if (turns && !ADJ) {
      col[0] = c * V;
      col[1] = half + c * V;
    } else {
      col[0] = 2 * c * V;
      col[1] = 2 * c * V + V;
    }
    two = col[1] < d;
    if (!two) col[1] = col[0];
  }
  static __device__ __forceinline__ constexpr int first(int i) { return ADJ ? 2 * i : i; }
  static __device__ __forceinline__ constexpr int second(int i) { return ADJ ? 2 * i + 1 : V + i; }
};

template <class T, int V>
__device__ __forceinline__ void load_head(const T* const (&p)[2], Words<T, V> (&r)[2]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) r[k] = *(const MPIPE_GLOBAL typename Vec<T, V>::At*)p[k];
}
template <class T, int V>
__device__ __forceinline__ void widen(const Words<T, V> (&r)[2], float (&v)[2 * V]) {
  constexpr int E = 4 / sizeof(T);   // elements of a word
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    const uint32_t w = r[i / V][i % V / E];
    v[i] = __uint_as_float(E == 1 ? w : i % 2 ? w & 0xFFFF0000u : w << 16);
  }
}
template <class T, int V, bool PAST>
__device__ __forceinline__ void store_head(const T* const (&p)[2], const float (&v)[2 * V]) {
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
    const auto to = (MPIPE_GLOBAL typename Vec<T, V>::At*)const_cast<T*>(p[k]);
    if constexpr (PAST) __builtin_nontemporal_store(r, to);
    else *to = r;
  }
}

// sum over the 1 << log_c adjacent lanes that hold one head
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float head_sum(float v, int log_c) {
  float w = dpp_add<0xB1>(v);     // lane ^ 1
  v = log_c > 0 ? w : v;
  w = dpp_add<0x4E>(v);           // lane ^ 2
  v = log_c > 1 ? w : v;
  w = dpp_add<0x141>(v);          // mirrored within 8
  v = log_c > 2 ? w : v;
  w = dpp_add<0x140>(v);          // mirrored within 16
  v = log_c > 3 ? w : v;
  if (log_c > 4) v += __shfl_xor(v, 16);
  return v;
}
__device__ __forceinline__ float inv_rms(float ss, float inv_d, float eps) {
  const float m = fmaf(ss, inv_d, eps), r = __builtin_amdgcn_rsqf(m);
  // one Newton step: the root to half a step (an infinite mean keeps its 0)
  return m < __builtin_inff() ? fmaf(0.5f * r, fmaf(-m * r, r, 1.f), r) : r;
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
// 1 << log_h heads.  It walks its share of a row's heads, then the next rows of its stride,
// `kRing` steps of loads ahead of the arithmetic.
//
// Every lane of a step loads and stores, so that the loads in flight can be counted and only
// the oldest waited for: lanes past the last row, head or column repeat the last one, with the
// same values to the same place, and are left out of the sums.
struct Place {
  int c, hs, rs, sub;
  bool extra;   // a column lane past the head's last
  __device__ __forceinline__ Place(int lane, int log_c, int log_h, int lanes) {
    const int l = lane & ((1 << log_c) - 1);
    c = min(l, lanes - 1);
    extra = l >= lanes;
    hs = (lane >> log_c) & ((1 << log_h) - 1);
    rs = lane >> (log_c + log_h);
    sub = lane & ((1 << (log_c + log_h)) - 1);
  }
};

// Where a wave is in its rows and heads.
struct Cursor {
  int rg, h;
  __device__ __forceinline__ void next(int h_step, int n, int rg_step) {
    h += h_step;
    if (h >= n) {
      h = 0;
      rg += rg_step;
    }
  }
};

// A view as a wave walks it: the lane's offsets from the step's first row and head.
template <class T> struct Walk {
  const T* base;   // first row, the wave's first head
  int64_t row, head, off[2];
  __device__ __forceinline__ Walk(const void* p, int64_t row_stride, int64_t head_stride,
                                  const Place& at, int head0, const int (&col)[2])
      : base(reinterpret_cast<const T*>(p) + head0 * head_stride), row(row_stride),
        head(head_stride) {
    for (int k = 0; k < 2; ++k) off[k] = at.rs * row + at.hs * head + col[k];
  }
  // the lane's two vectors at `row0` and head h; `drs`, `dhs`: how far it is past the last
  __device__ __forceinline__ void at(int64_t row0, int h, int drs, int dhs, bool edge,
                                     const T* (&p)[2]) const {
    const T* b = base + row0 * row + h * head;
    p[0] = b + off[0];
    p[1] = b + off[1];
    if (edge) {
      const int64_t back = drs * row + dhs * head;
      p[0] -= back;
      p[1] -= back;
    }
  }
};

constexpr int kTrig = 512;   // pairs of a wave's rows: at most 64 lanes * 8

// What both kernels keep of a wave's walk.
template <class T, int V, bool ADJ, int KP> struct Wave {
  const QkArgs& a;
  const int log_c, log_h, rs_log;
  const Place at;
  const Lane<V, ADJ> l;
  int rg0, rg_step, groups, head0, n;
  bool idle;
  float *cs, *sn;
  const uint64_t* turns;
  const int32_t* pos[KP];

  __device__ __forceinline__ Wave(const QkArgs& a, const SideArgs& sd, int w, float* trig,
                                  const uint64_t* turn_table, const uint8_t* axis_table)
      : a(a), log_c(a.log_c), log_h(sd.log_h), rs_log(6 - a.log_c - sd.log_h),
        at(threadIdx.x & 63, a.log_c, sd.log_h, a.lanes), l(at.c, a.half, a.d) {
    const int hg = w % sd.head_groups;
    rg0 = w / sd.head_groups;
    rg_step = sd.blocks * 4 / sd.head_groups;
    groups = sd.groups;
    idle = rg0 >= min(rg_step, groups);   // a grid's last waves may have no rows of their own
    rg0 = min(rg0, groups - 1);
    head0 = (hg * sd.iters) << log_h;
    n = min(sd.iters << log_h, sd.heads - head0);
    cs = trig;
    sn = trig + kTrig;
    turns = turn_table;
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int j = min(at.sub + (k << (log_c + log_h)), a.half - 1);
      pos[k] = a.pos + axis_table[j] * a.ld_pos + at.rs;
    }
  }
  __device__ __forceinline__ int64_t row0(int rg) const { return (int64_t)rg << rs_log; }
  // how far the lane is past the last row / head of a step
  __device__ __forceinline__ int past_rows(int rg) const {
    return max(0, at.rs - (int)min((int64_t)64, a.rows - 1 - row0(rg)));
  }
  __device__ __forceinline__ int past_heads(int h) const { return max(0, at.hs - (n - 1 - h)); }
  __device__ __forceinline__ bool edge(const Cursor& c) const {
    return row0(c.rg + 1) > a.rows || c.h + (1 << log_h) > n;
  }
  __device__ __forceinline__ void load_pos(int rg, int32_t (&p)[KP]) const {
    const int64_t r = row0(rg) - past_rows(rg);
#pragma unroll
    for (int k = 0; k < KP; ++k) p[k] = *(const MPIPE_GLOBAL int32_t*)(pos[k] + r);
  }
  // cos and sin of the step's rows: each row's lanes share its rot / 2 pairs and meet in LDS
  __device__ __forceinline__ void angles(const int32_t (&p)[KP], float (&c)[V], float (&s)[V]) const {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < KP; ++k) {
      const int j = at.sub + (k << (log_c + log_h));
      if (j < a.half) {
        float x, y;
        turn_cos_sin(turns[j], p[k], x, y);
        cs[at.rs * a.half + j] = x;
        sn[at.rs * a.half + j] = a.inverse ? -y : y;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    const int j0 = at.rs * a.half + (l.turns ? at.c * V : 0);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      c[i] = cs[j0 + i];
      s[i] = sn[j0 + i];
    }
  }
};

// the tables to LDS, where a step's branch reads them without touching the loads in flight
__device__ __forceinline__ void copy_tables(const QkArgs& a, uint64_t* turns) {
  for (int i = threadIdx.x; i < a.half; i += 256) turns[i] = a.table.turn[i];
  __syncthreads();
}

// KP: position loads of a step (2 or 8); PAST: outputs that no cache would hold for a reader
template <class T, int V, bool ADJ, bool NORM, int KP, bool PAST>
__global__ __launch_bounds__(256, KP == 2 ? 4 : 2) void qk_fwd_kernel(QkArgs a) {
  constexpr int kRing = 3;
  __shared__ float trig[4][2 * kTrig];
  __shared__ uint64_t turns[kMaxPairs];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int z = (int)blockIdx.x >= a.side[0].blocks;
  const SideArgs& sd = a.side[z];
  const int block = blockIdx.x - (z ? a.side[0].blocks : 0);
  const Wave<T, V, ADJ, KP> w(a, sd, block * 4 + wave, trig[wave], turns, a.table.axis);
  const Walk<T> x(sd.x, sd.x_row, sd.x_head, w.at, w.head0, w.l.col),
      y(sd.y, sd.y_row, sd.y_head, w.at, w.head0, w.l.col);
  float g[2 * V];
  if (NORM) {
    const T* gain = reinterpret_cast<const T*>(sd.gain);
    const T* const p[2] = {gain + w.l.col[0], gain + w.l.col[1]};
    Words<T, V> r[2];
    load_head<T, V>(p, r);
    widen<T, V>(r, g);
  }
  Words<T, V> r[kRing][2];
  int32_t pos[kRing][KP];
  Cursor ahead = {w.rg0, 0}, now = ahead;
  auto load = [&](Words<T, V> (&r)[2], int32_t (&p)[KP]) {
    const T* at[2];
    x.at(w.row0(ahead.rg), ahead.h, w.past_rows(ahead.rg), w.past_heads(ahead.h), w.edge(ahead), at);
    load_head<T, V>(at, r);
    w.load_pos(ahead.rg, p);
    Cursor c = ahead;
    c.next(1 << w.log_h, w.n, w.rg_step);
    if (c.rg < w.groups) ahead = c;   // at the end: once more the last
  };
#pragma unroll
  for (int i = 0; i < kRing; ++i) load(r[i], pos[i]);
  copy_tables(a, turns);
  if (w.idle) return;
  float c[V], s[V];
  for (;;) {
#pragma unroll
    for (int i = 0; i < kRing; ++i) {
      if (now.h == 0) w.angles(pos[i], c, s);
      float v[2 * V];
      widen<T, V>(r[i], v);
      if (NORM) {
        float ss = 0.f, st = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ss = fmaf(v[e], v[e], ss);
          st = fmaf(v[V + e], v[V + e], st);
        }
        ss = w.at.extra ? 0.f : ss + (w.l.two ? st : 0.f);
        const float k = inv_rms(head_sum(ss, w.log_c), a.inv_d, a.eps);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) v[e] = v[e] * k * g[e];
      }
      turn<V, ADJ>(w.l, c, s, v);
      const T* at[2];
      y.at(w.row0(now.rg), now.h, w.past_rows(now.rg), w.past_heads(now.h), w.edge(now), at);
      store_head<T, V, PAST>(at, v);
      load(r[i], pos[i]);
      now.next(1 << w.log_h, w.n, w.rg_step);
      if (now.rg >= w.groups) return;
    }
  }
}

template <class T, int V, bool ADJ, int KP, bool PAST>
__global__ __launch_bounds__(256, KP == 2 ? 3 : 2) void qk_bwd_kernel(QkArgs a) {
  constexpr int kRing = 2;
  __shared__ float trig[4][2 * kTrig];
  __shared__ uint64_t turns[kMaxPairs];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int z = (int)blockIdx.x >= a.side[0].blocks;
  const SideArgs& sd = a.side[z];
  const int block = blockIdx.x - (z ? a.side[0].blocks : 0);
  const Wave<T, V, ADJ, KP> w(a, sd, block * 4 + wave, trig[wave], turns, a.table.axis);
  float dg[2 * V];
#pragma unroll
  for (int e = 0; e < 2 * V; ++e) dg[e] = 0.f;
  {
    const Walk<T> x(sd.x, sd.x_row, sd.x_head, w.at, w.head0, w.l.col),
        dy(sd.dy, sd.dy_row, sd.dy_head, w.at, w.head0, w.l.col),
        y(sd.y, sd.y_row, sd.y_head, w.at, w.head0, w.l.col);
    float g[2 * V];
    {
      const T* gain = reinterpret_cast<const T*>(sd.gain);
      const T* const p[2] = {gain + w.l.col[0], gain + w.l.col[1]};
      Words<T, V> r[2];
      load_head<T, V>(p, r);
      widen<T, V>(r, g);
    }
    Words<T, V> rx[kRing][2], rd[kRing][2];
    int32_t pos[kRing][KP];
    Cursor ahead = {w.rg0, 0}, now = ahead;
    auto load = [&](Words<T, V> (&rx)[2], Words<T, V> (&rd)[2], int32_t (&p)[KP]) {
      const T* at[2];
      const bool edge = w.edge(ahead);
      const int64_t row0 = w.row0(ahead.rg);
      const int drs = w.past_rows(ahead.rg), dhs = w.past_heads(ahead.h);
      x.at(row0, ahead.h, drs, dhs, edge, at);
      load_head<T, V>(at, rx);
      dy.at(row0, ahead.h, drs, dhs, edge, at);
      load_head<T, V>(at, rd);
      w.load_pos(ahead.rg, p);
      Cursor c = ahead;
      c.next(1 << w.log_h, w.n, w.rg_step);
      if (c.rg < w.groups) ahead = c;
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i) load(rx[i], rd[i], pos[i]);
    copy_tables(a, turns);
    float c[V], s[V];
    for (bool more = !w.idle; more;) {
#pragma unroll
      for (int i = 0; i < kRing; ++i) {
        if (!more) break;
        if (now.h == 0) w.angles(pos[i], c, s);
        float v[2 * V], u[2 * V];
        widen<T, V>(rx[i], v);
        widen<T, V>(rd[i], u);
        turn<V, ADJ>(w.l, c, s, u);
        float ss = 0.f, st = 0.f, gs = 0.f, gt = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          ss = fmaf(v[e], v[e], ss);
          st = fmaf(v[V + e], v[V + e], st);
          gs = fmaf(u[e] * g[e], v[e], gs);
          gt = fmaf(u[V + e] * g[V + e], v[V + e], gt);
        }
        ss = w.at.extra ? 0.f : ss + (w.l.two ? st : 0.f);
        gs = w.at.extra ? 0.f : gs + (w.l.two ? gt : 0.f);
        const float k = inv_rms(head_sum(ss, w.log_c), a.inv_d, a.eps);
        const float m = k * k * head_sum(gs, w.log_c) * a.inv_d;
        const int drs = w.past_rows(now.rg), dhs = w.past_heads(now.h);
        if (drs + dhs == 0) {   // repeats add nothing (nor 0 times an infinity)
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) dg[e] = fmaf(u[e], v[e] * k, dg[e]);
        }
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) u[e] = k * fmaf(u[e], g[e], -v[e] * m);
        const T* at[2];
        y.at(w.row0(now.rg), now.h, drs, dhs, w.edge(now), at);
        store_head<T, V, PAST>(at, u);
        load(rx[i], rd[i], pos[i]);
        now.next(1 << w.log_h, w.n, w.rg_step);
        more = now.rg < w.groups;
      }
    }
  }
  if (!sd.part) return;
  // the lanes of one column: over the wave, then over the block's waves through LDS
  __syncthreads();
  float* cols = &trig[0][0];
#pragma unroll
  for (int e = 0; e < 2 * V; ++e) {
    for (int o = 1 << w.log_c; o < 64; o <<= 1) dg[e] += __shfl_xor(dg[e], o);
    if (lane < a.lanes && (e < V || w.l.two)) cols[wave * kMaxHeadDim + w.l.col[e / V] + e % V] = dg[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.d; i += 256)
    sd.part[(int64_t)block * a.d + i] = (cols[i] + cols[kMaxHeadDim + i]) +
                                        (cols[2 * kMaxHeadDim + i] + cols[3 * kMaxHeadDim + i]);
}

constexpr int kMaxBlocks = 4096, kMaxBwdBlocks = 1536;

// grad[z][c] (+)= sum of part[z][b][c] over the blocks, in order
struct GainArgs {
  const float* part[2];
  float* grad[2];
  int blocks[2];
  int d, accumulate;
};
// 8 columns x 128 lanes of blocks; blocks of a lane in order, then the lanes
__global__ __launch_bounds__(1024) void gain_reduce_kernel(GainArgs a) {
  __shared__ float lds[128][9];
  const int z = blockIdx.y, cl = threadIdx.x & 7, bl = threadIdx.x >> 3, c = blockIdx.x * 8 + cl;
  if (!a.grad[z]) return;
  float s = 0.f;
  constexpr int kEach = kMaxBwdBlocks / 128;   // all loads at once, those past the end once more
  const int blocks = a.blocks[z];
  if (blocks > 0) {
    float v[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      v[u] = a.part[z][(int64_t)min(bl + u * 128, blocks - 1) * a.d + c];
#pragma unroll
    for (int u = 0; u < kEach; ++u) s += bl + u * 128 < blocks ? v[u] : 0.f;
  }
  lds[bl][cl] = s;
  __syncthreads();
  for (int o = 64; o > 0; o >>= 1) {
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

// Heads a wave holds at once: the most (a row's angles are worked out once per wave) that
// leave at most an eighth of the slots over a row's heads idle, or the fewest idle.  Rows of
// less than two items a wave are spread over waves by their heads too (2743 rows, 39 + 2 heads
// of 256, norm backward: 3.3 -> 3.6 TB/s; four or eight items a wave gain nothing in the mean).
void divide(SideArgs& s, int64_t rows, int log_c, int min_log_h, int max_blocks) {
  if (s.heads == 0 || rows == 0) return;   // no blocks
  int best = min_log_h, idle = 1 << 30;
  for (int h = min_log_h; h <= 6 - log_c; ++h) {
    const int n = (s.heads + (1 << h) - 1) >> h, waste = (n << h) - s.heads;
    if (waste <= idle || waste * 8 <= n << h) {
      idle = waste;
      best = h;
    }
  }
  const int rs = 6 - log_c - best, iters = (s.heads + (1 << best) - 1) >> best;
  s.log_h = best;
  s.groups = (int)((rows + (1 << rs) - 1) >> rs);
  s.head_groups = std::max(1, std::min(std::min(iters, 4 * max_blocks),
                                       (8 * max_blocks + s.groups / 2) / s.groups));
  s.iters = (iters + s.head_groups - 1) / s.head_groups;
  s.head_groups = (iters + s.iters - 1) / s.iters;
  s.blocks = (int)std::min<int64_t>(((int64_t)s.groups * s.head_groups + 3) / 4, max_blocks);
}

// Slots of heads a wave must hold so that its lanes work out a row's angles two each at most.
// A side with fewer heads leaves the others idle: a launch of its own with eight angles a lane
// took 52 us against 46 (rotation of 40000 rows, 8 + 1 heads of 128), and 133 against 120 in
// the norm's backward with 16 + 2.
int min_slots_log2(const QkArgs& a) {
  int h = 0;
  while ((2 << (a.log_c + h)) < a.half) ++h;
  return h;
}
// The sides of a launch.  Blocks: `resident`, what the bf16 kernels of eight columns a vector and
// two angles a lane hold at once (four waves a SIMD forward, three backward; of the others fp32
// holds 6 and 4, eight angles a lane 2 to 4), or `many` where each of their waves would take
// `long_walk` steps and more.  Each side's share of them is its share of the steps, a row's angles
// counted as another.  Returns the position loads of a step (2 or 8).
int divide(QkArgs& a, int resident, int many, int long_walk) {
  const int min_log_h = min_slots_log2(a);
  const bool few = std::max(a.side[0].heads, a.side[1].heads) < 1 << min_log_h;
  double steps[2] = {0.0, 0.0};
  int max_blocks = resident;
  for (int pass = 0; pass < 2; ++pass) {
    for (int z = 0; z < 2; ++z) {
      const SideArgs& s = a.side[z];
      divide(a.side[z], a.rows, a.log_c, few ? 0 : min_log_h, max_blocks);
      steps[z] = (double)s.groups * s.head_groups * (s.iters + 1);
    }
    if (steps[0] + steps[1] < 4.0 * resident * long_walk) break;
    max_blocks = many;
  }
  if (a.side[0].blocks + a.side[1].blocks > max_blocks)
    for (SideArgs& s : a.side)
      if (s.blocks > 0) {
        const double share = steps[&s - a.side] / (steps[0] + steps[1]);
        s.blocks = std::max((s.head_groups + 3) / 4, std::min(s.blocks, (int)(max_blocks * share)));
      }
  return few ? 8 : 2;
}

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
  a.lanes = a.half / v + (a.d - 2 * a.half + 2 * v - 1) / (2 * v);
  a.log_c = log2_up(a.lanes);
  a.table = p.table;
  return a;
}

// Outputs of more than the 256 MB of last-level cache are stored past the caches where every
// store fills whole 128-byte lines (half a head each): 65536 rows, 28 + 4 heads of 128, rotation
// 201 -> 192 us, norm backward 321 -> 312 us.  Stores that share a line lose by it (45956 rows,
// 8 + 8 heads of 256 that turn half, rotation: 155 -> 197 us), and a smaller output is still
// cached for its reader.
bool past_caches(const QkProblem& p) {
  if (p.adjacent || p.rot_dim < p.head_dim) return false;
  const int esz = p.dtype == DT_BF16 ? 2 : 4;
  uint64_t at = (uint64_t)p.head_dim / 2 * esz;
  int64_t heads = 0;
  for (const QkSide& s : p.side)
    if (s.y.heads > 0) {
      heads += s.y.heads;
      at |= (uintptr_t)s.y.p | (uint64_t)(s.y.row * esz) | (uint64_t)(s.y.head * esz);
    }
  return at % 128 == 0 && p.rows * heads * p.head_dim * esz > int64_t(256) << 20;
}

template <class T, int V, bool ADJ, int KP, bool PAST>
void launch(const QkArgs& a, bool norm, bool bwd, hipStream_t s) {
  const dim3 grid(a.side[0].blocks + a.side[1].blocks);
  if (bwd) hipLaunchKernelGGL((qk_bwd_kernel<T, V, ADJ, KP, PAST>), grid, dim3(256), 0, s, a);
  else if (norm) hipLaunchKernelGGL((qk_fwd_kernel<T, V, ADJ, true, KP, PAST>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((qk_fwd_kernel<T, V, ADJ, false, KP, PAST>), grid, dim3(256), 0, s, a);
}
template <class T, int V>
void launch(const QkArgs& a, const QkProblem& p, bool bwd, int kp, hipStream_t s) {
  if (p.adjacent) {
    if (kp == 8) launch<T, V, true, 8, false>(a, p.norm, bwd, s);
    else launch<T, V, true, 2, false>(a, p.norm, bwd, s);
    return;
  }
  if constexpr (V * sizeof(T) == 16)   // (whole lines have 16-byte vectors)
    if (kp == 2 && past_caches(p)) return launch<T, V, false, 2, true>(a, p.norm, bwd, s);
  if (kp == 8) launch<T, V, false, 8, false>(a, p.norm, bwd, s);
  else launch<T, V, false, 2, false>(a, p.norm, bwd, s);
}

// `gain`: a backward, whose blocks leave their sums in scratch.
hipError_t run(const QkProblem& p, GainArgs* gain, float* scratch, hipStream_t s) {
  const int v = vector_of(p.dtype, p.rot_dim / 2, p.head_dim);
  QkArgs a = device_args(p, v);
  const int kp = gain ? divide(a, 768, kMaxBwdBlocks, 48) : divide(a, 1024, kMaxBlocks, 16);
  if (a.side[0].blocks + a.side[1].blocks == 0) return hipSuccess;
  if (gain)
    for (int z = 0; z < 2; ++z) {
      a.side[z].part = gain->grad[z] ? scratch : nullptr;
      gain->part[z] = scratch;
      gain->blocks[z] = a.side[z].blocks;
      scratch += (int64_t)a.side[z].blocks * p.head_dim;
    }
  if (p.dtype == DT_F32) launch<float, 4>(a, p, gain, kp, s);
  else if (v == 8) launch<bf16, 8>(a, p, gain, kp, s);
  else launch<bf16, 4>(a, p, gain, kp, s);
  return hipGetLastError();
}

}  // namespace

hipError_t qk_rope_fwd(const QkProblem& p, hipStream_t s) { return run(p, nullptr, nullptr, s); }

// at most kMaxBwdBlocks blocks a side, and no more than it has heads
size_t qk_norm_rope_bwd_scratch(int64_t rows, int heads_q, int heads_k, int head_dim) {
  const auto blocks = [&](int heads) { return (size_t)std::min<int64_t>(rows * heads, kMaxBwdBlocks); };
  return (blocks(heads_q) + blocks(heads_k)) * head_dim * 4 + 256;
}

hipError_t qk_norm_rope_bwd(const QkProblem& p, bool accumulate, float* scratch, hipStream_t s) {
  GainArgs r = {};
  for (int z = 0; z < 2; ++z) r.grad[z] = p.side[z].grad;
  const hipError_t e = run(p, &r, scratch, s);
  if (e != hipSuccess || (!r.grad[0] && !r.grad[1])) return e;
  r.d = p.head_dim;
  r.accumulate = accumulate;
  hipLaunchKernelGGL(gain_reduce_kernel, dim3(p.head_dim / 8, 2), dim3(1024), 0, s, r);
  return hipGetLastError();
}

}  // namespace mpipe
