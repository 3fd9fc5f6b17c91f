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
};

struct QkArgs {
  SideArgs side[2];
  const int32_t* pos;
  int64_t ld_pos, rows;
  float eps, inv_d;
  int d, half, inverse;
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

// A head is d / 2 units: the half pairs, then two columns of the tail each.
__device__ __forceinline__ void unit_columns(int u, int half, bool adjacent, int& c0, int& c1) {
  if (u < half && !adjacent) {
    c0 = u;
    c1 = u + half;
  } else {
    c0 = 2 * u;
    c1 = 2 * u + 1;
  }
}

// One wave per (row, head), up to two units per lane.
template <class T, bool NORM>
__global__ __launch_bounds__(256) void qk_fwd_kernel(QkArgs a, int adjacent) {
  const int lane = threadIdx.x & 63, z = blockIdx.y;
  const SideArgs& sd = a.side[z];
  for (int64_t item = blockIdx.x * 4ll + (threadIdx.x >> 6); item < a.rows * sd.heads;
       item += gridDim.x * 4ll) {
    const int64_t row = item / sd.heads, head = item - row * sd.heads;
    const T* x = reinterpret_cast<const T*>(sd.x) + row * sd.x_row + head * sd.x_head;
    T* y = reinterpret_cast<T*>(sd.y) + row * sd.y_row + head * sd.y_head;
    const T* g = reinterpret_cast<const T*>(sd.gain);
    float v[2][2], ss = 0.f;
    for (int k = 0; k < 2; ++k) {
      const int u = lane + 64 * k;
      if (2 * u >= a.d) continue;
      int c0, c1;
      unit_columns(u, a.half, adjacent, c0, c1);
      v[k][0] = (float)x[c0];
      v[k][1] = (float)x[c1];
      ss = fmaf(v[k][0], v[k][0], fmaf(v[k][1], v[k][1], ss));
    }
    float r = 1.f;
    if (NORM) r = 1.f / sqrtf(fmaf(warp_sum(ss), a.inv_d, a.eps));
    for (int k = 0; k < 2; ++k) {
      const int u = lane + 64 * k;
      if (2 * u >= a.d) continue;
      int c0, c1;
      unit_columns(u, a.half, adjacent, c0, c1);
      float p = v[k][0], q = v[k][1];
      if (NORM) {
        p = p * r * (float)g[c0];
        q = q * r * (float)g[c1];
      }
      if (u < a.half) {
        float c, s;
        turn_cos_sin(a.table.turn[u], a.pos[a.table.axis[u] * a.ld_pos + row], c, s);
        if (a.inverse) s = -s;
        const float p0 = p, ps = p * s, qs = q * s;
        p = fmaf(p0, c, -qs);
        q = fmaf(q, c, ps);
      }
      y[c0] = (T)p;
      y[c1] = (T)q;
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void qk_bwd_kernel(QkArgs a, int adjacent) {
  __shared__ float part[4][kMaxHeadDim];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = blockIdx.y;
  const SideArgs& sd = a.side[z];
  if ((int)blockIdx.x >= sd.blocks) return;
  const T* g = reinterpret_cast<const T*>(sd.gain);
  float dg[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
  for (int64_t item = blockIdx.x * 4ll + wave; item < a.rows * sd.heads; item += sd.blocks * 4ll) {
    const int64_t row = item / sd.heads, head = item - row * sd.heads;
    const T* x = reinterpret_cast<const T*>(sd.x) + row * sd.x_row + head * sd.x_head;
    const T* dy = reinterpret_cast<const T*>(sd.dy) + row * sd.dy_row + head * sd.dy_head;
    T* y = reinterpret_cast<T*>(sd.y) + row * sd.y_row + head * sd.y_head;
    float v[2][2], w[2][2], ss = 0.f, sw = 0.f;
    for (int k = 0; k < 2; ++k) {
      const int u = lane + 64 * k;
      if (2 * u >= a.d) continue;
      int c0, c1;
      unit_columns(u, a.half, adjacent, c0, c1);
      v[k][0] = (float)x[c0];
      v[k][1] = (float)x[c1];
      float p = (float)dy[c0], q = (float)dy[c1];
      if (u < a.half) {
        float c, s;
        turn_cos_sin(a.table.turn[u], a.pos[a.table.axis[u] * a.ld_pos + row], c, s);
        const float p0 = p, ps = p * s, qs = q * s;
        p = fmaf(p0, c, qs);
        q = fmaf(q, c, -ps);
      }
      w[k][0] = p;
      w[k][1] = q;
      ss = fmaf(v[k][0], v[k][0], fmaf(v[k][1], v[k][1], ss));
      sw = fmaf(v[k][0] * p, (float)g[c0], fmaf(v[k][1] * q, (float)g[c1], sw));
    }
    const float r = 1.f / sqrtf(fmaf(warp_sum(ss), a.inv_d, a.eps));
    const float m = r * r * warp_sum(sw) * a.inv_d;
    for (int k = 0; k < 2; ++k) {
      const int u = lane + 64 * k;
      if (2 * u >= a.d) continue;
      int c0, c1;
      unit_columns(u, a.half, adjacent, c0, c1);
      for (int e = 0; e < 2; ++e) {
        dg[k][e] = fmaf(w[k][e], v[k][e] * r, dg[k][e]);
        y[e ? c1 : c0] = (T)(r * fmaf(w[k][e], (float)g[e ? c1 : c0], -v[k][e] * m));
      }
    }
  }
  if (!sd.part) return;
  for (int k = 0; k < 2; ++k) {
    const int u = lane + 64 * k;
    if (2 * u >= a.d) continue;
    int c0, c1;
    unit_columns(u, a.half, adjacent, c0, c1);
    part[wave][c0] = dg[k][0];
    part[wave][c1] = dg[k][1];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.d; c += 256)
    sd.part[(int64_t)blockIdx.x * a.d + c] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
}

// grad[z][c] (+)= sum of part[z][b][c] over the blocks, in order
struct GainArgs {
  const float* part[2];
  float* grad[2];
  int blocks[2];
  int d, accumulate;
};
__global__ __launch_bounds__(64) void gain_reduce_kernel(GainArgs a) {
  const int c = blockIdx.x * 64 + threadIdx.x, z = blockIdx.y;
  if (c >= a.d || !a.grad[z]) return;
  float s = 0.f;
  for (int b = 0; b < a.blocks[z]; ++b) s += a.part[z][(int64_t)b * a.d + c];
  a.grad[z][c] = a.accumulate ? a.grad[z][c] + s : s;
}

int bwd_blocks(int64_t rows, int heads) {
  return (int)std::min<int64_t>((rows * heads + 3) / 4, 1024);
}

QkArgs device_args(const QkProblem& p) {
  QkArgs a;
  for (int z = 0; z < 2; ++z) {
    const QkSide& s = p.side[z];
    a.side[z] = {(const char*)s.x.p, (const char*)s.dy.p, (char*)s.y.p, s.x.row, s.x.head,
                 s.dy.row, s.dy.head, s.y.row, s.y.head, s.gain, nullptr, s.x.heads, 0};
  }
  a.pos = p.pos;
  a.ld_pos = p.ld_pos;
  a.rows = p.rows;
  a.eps = p.eps;
  a.inv_d = 1.f / (float)p.head_dim;
  a.d = p.head_dim;
  a.half = p.rot_dim / 2;
  a.inverse = p.inverse;
  a.table = p.table;
  return a;
}

}  // namespace

hipError_t qk_rope_fwd(const QkProblem& p, hipStream_t s) {
  const int most = std::max(p.side[0].x.heads, p.side[1].x.heads);
  if (p.rows == 0 || most == 0) return hipSuccess;
  const QkArgs a = device_args(p);
  const dim3 grid((unsigned)std::min<int64_t>((p.rows * most + 3) / 4, 1 << 20), 2);
#define MPIPE_QK(T, N) hipLaunchKernelGGL((qk_fwd_kernel<T, N>), grid, dim3(256), 0, s, a, p.adjacent)
  if (p.dtype == DT_BF16) {
    if (p.norm) MPIPE_QK(bf16, true); else MPIPE_QK(bf16, false);
  } else {
    if (p.norm) MPIPE_QK(float, true); else MPIPE_QK(float, false);
  }
#undef MPIPE_QK
  return hipGetLastError();
}

size_t qk_norm_rope_bwd_scratch(int64_t rows, int heads_q, int heads_k, int head_dim) {
  return ((size_t)bwd_blocks(rows, heads_q) + bwd_blocks(rows, heads_k)) * head_dim * 4 + 256;
}

hipError_t qk_norm_rope_bwd(const QkProblem& p, bool accumulate, float* scratch, hipStream_t s) {
  QkArgs a = device_args(p);
  GainArgs r;
  int blocks = 0;
  bool any = false;
  for (int z = 0; z < 2; ++z) {
    a.side[z].blocks = bwd_blocks(p.rows, p.side[z].x.heads);
    a.side[z].part = p.side[z].grad ? scratch : nullptr;
    r.part[z] = scratch;
    r.grad[z] = p.side[z].grad;
    r.blocks[z] = a.side[z].blocks;
    scratch += (int64_t)a.side[z].blocks * p.head_dim;
    blocks = std::max(blocks, a.side[z].blocks);
    any |= p.side[z].grad != nullptr;
  }
  if (blocks > 0) {
    const dim3 grid(blocks, 2);
    if (p.dtype == DT_BF16)
      hipLaunchKernelGGL(qk_bwd_kernel<bf16>, grid, dim3(256), 0, s, a, p.adjacent);
    else
      hipLaunchKernelGGL(qk_bwd_kernel<float>, grid, dim3(256), 0, s, a, p.adjacent);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!any) return hipSuccess;
  r.d = p.head_dim;
  r.accumulate = accumulate;
  hipLaunchKernelGGL(gain_reduce_kernel, dim3((p.head_dim + 63) / 64, 2), dim3(64), 0, s, r);
  return hipGetLastError();
}

}  // namespace mpipe
