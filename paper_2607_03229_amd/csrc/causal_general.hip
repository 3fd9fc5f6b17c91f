// Causal attention with grouped heads for every type, alignment and head width: fp32 MFMA.
// fp32 problems run here, and bf16 ones whose heads are wider than 128 or not 16-byte aligned.
//
// Per (16 rows of a work item, head) one block of four waves; the waves take the other side's
// 16-row tiles in turn and their partial results are added in wave order through LDS.  All
// products run on v_mfma_f32_16x16x4_f32, whose operands come straight from memory: in an operand
// lane (g, r) = (l / 16, l % 16) holds row (or column) r at reduction index g.
//   row form         lane reads four values of row r; piece f gives the reduction indices
//                    d = 16f + 4g + s of four successive MFMAs s
//   transposed form  lane reads X[4g + s][16 dt + r], one value per MFMA s: the reduction runs
//                    over the tile's rows as a score accumulator (row 4g + s in element s)
//                    already holds its other operand
// so scores never leave their registers.  Values are widened to fp32 as they are read: bf16
// products are then exact and weights are not rounded.
//
// Bound by the CU's path of loads: each wave takes the other side's rows from the caches itself, in both
// forms, eight operations a byte.  Counted on MI355X, eight fp32 sequences of 2048, 8 heads of 64: that
// path is busy for 93 % of the time in all three kernels, the matrix unit for 52, 51 and 44 % (forward
// 0.43 ms, 81 of the 152 TFLOP/s that a large product reaches; backward 1.62 ms, 53 TFLOP/s of five
// products, seven are made).  16/4 heads of 128: 96, 72 and 54 %, and 49, 38 and 37 %; the last two have
// registers for one wave a SIMD.  Below some 1000 rows it is one tile's chain of loads and products: five
// of up to 333, 6 heads of 64: 12.7, 17.0 and 20.8 us.  bf16 at width 256, where the backward spills
// registers too: four of 2048, 8/2 heads of 256, forward 1.63 ms, backward 5.7 (heads of 128, on bf16
// products, 0.06 and 0.19).
//
// A key that a query does not see has weight 0, but 0 times an infinity or a NaN of its value
// would still reach the sum.  Only tiles that the diagonal cuts hold such pairs, and only an
// output that is not finite can be touched: a wave that finds one goes over its tiles again and
// adds the pairs of cut tiles one by one.
#include "attn_kernels.h"
#include "common.h"

namespace mpipe {
namespace {

typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
typedef __attribute__((ext_vector_type(4), aligned(2))) bf16 bf16x4_any;

__device__ __forceinline__ f32x4 load4(const float* p) {
  const f32x4_any x = *reinterpret_cast<const f32x4_any*>(p);
  return f32x4{x[0], x[1], x[2], x[3]};
}
__device__ __forceinline__ f32x4 load4(const bf16* p) {
  const bf16x4_any x = *reinterpret_cast<const bf16x4_any*>(p);
  return f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
}
__device__ __forceinline__ void store4(float* p, const f32x4& x) {
  *reinterpret_cast<f32x4_any*>(p) = f32x4_any{x[0], x[1], x[2], x[3]};
}
__device__ __forceinline__ void store4(bf16* p, const f32x4& x) {
  *reinterpret_cast<bf16x4_any*>(p) = bf16x4_any{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
}

// One head's rows in memory, d columns of which are real.
template <class T> struct Rows {
  const T* p;
  int64_t ld;
  int d, last;   // last row
};
template <class T>
__device__ __forceinline__ Rows<T> rows_of(const AttnView& v, int head, int row0, int n, int d) {
  return {reinterpret_cast<const T*>(v.p) + v.head * head + v.row * row0, v.row, d, n - 1};
}
template <int DP> struct RowForm {
  f32x4 v[DP / 16];
};
// (EXACT: d is DP.  All loads are made, of the row's own values where there is no column: a branch
// around each took as long as the products.)
template <int DP, bool EXACT, class T>
__device__ __forceinline__ void load_rows(RowForm<DP>& R, const Rows<T>& X, int row, int g) {
  const T* p = X.p + (int64_t)min(row, X.last) * X.ld;
#pragma unroll
  for (int f = 0; f < DP / 16; ++f) {
    const bool in = EXACT || 16 * f + 4 * g < X.d;
    const f32x4 x = load4(p + (in ? 16 * f + 4 * g : 4 * (g & 1)));   // (d is at least 8)
#pragma unroll
    for (int e = 0; e < 4; ++e) R.v[f][e] = in ? x[e] : 0.f;
  }
}
// Rows past the last are the last's, and columns past d the row's first ones: no pair of the
// former counts, and nobody stores the sums of the latter.
template <int DP> struct ColForm {
  float v[4][DP / 16];
};
template <int DP, bool EXACT, class T>
__device__ __forceinline__ void load_cols(ColForm<DP>& C, const Rows<T>& X, int r0, int g, int r) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const T* p = X.p + (int64_t)min(r0 + 4 * g + s, X.last) * X.ld;
#pragma unroll
    for (int dt = 0; dt < DP / 16; ++dt)
      C.v[s][dt] = (float)p[EXACT || 16 * dt + r < X.d ? 16 * dt + r : r & 7];
  }
}
// element s of lane (g, r): sum over d of A[row 4g + s][d] B[row r][d]
template <int DP>
__device__ __forceinline__ f32x4 dot_rows(const RowForm<DP>& A, const RowForm<DP>& B) {
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int f = 0; f < DP / 16; ++f)
#pragma unroll
    for (int s = 0; s < 4; ++s)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(A.v[f][s], B.v[f][s], acc, 0, 0, 0);
  return acc;
}
// acc[dt] (element s: component 16 dt + 4g + s of row r) += sum over rows X[row][.] b[row][r]
template <int DP>
__device__ __forceinline__ void accum_cols(f32x4 (&acc)[DP / 16], const ColForm<DP>& X,
                                           const f32x4& b) {
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int dt = 0; dt < DP / 16; ++dt)
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(X.v[s][dt], b[s], acc[dt], 0, 0, 0);
}
// The same for a cut tile, pair by pair: `seen` bit s says whether pair (4g + s, r) counts.
template <int DP, class T>
__device__ __forceinline__ void accum_pairs(f32x4 (&acc)[DP / 16], const Rows<T>& X, int r0,
                                            const f32x4& b, int seen, int g, int r) {
  for (int i = 0; i < 16; ++i) {
    const int from = (i >> 2) * 16 + r;
    float w = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float x = __shfl(b[s], from);
      w = (i & 3) == s ? x : w;
    }
    const bool in = (__shfl(seen, from) >> (i & 3)) & 1;
    const T* p = X.p + (int64_t)min(r0 + i, X.last) * X.ld + 4 * g;
#pragma unroll
    for (int dt = 0; dt < DP / 16; ++dt)
      if (16 * dt + 4 * g < X.d) {
        const f32x4 x = load4(p + 16 * dt);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[dt][e] = in ? fmaf(w, x[e], acc[dt][e]) : acc[dt][e];
      }
  }
}
template <int N> __device__ __forceinline__ bool all_finite(const f32x4 (&acc)[N]) {
  float z = 0.f;   // 0 times anything finite
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) z = fmaf(acc[i][e], 0.f, z);
  return __all(z == 0.f);
}
template <int N> __device__ __forceinline__ void clear(f32x4 (&acc)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}
// Sum of the four waves' accumulators in wave order, in wave 0; a wave at a time, so that LDS
// holds one of them.
template <int N>
__device__ __forceinline__ void add_waves(f32x4 (&acc)[N], f32x4 (*red)[64], int w, int l) {
  for (int k = 1; k < 4; ++k) {
    if (w == k) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[i][l] = acc[i];
    }
    __syncthreads();
    if (w == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] += red[i][l];
    }
    __syncthreads();
  }
}

// The block's sequence, its 16 rows and head.  The key head is the fastest index: blocks go
// round the eight XCDs, so those that read the same keys share an L2.
struct Place {
  int q_row, q_len, k_row, k_len, r0, head_k, gq;
};
__device__ __forceinline__ Place place_of(const CausalArgs& p, int per_head) {
  Place a;
  int b = blockIdx.x;
  a.head_k = b % p.heads_k;
  b /= p.heads_k;
  a.gq = b % per_head;
  b /= per_head;
  const uint32_t it = (uint32_t)p.pool.word[kAttnWords - 1 - b / p.sub];
  const int32_t* s = p.pool.word + 4 * (it & 255);
  a.q_row = s[0];
  a.q_len = s[1];
  a.k_row = s[2];
  a.k_len = s[3];
  a.r0 = 16 * ((int)(it >> 8) * p.sub + b % p.sub);
  return a;
}

// ---- forward: S^T = K Q^T (a query per column), online softmax per wave, O^T += V^T P^T -----
template <class T, int DP, bool EXACT>
__global__ __launch_bounds__(256) void fwd_kernel(CausalArgs p) {
  constexpr int ND = DP / 16;
  __shared__ f32x4 red[ND][64];
  __shared__ float2 ml[4][64];
  const Place a = place_of(p, p.group);
  if (a.r0 >= a.q_len) return;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, g = l >> 4, r = l & 15;
  const int head = a.head_k * p.group + a.gq;
  const int row = min(a.r0 + r, a.q_len - 1), shift = a.k_len - a.q_len;
  const int last_key = row + shift;                       // that the lane's query sees
  const int keys = min(a.r0 + 15, a.q_len - 1) + shift + 1;   // that any query of the block sees
  const int nt = keys > 0 ? (keys + 15) / 16 : 0;
  const Rows<T> Q = rows_of<T>(p.q, head, a.q_row, a.q_len, p.d);
  const Rows<T> K = rows_of<T>(p.k, a.head_k, a.k_row, a.k_len, p.d);
  const Rows<T> V = rows_of<T>(p.v, a.head_k, a.k_row, a.k_len, p.d);
  RowForm<DP> q, k;
  ColForm<DP> v;
  load_rows<DP, EXACT>(q, Q, a.r0 + r, g);
  float m, sum;
  f32x4 o[ND];
  auto walk = [&](bool by_pairs) {
    m = -INFINITY;
    sum = 0.f;
    clear(o);
    for (int t = w; t < nt; t += 4) {
      const int k0 = 16 * t;
      load_rows<DP, EXACT>(k, K, k0 + r, g);
      load_cols<DP, EXACT>(v, V, k0, g, r);
      f32x4 s = dot_rows<DP>(k, q);
      int seen = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = k0 + 4 * g + e <= last_key;
        seen |= in ? 1 << e : 0;
        s[e] = in ? s[e] * p.scale : -INFINITY;
      }
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      // where all scores so far are -inf there is no maximum to subtract: terms are 0
      const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn, c = expf(m - ref);
      m = mn;
      sum *= c;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = expf(s[e] - ref);
        sum += s[e];   // this lane's keys; the lane groups are added after the loop
      }
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] *= c;
      if (by_pairs && __any(seen != 15)) accum_pairs<DP>(o, V, k0, s, seen, g, r);
      else accum_cols<DP>(o, v, s);
    }
  };
  walk(false);
  if (!all_finite(o)) walk(true);
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  ml[w][l] = make_float2(m, sum);
  __syncthreads();
  float M = -INFINITY, tot = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) M = fmaxf(M, ml[i][l].x);
  const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int i = 0; i < 4; ++i) tot += ml[i][l].y * expf(ml[i][l].x - ref);
  const float mine = expf(m - ref);
  // a wave without weight for this query (no key, or scores of -inf) holds zeros
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) o[dt] = m == -INFINITY ? f32x4{0.f, 0.f, 0.f, 0.f} : o[dt] * mine;
  add_waves<ND>(o, red, w, l);
  if (w > 0 || a.r0 + r >= a.q_len) return;
  T* O = reinterpret_cast<T*>(const_cast<void*>(p.o.p)) + p.o.head * head +
         p.o.row * (int64_t)(a.q_row + row) + 4 * g;
  const float inv = last_key < 0 ? 0.f : 1.0f / tot;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
    if (16 * dt + 4 * g < p.d) store4(O + 16 * dt, o[dt] * inv);
  if (g == 0 && p.lse) p.lse[head * p.ld_lse + a.q_row + row] = M + logf(tot);
}

// Whether the backward's registers leave a SIMD one wave only, which then loads a tile while it works
// on the one before.  (Wider heads spill as it is.)
template <int DP> constexpr bool alone = DP == 128;

// ---- backward: dQ^T += K^T dS^T over the keys; delta = dO . O of the block's queries ---------
template <class T, int DP, bool EXACT>
__global__ __launch_bounds__(256) void dq_kernel(CausalArgs p) {
  constexpr int ND = DP / 16;
  __shared__ f32x4 red[ND][64];
  const Place a = place_of(p, p.group);
  if (a.r0 >= a.q_len) return;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, g = l >> 4, r = l & 15;
  const int head = a.head_k * p.group + a.gq;
  const int row = min(a.r0 + r, a.q_len - 1), shift = a.k_len - a.q_len;
  const int last_key = row + shift;
  const int keys = min(a.r0 + 15, a.q_len - 1) + shift + 1;
  const int nt = keys > 0 ? (keys + 15) / 16 : 0;
  const Rows<T> K = rows_of<T>(p.k, a.head_k, a.k_row, a.k_len, p.d);
  const Rows<T> V = rows_of<T>(p.v, a.head_k, a.k_row, a.k_len, p.d);
  RowForm<DP> q, d_o, k, v;
  ColForm<DP> kt;
  load_rows<DP, EXACT>(q, rows_of<T>(p.q, head, a.q_row, a.q_len, p.d), a.r0 + r, g);
  load_rows<DP, EXACT>(d_o, rows_of<T>(p.d_o, head, a.q_row, a.q_len, p.d), a.r0 + r, g);
  load_rows<DP, EXACT>(k, rows_of<T>(p.o, head, a.q_row, a.q_len, p.d), a.r0 + r, g);
  float del = 0.f;
#pragma unroll
  for (int f = 0; f < ND; ++f)
#pragma unroll
    for (int e = 0; e < 4; ++e) del = fmaf(k.v[f][e], d_o.v[f][e], del);
  del += __shfl_xor(del, 16);
  del += __shfl_xor(del, 32);
  const float lse = p.lse[head * p.ld_lse + a.q_row + row];
  if (w == 0 && g == 0 && a.r0 + r < a.q_len) p.delta[head * p.rows_q + a.q_row + row] = del;
  f32x4 dq[ND];
  auto walk = [&](bool by_pairs) {
    clear(dq);
    auto rows = [&](int k0) {
      load_rows<DP, EXACT>(k, K, k0 + r, g);
      load_rows<DP, EXACT>(v, V, k0 + r, g);
    };
    auto cols = [&](int k0) { load_cols<DP, EXACT>(kt, K, k0, g, r); };
    if (alone<DP> && w < nt) {
      rows(16 * w);
      cols(16 * w);
    }
    for (int t = w; t < nt; t += 4) {
      const int k0 = 16 * t;
      if constexpr (!alone<DP>) {
        rows(k0);
        cols(k0);
      }
      const f32x4 s = dot_rows<DP>(k, q), dp = dot_rows<DP>(v, d_o);
      if constexpr (alone<DP>) rows(k0 + 64);   // past the last row: that one
      f32x4 ds;
      int seen = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = k0 + 4 * g + e <= last_key;
        seen |= in ? 1 << e : 0;
        ds[e] = in ? expf(s[e] * p.scale - lse) * (dp[e] - del) : 0.f;
      }
      if (by_pairs && __any(seen != 15)) accum_pairs<DP>(dq, K, k0, ds, seen, g, r);
      else accum_cols<DP>(dq, kt, ds);
      if constexpr (alone<DP>) cols(k0 + 64);
    }
  };
  walk(false);
  if (!all_finite(dq)) walk(true);
  add_waves<ND>(dq, red, w, l);
  if (w > 0 || a.r0 + r >= a.q_len) return;
  T* out = reinterpret_cast<T*>(const_cast<void*>(p.dq.p)) + p.dq.head * head +
           p.dq.row * (int64_t)(a.q_row + row) + 4 * g;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
    if (16 * dt + 4 * g < p.d) store4(out + 16 * dt, dq[dt] * p.scale);
}

// ---- backward: per 16 keys, over the group's heads and the queries that see them -------------
// S = Q K^T (a key per column), dV^T += dO^T P, dK^T += Q^T dS.  Where there are few keys, p.parts
// blocks share 16 of them.
template <class T, int DP, bool EXACT>
__global__ __launch_bounds__(256) void dkdv_kernel(CausalArgs p) {
  constexpr int ND = DP / 16;
  __shared__ f32x4 red[ND][64];
  const Place a = place_of(p, p.parts);
  if (a.r0 >= a.k_len) return;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, g = l >> 4, r = l & 15;
  const int row = min(a.r0 + r, a.k_len - 1), shift = a.k_len - a.q_len;
  const int first_q = row - shift;                // first query that sees the lane's key
  const int t0 = max(a.r0 - shift, 0) / 16;       // first tile with one that sees any of them
  const int nt = max((a.q_len + 15) / 16 - t0, 0);
  const int c0 = (int)((int64_t)nt * p.group * a.gq / p.parts);         // the block's part of the
  const int c1 = (int)((int64_t)nt * p.group * (a.gq + 1) / p.parts);   // group's tiles
  RowForm<DP> k, v, q, d_o;
  ColForm<DP> qt, dt_;
  load_rows<DP, EXACT>(k, rows_of<T>(p.k, a.head_k, a.k_row, a.k_len, p.d), a.r0 + r, g);
  load_rows<DP, EXACT>(v, rows_of<T>(p.v, a.head_k, a.k_row, a.k_len, p.d), a.r0 + r, g);
  f32x4 dk[ND], dv[ND], lse, del;
  auto walk = [&](bool by_pairs) {
    clear(dk);
    clear(dv);
    // tile c of the group's heads, one head behind the other; past the last, that one
    struct At {
      int head, r0;
    };
    auto at_tile = [&](int c) {
      c = min(c, nt * p.group - 1);
      return At{a.head_k * p.group + c / nt, 16 * (t0 + c % nt)};
    };
    auto q_of = [&](const At& x) { return rows_of<T>(p.q, x.head, a.q_row, a.q_len, p.d); };
    auto do_of = [&](const At& x) { return rows_of<T>(p.d_o, x.head, a.q_row, a.q_len, p.d); };
    auto rows = [&](const At& x) {
      load_rows<DP, EXACT>(q, q_of(x), x.r0 + r, g);
      load_rows<DP, EXACT>(d_o, do_of(x), x.r0 + r, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t i = a.q_row + min(x.r0 + 4 * g + e, a.q_len - 1);
        lse[e] = p.lse[x.head * p.ld_lse + i];
        del[e] = p.delta[x.head * p.rows_q + i];
      }
    };
    auto cols = [&](const At& x) {
      load_cols<DP, EXACT>(qt, q_of(x), x.r0, g, r);
      load_cols<DP, EXACT>(dt_, do_of(x), x.r0, g, r);
    };
    if (alone<DP> && c0 + w < c1) {
      rows(at_tile(c0 + w));
      cols(at_tile(c0 + w));
    }
    for (int c = c0 + w; c < c1; c += 4) {
      const At x = at_tile(c);
      if constexpr (!alone<DP>) {
        rows(x);
        cols(x);
      }
      const f32x4 s = dot_rows<DP>(q, k), dp = dot_rows<DP>(d_o, v);
      f32x4 pr, ds;
      int seen = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int qr = x.r0 + 4 * g + e;
        const bool in = qr >= first_q && qr < a.q_len;
        seen |= in ? 1 << e : 0;
        const float pe = expf(s[e] * p.scale - lse[e]);
        pr[e] = in ? pe : 0.f;
        ds[e] = in ? pe * (dp[e] - del[e]) : 0.f;
      }
      if constexpr (alone<DP>) rows(at_tile(c + 4));
      if (by_pairs && __any(seen != 15)) {
        accum_pairs<DP>(dv, do_of(x), x.r0, pr, seen, g, r);
        accum_pairs<DP>(dk, q_of(x), x.r0, ds, seen, g, r);
      } else {
        accum_cols<DP>(dv, dt_, pr);
        accum_cols<DP>(dk, qt, ds);
      }
      if constexpr (alone<DP>) cols(at_tile(c + 4));
    }
  };
  walk(false);
  if (!(all_finite(dk) && all_finite(dv))) walk(true);
  add_waves<ND>(dk, red, w, l);
  add_waves<ND>(dv, red, w, l);
  if (p.parts > 1) {
    f32x4* out = reinterpret_cast<f32x4*>(p.partial) + (int64_t)blockIdx.x * (2 * ND * 64) + l;
    if (w > 0) return;
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      out[64 * i] = dk[i];
      out[64 * (ND + i)] = dv[i];
    }
    return;
  }
  if (w > 0 || a.r0 + r >= a.k_len) return;
  const int64_t at = a.k_row + row;
  T* dK = reinterpret_cast<T*>(const_cast<void*>(p.dk.p)) + p.dk.head * a.head_k + p.dk.row * at + 4 * g;
  T* dV = reinterpret_cast<T*>(const_cast<void*>(p.dv.p)) + p.dv.head * a.head_k + p.dv.row * at + 4 * g;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
    if (16 * dt + 4 * g < p.d) {
      store4(dK + 16 * dt, dk[dt] * p.scale);
      store4(dV + 16 * dt, dv[dt]);
    }
}

// The sums of 16 keys' parts, in their order.
template <class T, int DP, bool EXACT>
__global__ __launch_bounds__(256) void parts_kernel(CausalArgs p) {
  constexpr int ND = DP / 16;
  const Place a = place_of(p, 1);
  const int64_t tile = blockIdx.x / p.heads_k;
  for (int i = threadIdx.x; i < 2 * ND * 64; i += 256) {
    const int l = i & 63, g = l >> 4, r = l & 15, dt = i / 64 % ND;
    if (a.r0 + r >= a.k_len || 16 * dt + 4 * g >= p.d) continue;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int j = 0; j < p.parts; ++j)
      x += reinterpret_cast<const f32x4*>(p.partial)[((tile * p.parts + j) * p.heads_k + a.head_k) * (2 * ND * 64) + i];
    const bool of_k = i < ND * 64;
    const AttnView& out = of_k ? p.dk : p.dv;
    store4(reinterpret_cast<T*>(const_cast<void*>(out.p)) + out.head * a.head_k +
               out.row * (int64_t)(a.k_row + a.r0 + r) + 16 * dt + 4 * g,
           of_k ? x * p.scale : x);
  }
}

template <class Kernel>
hipError_t launch(Kernel kernel, const CausalArgs& a, int64_t blocks, hipStream_t s) {
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

#define MPIPE_GENERAL_WIDTH(KERNEL, T, DP) \
  (a.d == DP ? launch(KERNEL<T, DP, true>, a, blocks, s) : launch(KERNEL<T, DP, false>, a, blocks, s))
#define MPIPE_GENERAL_TYPE(KERNEL, T)                       \
  (a.d <= 32    ? MPIPE_GENERAL_WIDTH(KERNEL, T, 32)        \
   : a.d <= 64  ? MPIPE_GENERAL_WIDTH(KERNEL, T, 64)        \
   : a.d <= 96  ? MPIPE_GENERAL_WIDTH(KERNEL, T, 96)        \
   : a.d <= 128 ? MPIPE_GENERAL_WIDTH(KERNEL, T, 128)       \
                : MPIPE_GENERAL_WIDTH(KERNEL, T, 256))
#define MPIPE_GENERAL(KERNEL, BLOCKS)                       \
  const int64_t blocks = (BLOCKS);                          \
  return dtype == DT_BF16 ? MPIPE_GENERAL_TYPE(KERNEL, bf16) : MPIPE_GENERAL_TYPE(KERNEL, float);

hipError_t causal_general_fwd(int dtype, const CausalArgs& a, int items, hipStream_t s) {
  MPIPE_GENERAL(fwd_kernel, (int64_t)items * a.sub * a.heads_k * a.group)
}
hipError_t causal_general_dq(int dtype, const CausalArgs& a, int items, hipStream_t s) {
  MPIPE_GENERAL(dq_kernel, (int64_t)items * a.sub * a.heads_k * a.group)
}
static hipError_t general_dkdv(int dtype, const CausalArgs& a, int items, hipStream_t s) {
  MPIPE_GENERAL(dkdv_kernel, (int64_t)items * a.sub * a.heads_k * a.parts)
}
static hipError_t general_parts(int dtype, const CausalArgs& a, int items, hipStream_t s) {
  MPIPE_GENERAL(parts_kernel, (int64_t)items * a.sub * a.heads_k)
}
hipError_t causal_general_dkdv(int dtype, const CausalArgs& a, int items, hipStream_t s) {
  const hipError_t e = general_dkdv(dtype, a, items, s);
  return e || a.parts == 1 ? e : general_parts(dtype, a, items, s);
}
#undef MPIPE_GENERAL
#undef MPIPE_GENERAL_TYPE
#undef MPIPE_GENERAL_WIDTH

}  // namespace mpipe
