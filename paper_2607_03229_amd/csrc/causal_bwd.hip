// Causal attention backward, bf16: dQ over query tiles, then dK and dV over key tiles.  Both
// recompute the weights from q, k and lse; no atomics, every sum in a fixed order.
#include <type_traits>

#include "causal_bf16.h"

namespace mpipe {
namespace {

constexpr int NWV = 8;
constexpr int STAGES = 3;

// ---- dQ -----------------------------------------------------------------------------------
// A wave has 32 queries, one per column: S^T = K Q^T and dP^T = V dO^T over 32 keys, dS^T from
// both, dQ^T += K^T dS^T.  Half of the waves run their products while the others form dS.
// Also writes what the other kernel needs of every query: -lse * log2(e), and -dO . O.
template <int DP>
__global__ __launch_bounds__(64 * NWV, 2) void causal_dq_kernel(CausalArgs p) {
  using T = Tile<DP>;
  constexpr int SL = T::SLOTS, DT = T::DT;
  __shared__ uint4 ks[STAGES][SL], vs[STAGES][SL];
  const AttnPlace a = attn_place(p, p.group, kBackwardQRows);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int c = l & 31, h = l >> 5;
  const bool late = w >= NWV / 2;
  const int head = a.head_k * p.group + a.gq, shift = a.k_len - a.q_len;
  const int q0 = a.r0 + 32 * w, row = min(q0 + c, a.q_len - 1);
  const int last_key = row + shift;
  const int wave_keys = q0 < a.q_len ? min(q0 + 31, a.q_len - 1) + shift + 1 : 0;
  const int first_cut = (q0 + shift + 1) & ~31;
  const int keys = min(a.r0 + kBackwardQRows - 1, a.q_len - 1) + shift + 1;
  const int nt = keys > 0 ? (keys + 63) / 64 : 0;
  const bf16* K = head_of(p.k, a.head_k, a.k_row);
  const bf16* V = head_of(p.v, a.head_k, a.k_row);
  const float sl2 = p.scale * kLog2e;

  RowOp<DP> q, d_o;
  load_row<DP>(q, head_of(p.q, head, a.q_row + row), p.d, h);
  load_row<DP>(d_o, head_of(p.d_o, head, a.q_row + row), p.d, h);
  float nd = 0.f;
  {
    RowOp<DP> o;
    load_row<DP>(o, head_of(p.o, head, a.q_row + row), p.d, h);
#pragma unroll
    for (int f = 0; f < T::KF; ++f)
#pragma unroll
      for (int e = 0; e < 8; ++e) nd = fmaf((float)o.f[f][e], -(float)d_o.f[f][e], nd);
    nd += __shfl_xor(nd, 32);
  }
  const float nl2 = -p.lse[head * p.ld_lse + a.q_row + row] * kLog2e;
  if (h == 0 && q0 + c < a.q_len) {
    float* out = p.delta + (int64_t)head * p.rows_q + a.q_row + row;
    out[0] = nl2;
    out[(int64_t)p.heads_k * p.group * p.rows_q] = nd;
  }
  PairCopy<DP, NWV> copy;
  copy.init(w, l, p.k.row, p.v.row);
  RowReads<DP> rread;
  rread.init(c, h);
  ColReads<DP> cread;
  cread.init(l);
  const uint32_t ks0 = lds_at(ks), vs0 = lds_at(vs);
  auto issue = [&](int t) __attribute__((always_inline)) {
    if (t >= nt) return;
    const uint32_t stage = stage_of<STAGES>(t) * (SL * 16);
#pragma unroll
    for (int i = 0; i < PairCopy<DP, NWV>::N; ++i) {
      const bool of_k = copy.of_x(i, w);
      copy.copy(i, w, l, (of_k ? ks0 : vs0) + stage, (of_k ? K : V) + 64 * t * (of_k ? p.k.row : p.v.row),
                a.k_len - 64 * t, p.d);
    }
  };

  f32x16 dq[DT];
  auto walk = [&](auto by_pairs) __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dq[dt] = zero16();
    f32x16 s, dp;
    bf16x8 ds[2];
    // step u: keys 32u .. 32u + 31
    auto scores = [&](int u) __attribute__((always_inline)) {
      if (32 * u >= wave_keys) return;
      const uint32_t stage = stage_of<STAGES>(u >> 1) * (SL * 16) + 32 * (u & 1) * T::NC * 16;
      s = dp = zero16();
#pragma unroll
      for (int f = 0; f < T::KF; ++f) {
        s = mfma(rread.get(rread.base(ks0 + stage, f), 0), q.f[f], s);
        dp = mfma(rread.get(rread.base(vs0 + stage, f), 0), d_o.f[f], dp);
      }
    };
    auto slopes = [&](int u) __attribute__((always_inline)) {
      if (32 * u >= wave_keys) return;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = exp2_fast(fmaf(s[i], sl2, nl2)) * (dp[i] + nd);
      if (32 * u >= first_cut) {
        const int lim = last_key - 32 * u - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = acc_row(i, 0) <= lim ? s[i] : 0.f;
      }
      ds[0] = pack8(s, 0);
      ds[1] = pack8(s, 1);
    };
    auto sums = [&](int u) __attribute__((always_inline)) {
      if (32 * u >= wave_keys) return;
      const uint32_t stage = stage_of<STAGES>(u >> 1);
      if (by_pairs.value && 32 * u >= first_cut) {
        add_pairs<DP, 32>(dq, ds, ks[stage] + 32 * (u & 1) * T::NC, l,
                          [&](int r) { return 32 * u + r <= last_key; });
        return;
      }
      const auto at = cread.base(ks0 + stage * (SL * 16) + 32 * (u & 1) * T::NC * 16);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dq[dt] = mfma(cread.get(at, 16 * j, dt), ds[j], dq[dt]);
    };
    // Slots as in the forward, two steps to a tile.  Tile x is read first by the early group in slot
    // 4x - 1 and last by the late one in slot 4x + 4; it is sent for in slots 4x - 4 and 4x - 3, and
    // waited for by the end of slot 4x - 2.
    issue(0);
    wait_copies<0>();
    lds_barrier();
    scores(0);
    if (late) lds_barrier();
    for (int t = 0; t < nt; ++t)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int u = 2 * t + b;
        if (b == 0) issue(t + 1);
        slopes(u);
        if (b == 1 && !late) wait_copies<0>();
        lds_barrier();
        __builtin_amdgcn_s_setprio(1);
        if (u + 1 < 2 * nt) scores(u + 1);
        sums(u);
        __builtin_amdgcn_s_setprio(0);
        if (b == 0 && late) wait_copies<0>();
        lds_barrier();
      }
    if (!late) lds_barrier();
  };
  walk(std::false_type());
  // a pair that does not count must not reach the sum: see add_pairs
  if (__syncthreads_or(!finite16(dq))) walk(std::true_type());
  if (q0 + c >= a.q_len) return;
  store_row<DP>(out_of(p.dq, head, a.q_row + row), dq, p.scale, p.d, h);
}

// ---- dK, dV -------------------------------------------------------------------------------
// Two waves have the same 32 keys, one per column, and walk over the queries that see them, 64
// at a time, of every head of the group.  The first forms S = Q K^T, the weights P and dV^T +=
// dO^T P; the second, a slot behind, dP = dO V^T, dS from the P that the first left in LDS, and
// dK^T += Q^T dS.  Neither holds more than one accumulator of head_dim columns, one operand and
// one tile of scores, so two waves fit a SIMD; they run on the same one (w and w + 4), and one's
// products meet the other's exponentials.
template <int DP>
__global__ __launch_bounds__(64 * NWV, 2) void causal_dkdv_kernel(CausalArgs p) {
  using T = Tile<DP>;
  constexpr int SL = T::SLOTS, DT = T::DT;
  __shared__ uint4 qs[STAGES][SL], ds_[STAGES][SL];
  __shared__ uint4 weights[NWV / 2][4][64];      // P of one tile, bf16, as the lanes hold it
  __shared__ __attribute__((aligned(16))) float nl2s[STAGES][64], nds[STAGES][64];
  const AttnPlace a = attn_place(p, 1, kBackwardKRows);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int c = l & 31, h = l >> 5, pair = w & 3;
  const bool second = w >= NWV / 2;
  const int shift = a.k_len - a.q_len;
  const int k0 = a.r0 + 32 * pair, row = min(k0 + c, a.k_len - 1);
  const int first_q = max(row - shift, 0);            // first query that sees the lane's key
  const int t0 = max(a.r0 - shift, 0) / 64;           // first tile with a query that sees any
  const int n_tiles = max((a.q_len + 63) / 64 - t0, 0), nt = n_tiles * p.group;
  const int whole_q = max(min(k0 + 31, a.k_len - 1) - shift, 0);   // sees all of the wave's keys
  const int wave_q = k0 < a.k_len ? max(k0 - shift, 0) : INT32_MAX - 64;   // sees any
  const float sl2 = p.scale * kLog2e;
  RowOp<DP> kv;
  load_row<DP>(kv, head_of(second ? p.v : p.k, a.head_k, a.k_row + row), p.d, h);
  PairCopy<DP, NWV> copy;
  copy.init(w, l, p.q.row, p.d_o.row);
  RowReads<DP> rread;
  rread.init(c, h);
  ColReads<DP> cread;
  cread.init(l);
  // the first wave's rows are of Q and columns of dO, the second's the other way round
  const uint32_t rows0 = second ? lds_at(ds_) : lds_at(qs), cols0 = second ? lds_at(qs) : lds_at(ds_);
  auto issue = [&](int t) __attribute__((always_inline)) {
    if (t >= nt) return;
    const int head = a.head_k * p.group + t / n_tiles, r0 = 64 * (t0 + t % n_tiles);
    const uint32_t stage = stage_of<STAGES>(t);
    const bf16* Q = head_of(p.q, head, a.q_row) + r0 * p.q.row;
    const bf16* dO = head_of(p.d_o, head, a.q_row) + r0 * p.d_o.row;
    const uint32_t at = stage * (SL * 16);
#pragma unroll
    for (int i = 0; i < PairCopy<DP, NWV>::N; ++i) {
      const bool of_q = copy.of_x(i, w);
      copy.copy(i, w, l, (of_q ? lds_at(qs) : lds_at(ds_)) + at, of_q ? Q : dO, a.q_len - r0, p.d);
    }
    if (pair == 0) {
      const float* X = p.delta + (int64_t)head * p.rows_q + a.q_row + min(r0 + l, a.q_len - 1);
      if (second) X += (int64_t)p.heads_k * p.group * p.rows_q;
      copy4(lds_at(second ? nds[stage] : nl2s[stage]), X);
    }
  };

  f32x16 acc[DT];
  auto walk = [&](auto by_pairs) __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = zero16();
    f32x16 s[2];
    bf16x8 x[4];
    auto q_of = [&](int t) { return 64 * (t0 + t % n_tiles); };
    auto idle = [&](int r0) { return r0 + 63 < wave_q; };   // no query of the tile sees a key here
    auto cut = [&](int r0) { return r0 < whole_q || r0 + 64 > a.q_len; };
    auto products = [&](int t) __attribute__((always_inline)) {
      if (idle(q_of(t))) return;
      const uint32_t stage = stage_of<STAGES>(t);
      const uint32_t tile = rows0 + stage * (SL * 16);
#pragma unroll
      for (int q2 = 0; q2 < 2; ++q2) {
        if (second) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(&nds[stage][32 * q2 + 8 * i + 4 * h]);
            s[q2][4 * i] = v.x;
            s[q2][4 * i + 1] = v.y;
            s[q2][4 * i + 2] = v.z;
            s[q2][4 * i + 3] = v.w;
          }
        } else {
          s[q2] = zero16();
        }
      }
#pragma unroll
      for (int f = 0; f < T::KF; ++f) {
        const uint32_t at = rread.base(tile, f);
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) s[q2] = mfma(rread.get(at, 32 * q2), kv.f[f], s[q2]);
      }
    };
    auto form = [&](int t) __attribute__((always_inline)) {
      const int r0 = q_of(t);
      if (idle(r0)) return;
      if (!second) {
        const float* nl2 = nl2s[stage_of<STAGES>(t)];
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(&nl2[32 * q2 + 8 * i + 4 * h]);
            s[q2][4 * i] = exp2_fast(fmaf(s[q2][4 * i], sl2, v.x));
            s[q2][4 * i + 1] = exp2_fast(fmaf(s[q2][4 * i + 1], sl2, v.y));
            s[q2][4 * i + 2] = exp2_fast(fmaf(s[q2][4 * i + 2], sl2, v.z));
            s[q2][4 * i + 3] = exp2_fast(fmaf(s[q2][4 * i + 3], sl2, v.w));
          }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 v = weights[pair][j][l];
          const bf16x8 pw = *reinterpret_cast<const bf16x8*>(&v);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[j >> 1][8 * (j & 1) + e] *= (float)pw[e];
        }
      }
      // (a weight that does not count is 0; its dS only needs to be told where dP is not finite)
      if ((!second || by_pairs.value) && cut(r0)) {
        const int lo = first_q - r0 - 4 * h, hi = a.q_len - r0 - 4 * h;
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = 32 * q2 + acc_row(i, 0);
            s[q2][i] = r >= lo && r < hi ? s[q2][i] : 0.f;
          }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = pack8(s[j >> 1], j & 1);
      if (!second) {
#pragma unroll
        for (int j = 0; j < 4; ++j) weights[pair][j][l] = *reinterpret_cast<const uint4*>(&x[j]);
      }
    };
    auto sums = [&](int t) __attribute__((always_inline)) {
      const int r0 = q_of(t);
      if (idle(r0)) return;
      const uint32_t stage = stage_of<STAGES>(t);
      if (by_pairs.value && cut(r0)) {
        add_pairs<DP, 64>(acc, x, second ? qs[stage] : ds_[stage], l,
                          [&](int r) { return r0 + r >= first_q && r0 + r < a.q_len; });
        return;
      }
      const auto at = cread.base(cols0 + stage * (SL * 16));
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] = mfma(cread.get(at, 16 * j, dt), x[j], acc[dt]);
    };
    // The first waves form P of tile t in slot 2t and multiply in slot 2t + 1, the second ones a slot
    // later.  Tile x is read from slot 2x - 1 to slot 2x + 2, sent for in slot 2x - 3 and waited
    // for by the end of slot 2x - 2.
    issue(0);
    issue(1);
    wait_copies<0>();
    lds_barrier();
    if (nt > 0) products(0);
    if (second) lds_barrier();
    for (int t = 0; t < nt; ++t) {
      if (second) issue(t + 2);
      form(t);
      if (!second) wait_copies<0>();
      lds_barrier();
      if (!second) issue(t + 2);
      __builtin_amdgcn_s_setprio(1);
      if (t + 1 < nt) products(t + 1);
      sums(t);
      __builtin_amdgcn_s_setprio(0);
      if (second) wait_copies<0>();
      lds_barrier();
    }
    if (!second) lds_barrier();
  };
  walk(std::false_type());
  // a pair that does not count must not reach the sum: see add_pairs
  if (__syncthreads_or(!finite16(acc))) walk(std::true_type());
  if (k0 + c >= a.k_len) return;
  store_row<DP>(out_of(second ? p.dk : p.dv, a.head_k, a.k_row + row), acc, second ? p.scale : 1.f, p.d, h);
}

template <class Kernel>
hipError_t launch(Kernel kernel, const CausalArgs& a, int64_t blocks, hipStream_t s) {
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * NWV), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t causal_bf16_dq(const CausalArgs& a, int items, hipStream_t s) {
  const int64_t n = (int64_t)items * a.heads_k * a.group;
  return a.d <= 32   ? launch(causal_dq_kernel<32>, a, n, s)
         : a.d <= 64 ? launch(causal_dq_kernel<64>, a, n, s)
         : a.d <= 96 ? launch(causal_dq_kernel<96>, a, n, s)
                     : launch(causal_dq_kernel<128>, a, n, s);
}
hipError_t causal_bf16_dkdv(const CausalArgs& a, int items, hipStream_t s) {
  const int64_t n = (int64_t)items * a.heads_k;
  return a.d <= 32   ? launch(causal_dkdv_kernel<32>, a, n, s)
         : a.d <= 64 ? launch(causal_dkdv_kernel<64>, a, n, s)
         : a.d <= 96 ? launch(causal_dkdv_kernel<96>, a, n, s)
                     : launch(causal_dkdv_kernel<128>, a, n, s);
}

}  // namespace mpipe
