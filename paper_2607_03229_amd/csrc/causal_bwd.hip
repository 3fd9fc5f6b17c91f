// Causal attention backward, bf16: dQ over query tiles, then dK and dV over key tiles.  Both
// recompute the weights from q, k and lse; no atomics, every sum in a fixed order.
//   P = exp(scale q k - lse), D = dO . O, dS = P (dO v - D)
//   dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO, the last two over the heads of a group
// Scores, D and all sums are fp32; P and dS are rounded to bf16 (half a step of 2^-8) as operands of
// their products, and P enters dS with 24 bits.
//
// Bound by the matrix unit, at the clock that its power leaves: 6 d operations a pair in dQ and 8 d in
// dK and dV (a kernel of its own for dQ: added to by many key tiles at once it would need atomics, or
// ordered turns, which were not measured).  On MI355X, eight sequences of up to 8192, 28/4 heads of 128:
// dQ 3.51 ms, 1.16 PFLOP/s of the pairs that count; dK and dV 5.14 ms, 1.06 PFLOP/s (first kernels: 336 ms
// for both); the matrix unit busy for 62 and 58 % of the time at 1.75 of 2.4 GHz, no cycle lost to LDS
// banks.  Short sequences wait for their first tiles instead: 64 of up to 700, 16 heads of 80, 162 and
// 265 us, 18 and 19 % busy.
#include <type_traits>

#include "causal_bf16.h"

namespace mpipe {
namespace {

constexpr int STAGES = 3, KSTAGES = 4;   // of tiles of dQ, and of dK and dV

// ---- dQ -----------------------------------------------------------------------------------
// A wave has 32 queries, one per column: S^T = K Q^T and dP^T = V dO^T over 32 keys, dS^T from
// both, dQ^T += K^T dS^T.  Half of the waves run their products while the others form dS.
// Also writes what the other kernel needs of every query: -lse * log2(e), and -dO . O.
template <int DP, int NWV>
__global__ __launch_bounds__(64 * NWV, 2) void causal_dq_kernel(CausalArgs p) {
  using T = Tile<DP>;
  constexpr int SL = T::SLOTS, DT = T::DT;
  __shared__ uint4 ks[STAGES][SL], vs[STAGES][SL];
  const AttnPlace a = attn_place(p, p.group, 32 * NWV);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int c = l & 31, h = l >> 5;
  const bool late = NWV == 8 && w >= NWV / 2;
  const int head = a.head_k * p.group + a.gq, shift = a.k_len - a.q_len;
  const int q0 = a.r0 + 32 * w, row = min(q0 + c, a.q_len - 1);
  const int last_key = row + shift;
  const int wave_keys = q0 < a.q_len ? min(q0 + 31, a.q_len - 1) + shift + 1 : 0;
  const int first_cut = (q0 + shift + 1) & ~31;
  const int keys = min(a.r0 + 32 * NWV - 1, a.q_len - 1) + shift + 1;
  const int nt = keys > 0 ? (keys + 63) / 64 : 0;
  const bf16* K = head_of(p.k, a.head_k, a.k_row);
  const bf16* V = head_of(p.v, a.head_k, a.k_row);
  const float sl2 = p.scale * kLog2e;

  const float nl2 = -p.lse[head * p.ld_lse + a.q_row + row] * kLog2e;
  float nd = 0.f;
  {
    RowOp<DP> o, d_o;
    load_row<DP>(o, head_of(p.o, head, a.q_row + row), p.d, h);
    load_row<DP>(d_o, head_of(p.d_o, head, a.q_row + row), p.d, h);
#pragma unroll
    for (int f = 0; f < T::KF; ++f)
#pragma unroll
      for (int e = 0; e < 8; ++e) nd = fmaf((float)o.f[f][e], -(float)d_o.f[f][e], nd);
    nd = add_halves(nd);
    if (wave_keys > 0 && wave_keys <= 32) {
      // dO . O is the sum of P dP, but for the rounding of O.  Of few keys O is as large as their
      // values, and its rounding as large as that of all else: what the sum of P (dP - dO . O)
      // leaves is taken off.  (350 rows of normal values: error of dQ 0.0028 -> 0.0024, of which
      // 0.0017 is its own rounding.)
      RowOp<DP> q, k, v;
      load_row<DP>(q, head_of(p.q, head, a.q_row + row), p.d, h);
      load_row<DP>(k, K + min(c, a.k_len - 1) * p.k.row, p.d, h);
      load_row<DP>(v, V + min(c, a.k_len - 1) * p.v.row, p.d, h);
      f32x16 s = zero16(), dp = zero16();
#pragma unroll
      for (int f = 0; f < T::KF; ++f) {
        s = mfma(k.f[f], q.f[f], s);
        dp = mfma(v.f[f], d_o.f[f], dp);
      }
      float off = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = exp2_fast(fmaf(s[i], sl2, nl2)) * (dp[i] + nd);
        off += acc_row(i, 0) <= last_key - 4 * h ? x : 0.f;
      }
      nd -= add_halves(off);
    }
  }
  if (h == 0 && q0 + c < a.q_len) {
    float* out = p.delta + (int64_t)head * p.rows_q + a.q_row + row;
    out[0] = nl2;
    out[(int64_t)p.heads_k * p.group * p.rows_q] = nd;
  }
  const uint32_t ks0 = lds_at(ks), vs0 = lds_at(vs);
  constexpr int AHEAD = T::KF < 4 ? 2 * T::KF : 6;   // row reads before their products begin
  f32x16 dq[DT];
  auto walk = [&](auto by_pairs) __attribute__((always_inline)) {
    // (of each walk its own, and pair by pair of each step: over all of it they would have to
    // leave the registers)
    RowOp<DP> q, d_o;
    auto operands = [&]() __attribute__((always_inline)) {
      load_row<DP>(q, head_of(p.q, head, a.q_row + row), p.d, h);
      load_row<DP>(d_o, head_of(p.d_o, head, a.q_row + row), p.d, h);
    };
    operands();
    PairCopy<DP, NWV> copy;
    copy.init(w, l, p.k.row, p.v.row, p.d);
    RowReads<DP> rread;
    rread.init(c, h);
    ColReads<DP> cread;
    cread.init(l);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dq[dt] = zero16();
    Feed kf, vf;
    kf.start(K, p.k.row, 0, min(a.k_len, 64 * nt), p.d);
    vf.start(V, p.v.row, 0, min(a.k_len, 64 * nt), p.d);
    auto issue = [&](uint32_t stage) __attribute__((always_inline)) {
      copy.copy(w, ks0 + stage, vs0 + stage, kf.next(), vf.next());
    };
    f32x16 s, dp;
    bf16x8 ds[2], first[AHEAD];
    // step u: keys 32u .. 32u + 31, half a tile, at `at` in the rings
    auto fetch = [&](uint32_t at) __attribute__((always_inline)) {
#pragma unroll
      for (int f = 0; f < AHEAD / 2; ++f) {
        first[2 * f] = rread.get(rread.base(ks0 + at, f), 0);
        first[2 * f + 1] = rread.get(rread.base(vs0 + at, f), 0);
      }
    };
    auto scores = [&](uint32_t at) __attribute__((always_inline)) {
      if constexpr (by_pairs.value) operands();
      s = dp = zero16();
#pragma unroll
      for (int f = 0; f < T::KF; ++f) {
        s = mfma(f < AHEAD / 2 ? first[2 * f] : rread.get(rread.base(ks0 + at, f), 0), q.f[f], s);
        dp = mfma(f < AHEAD / 2 ? first[2 * f + 1] : rread.get(rread.base(vs0 + at, f), 0), d_o.f[f], dp);
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
    // scores of step u + 1 at `next`, sums of step u at `at`; with the first step of a tile, the
    // tile after the next into `then`
    auto products = [&](int u, uint32_t at, uint32_t next, uint32_t then, auto sends) __attribute__((always_inline)) {
      if (32 * u >= wave_keys) {
        if constexpr (sends.value) issue(then);
        return;
      }
      scores(next);   // (past the wave's last step: of whatever lies there, for nobody)
      if constexpr (sends.value) issue(then);
      if (by_pairs.value && 32 * u >= first_cut) {
        add_pairs<DP, 32>(dq, ds, &ks[0][0] + at / 16, l, [&](int r) { return 32 * u + r <= last_key; });
        return;
      }
      const auto cols = cread.base(ks0 + at);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dq[dt] = mfma(cread.get(cols, 16 * j, dt), ds[j], dq[dt]);
      if constexpr (!by_pairs.value) {
        // 2 KF products of scores, the first AHEAD of them fetched; 4 DT half reads and 2 DT sums
        constexpr int REST = 2 * T::KF - AHEAD, EACH = (4 * DT + AHEAD - 1) / AHEAD;
        order_step<REST, 1>();
        order_step<AHEAD, EACH>();
        order_step<2 * DT, 0>();
      }
    };
    // Slots as in the forward, two steps to a tile.  Tile x is first read in the early group's slot
    // 4x - 2 (the operands fetched ahead) and last in the late group's 4x + 4; it is sent for in the
    // products of step 2x - 4, slots 4x - 7 and 4x - 6, and has arrived by the end of slot 4x - 3.
    constexpr uint32_t HALF = 32 * T::NC * 16;
    Ring ring;   // c: tile t
    ring.start(SL * 16);
    issue(ring.c);
    issue(ring.a);
    wait_copies<0>();
    lds_barrier();
    if (wave_keys > 0) {
      fetch(ring.c);
      scores(ring.c);
    }
    if (late) bare_barrier();
    for (int t = 0; t < nt; ++t) {
      slopes(2 * t);
      fetch(ring.c + HALF);
      wait_copies<0>();
      bare_barrier();
      __builtin_amdgcn_s_setprio(1);
      products(2 * t, ring.c, ring.c + HALF, ring.b, std::true_type());
      __builtin_amdgcn_s_setprio(0);
      bare_barrier();
      slopes(2 * t + 1);
      fetch(ring.a);
      bare_barrier();
      __builtin_amdgcn_s_setprio(1);
      products(2 * t + 1, ring.c + HALF, ring.a, 0, std::false_type());
      __builtin_amdgcn_s_setprio(0);
      bare_barrier();
      ring.next();
    }
    if (NWV == 8 && !late) bare_barrier();
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
// products meet the other's exponentials.  Where there are few key tiles, p.parts blocks share one,
// and a kernel of its own adds what they leave in fp32 (67 MB at most: 12 us).
template <int DP, int NWV>
__global__ __launch_bounds__(64 * NWV, 2) void causal_dkdv_kernel(CausalArgs p) {
  using T = Tile<DP>;
  constexpr int SL = T::SLOTS, DT = T::DT;
  __shared__ uint4 qs[KSTAGES][SL], ds_[KSTAGES][SL];
  // P of one tile as the lanes hold it: the upper 16 bits of fp32, and the next eight.  (Rounded to
  // bf16, as it enters dV, it would also be dS's largest error: dK's 0.0024 -> 0.0030.)
  __shared__ uint4 weights[NWV / 2][4][64], weights_low[NWV / 2][2][64];
  __shared__ __attribute__((aligned(16))) float nl2s[KSTAGES][64], nds[KSTAGES][64];
  const AttnPlace a = attn_place(p, p.parts, 16 * NWV);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int c = l & 31, h = l >> 5, pair = w % (NWV / 2);
  const bool of_second = w >= NWV / 2;
  const int shift = a.k_len - a.q_len;
  const int k0 = a.r0 + 32 * pair, row = min(k0 + c, a.k_len - 1);
  const int first_q = max(row - shift, 0);            // first query that sees the lane's key
  const int t0 = max(a.r0 - shift, 0) / 64;           // first tile with a query that sees any
  const int n_tiles = max((a.q_len + 63) / 64 - t0, 0);
  // the block's part of the group's tiles, and where it begins
  const int first_t = (int)((int64_t)n_tiles * p.group * a.gq / p.parts);
  const int nt = (int)((int64_t)n_tiles * p.group * (a.gq + 1) / p.parts) - first_t;
  const int first_head = nt > 0 ? first_t / n_tiles : 0, first_tile = nt > 0 ? first_t % n_tiles : 0;
  const int whole_q = max(min(k0 + 31, a.k_len - 1) - shift, 0);   // sees all of the wave's keys
  const float sl2 = p.scale * kLog2e;
  const uint32_t qs0 = lds_at(qs), ds0 = lds_at(ds_), nl2s0 = lds_at(nl2s), nds0 = lds_at(nds);
  constexpr int AHEAD = T::KF < 4 ? 2 * T::KF : 8;   // row reads before their products begin
  f32x16 acc[DT];
  auto walk = [&](auto by_pairs, auto is_second) __attribute__((always_inline)) {
    constexpr bool second = is_second.value;
    // (of each walk its own: over both they would have to leave the registers)
    RowOp<DP> kv;
    load_row<DP>(kv, head_of(second ? p.v : p.k, a.head_k, a.k_row + row), p.d, h);
    PairCopy<DP, NWV> copy;
    copy.init(w, l, p.q.row, p.d_o.row, p.d);
    RowReads<DP> rread;
    rread.init(c, h);
    ColReads<DP> cread;
    cread.init(l);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = zero16();
    // the first waves' rows are of Q and columns of dO, the second ones' the other way round
    const uint32_t rows0 = second ? ds0 : qs0, cols0 = second ? qs0 : ds0;
    // Tiles head by head: Q, dO, and of each query -lse * log2(e) (the first waves') or -dO . O
    const int head0 = a.head_k * p.group + first_head, t1 = t0 + first_tile;
    Feed qf, of;
    qf.start(head_of(p.q, head0, a.q_row), p.q.row, t1, a.q_len, p.d);
    of.start(head_of(p.d_o, head0, a.q_row), p.d_o.row, t1, a.q_len, p.d);
    uint64_t stats = (uint64_t)(p.delta + ((second ? (int64_t)p.heads_k * p.group : 0) + head0) * p.rows_q + a.q_row + 64 * t1);
    const uint32_t stats_tail = 4u * (uint32_t)((a.q_len - 1) % 64 + 1);
    int heads_left = nt > 0 ? p.group - 1 - first_head : 0;
    struct Next {
      buffer_t q, d_o, stats;
    };
    auto next_tile = [&]() __attribute__((always_inline)) {
      if (qf.left == 0 && heads_left > 0) {   // on to the next head's first tile
        --heads_left;
        qf.left = of.left = n_tiles;
        qf.base += 2 * p.q.head - n_tiles * qf.step;
        of.base += 2 * p.d_o.head - n_tiles * of.step;
        stats += 4 * p.rows_q - 256 * (int64_t)n_tiles;
      }
      Next x;
      x.stats = buffer_t{(uint32_t)stats, (uint32_t)(stats >> 32) & 0xffff,
                         qf.left > 1 ? 256u : qf.left == 1 ? stats_tail : 0u, 0x00027000u};
      x.q = qf.next();
      x.d_o = of.next();
      stats += 256;
      return x;
    };
    uint32_t stage_sent = 0;
    auto issue = [&](const Next& x) __attribute__((always_inline)) {
      copy.copy(w, qs0 + stage_sent * (SL * 16), ds0 + stage_sent * (SL * 16), x.q, x.d_o);
      // (64 values; each of the waves that read them sends for all, rather than one by a branch)
      copy4((second ? nds0 : nl2s0) + 256 * stage_sent, 4 * l, x.stats);
      stage_sent = (stage_sent + 1) % KSTAGES;
    };
    f32x16 s[2];
    bf16x8 x[4], first[AHEAD];
    int tile_t = first_tile;   // tile t's place among those of its head
    auto cut = [&](int r0) { return r0 < whole_q || r0 + 64 > a.q_len; };
    auto fetch = [&](uint32_t at) __attribute__((always_inline)) {
#pragma unroll
      for (int f = 0; f < AHEAD / 2; ++f) {
        const uint32_t b = rread.base(rows0 + at, f);
        first[2 * f] = rread.get(b, 0);
        first[2 * f + 1] = rread.get(b, 32);
      }
    };
    auto scores = [&](uint32_t at) __attribute__((always_inline)) {
      s[0] = s[1] = zero16();
#pragma unroll
      for (int f = 0; f < AHEAD / 2; ++f)
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) s[q2] = mfma(first[2 * f + q2], kv.f[f], s[q2]);
#pragma unroll
      for (int f = AHEAD / 2; f < T::KF; ++f) {
        const uint32_t b = rread.base(rows0 + at, f);
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) s[q2] = mfma(rread.get(b, 32 * q2), kv.f[f], s[q2]);
      }
    };
    auto form = [&](int r0, int stage) __attribute__((always_inline)) {
      const float* of_row = second ? nds[stage] : nl2s[stage];
#pragma unroll
      for (int q2 = 0; q2 < 2; ++q2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 n = *reinterpret_cast<const f32x4*>(&of_row[32 * q2 + 8 * i + 4 * h]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float& v = reinterpret_cast<float*>(&s[q2])[4 * i + e];
            v = second ? v + n[e] : exp2_fast(fmaf(v, sl2, n[e]));
          }
        }
      if constexpr (second) {
        const uint4 v2[2] = {weights_low[pair][0][l], weights_low[pair][1][l]};
        const uint32_t* low = reinterpret_cast<const uint32_t*>(v2);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 v = weights[pair][j][l];
          const uint32_t* up = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // (selector bytes 0 to 3 are of the second word, 4 to 7 of the first, 12 is zero)
            const uint32_t which = (e & 1 ? 0x0706000cu : 0x0504000cu) | (e & 3) << 8;
            s[j >> 1][8 * (j & 1) + e] *=
                __uint_as_float(__builtin_amdgcn_perm(up[e >> 1], low[2 * j + (e >> 2)], which));
          }
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
      if constexpr (!second) {
        uint32_t up[16], low[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(s[i >> 2][4 * (i & 3) + e]);
          up[2 * i] = __builtin_amdgcn_perm(v[1], v[0], 0x07060302u);
          up[2 * i + 1] = __builtin_amdgcn_perm(v[3], v[2], 0x07060302u);
          low[i] = __builtin_amdgcn_perm(v[3], v[2], 0x05010c0cu) | __builtin_amdgcn_perm(v[1], v[0], 0x0c0c0501u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) weights[pair][j][l] = make_uint4(up[4 * j], up[4 * j + 1], up[4 * j + 2], up[4 * j + 3]);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          weights_low[pair][j][l] = make_uint4(low[4 * j], low[4 * j + 1], low[4 * j + 2], low[4 * j + 3]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = pack8(s[j >> 1], j & 1);
    };
    // scores of the next tile, sums of this one
    auto products = [&](int r0, uint32_t at, uint32_t next, const Next& then) __attribute__((always_inline)) {
      scores(next);   // (past the last tile: of whatever lies there, for nobody)
      issue(then);
      if (by_pairs.value && cut(r0)) {
        add_pairs<DP, 64>(acc, x, (second ? &qs[0][0] : &ds_[0][0]) + at / 16, l,
                          [&](int r) { return r0 + r >= first_q && r0 + r < a.q_len; });
        return;
      }
      const auto cols = cread.base(cols0 + at);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[dt] = mfma(cread.get(cols, 16 * j, dt), x[j], acc[dt]);
      if constexpr (!by_pairs.value) {
        // 2 KF products of scores, the first AHEAD of them fetched; 8 DT half reads and 4 DT sums
        constexpr int REST = 2 * T::KF - AHEAD, LATER = 8 * DT - 2 * AHEAD;
        order_step<REST, 1>();
        order_step<AHEAD, 2>();
        order_step<LATER / 2, 2>();
        order_step<4 * DT - LATER / 2, 0>();
      }
    };
    // The first waves form P of tile t in slot 2t and multiply in slot 2t + 1, the second ones a slot
    // later.  Tile x is read from slot 2x - 2 (the operands fetched ahead) to slot 2x + 2, sent for in
    // slots 2x - 5 and 2x - 4, and has arrived by the end of slot 2x - 3.
    issue(next_tile());
    issue(next_tile());
    issue(next_tile());
    wait_copies<0>();
    lds_barrier();
    fetch(0);
    scores(0);
    if constexpr (second) bare_barrier();
    for (int t = 0; t < nt; ++t) {
      const int r0 = 64 * (t0 + tile_t);
      if (++tile_t == n_tiles) tile_t = 0;
      uint32_t at = t % KSTAGES * (SL * 16), next = (t + 1) % KSTAGES * (SL * 16);
      asm("" : "+s"(at), "+s"(next));
      form(r0, t % KSTAGES);
      const Next then = next_tile();
      asm volatile("" ::: "memory");
      fetch(next);
      wait_copies_and_writes<0, AHEAD>();
      bare_barrier();
      __builtin_amdgcn_s_setprio(1);
      products(r0, at, next, then);
      __builtin_amdgcn_s_setprio(0);
      bare_barrier();
    }
    if constexpr (!second) bare_barrier();
  };
  if (of_second) walk(std::false_type(), std::true_type());
  else walk(std::false_type(), std::false_type());
  // a pair that does not count must not reach the sum: see add_pairs
  if (__syncthreads_or(!finite16(acc))) {
    if (of_second) walk(std::true_type(), std::true_type());
    else walk(std::true_type(), std::false_type());
  }
  if (p.parts > 1) {
    f32x4* out = reinterpret_cast<f32x4*>(p.partial) + ((int64_t)blockIdx.x * NWV + w) * (256 * DT) + l;
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) out[64 * i] = f32x4_of(acc[i >> 2], i & 3);
    return;
  }
  if (k0 + c >= a.k_len) return;
  store_row<DP>(out_of(of_second ? p.dk : p.dv, a.head_k, a.k_row + row), acc, of_second ? p.scale : 1.f, p.d, h);
}

// The sums of a key tile's parts, in their order, 32 columns a block; lanes as above.
template <int DP, int NWV>
__global__ __launch_bounds__(64 * NWV) void causal_parts_kernel(CausalArgs p) {
  constexpr int DT = Tile<DP>::DT;
  const AttnPlace a = attn_place(p, 1, 16 * NWV);
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, c = l & 31, h = l >> 5, dt = blockIdx.y;
  const int row = a.r0 + 32 * (w % (NWV / 2)) + c;
  const bool of_second = w >= NWV / 2;
  const int64_t item = blockIdx.x / p.heads_k;
  f32x16 acc = zero16();
#pragma unroll 4
  for (int i = 0; i < p.parts; ++i) {
    const int64_t block = (item * p.parts + i) * p.heads_k + a.head_k;
    const f32x4* in = reinterpret_cast<const f32x4*>(p.partial) + (block * NWV + w) * (256 * DT) + 256 * dt + l;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 x = in[64 * j];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[4 * j + e] += x[e];
    }
  }
  if (row >= a.k_len) return;
  store_columns(out_of(of_second ? p.dk : p.dv, a.head_k, a.k_row + row), acc, of_second ? p.scale : 1.f, dt, p.d, h);
}

template <int DP, int NWV> hipError_t launch_dq(const CausalArgs& a, int items, hipStream_t s) {
  static_assert(64 * NWV <= kAttnThreads, "threads of a grid");
  hipLaunchKernelGGL((causal_dq_kernel<DP, NWV>), dim3((unsigned)items * a.heads_k * a.group),
                     dim3(64 * NWV), 0, s, a);
  return hipGetLastError();
}
template <int DP> hipError_t launch_dkdv(const CausalArgs& a, int items, hipStream_t s) {
  constexpr int NWV = causal_k_waves(DP);
  static_assert(64 * NWV <= kAttnThreads, "threads of a grid");
  hipLaunchKernelGGL((causal_dkdv_kernel<DP, NWV>), dim3((unsigned)items * a.heads_k * a.parts),
                     dim3(64 * NWV), 0, s, a);
  if (a.parts > 1)
    hipLaunchKernelGGL((causal_parts_kernel<DP, NWV>), dim3((unsigned)items * a.heads_k, DP / 32),
                       dim3(64 * NWV), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t causal_bf16_dq(const CausalArgs& a, int items, hipStream_t s) {
  switch (causal_width(a.d)) {
    case 32: return launch_dq<32, 4>(a, items, s);
    case 64: return launch_dq<64, 4>(a, items, s);
    case 96: return launch_dq<96, 4>(a, items, s);
    default: return a.q_waves == 4 ? launch_dq<128, 4>(a, items, s) : launch_dq<128, 8>(a, items, s);
  }
}
hipError_t causal_bf16_dkdv(const CausalArgs& a, int items, hipStream_t s) {
  switch (causal_width(a.d)) {
    case 32: return launch_dkdv<32>(a, items, s);
    case 64: return launch_dkdv<64>(a, items, s);
    case 96: return launch_dkdv<96>(a, items, s);
    default: return launch_dkdv<128>(a, items, s);
  }
}

}  // namespace mpipe
