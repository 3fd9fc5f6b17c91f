// Causal attention forward, bf16: o = softmax(scale q k^T) v over the keys j <= i + k_len - q_len of
// query i, tile by tile of 64 keys with the running maximum m and sum of a softmax:
//   m' = max(m, s), o = o 2^(m - m') + P v, sum = sum 2^(m - m') + P, P = 2^(s - m')
// (scores times log2(e); o and sum follow m only where it rises by more than 8: P then stays below
// 2^8, and bf16 keeps it as well as below 1).
//
// A wave has 32 queries, one per column: S^T = K Q^T leaves a query's scores in two lanes, so
// maxima and sums take one exchange, and P^T is already the operand of O^T += V^T P^T, whose V comes
// from LDS by transposing reads: nothing is shuffled or written back between the products.  Scores,
// m, sum and o are fp32; P is rounded to bf16 (half a step of 2^-8), as the matrix unit takes it.
//
// Bound by the matrix unit (4 d operations a pair) and the vector unit beside it, at the clock that
// their power leaves.  Two waves share a SIMD and run a phase apart: one's 2 KF + 4 DT products meet the
// other's 64 exponentials.  Tiles go global to LDS in copies three tiles ahead.  Measured on MI355X:
// eight sequences of up to 8192, 28/4 heads of 128, 2.52 ms, 1.08 PFLOP/s of the pairs that count (first
// kernel, fp32 products of 16 rows: 73 ms), the matrix unit busy for 55 % of the time and the vector unit
// for 50, at 1.65 to 1.8 of 2.4 GHz, no cycle lost to LDS banks; 512 rows after 32256, four sequences,
// 32/8 heads, 0.92 ms, 1.19 PFLOP/s, 64 and 55 %; one sequence of 77 7 us.
#include <type_traits>

#include "causal_bf16.h"

namespace mpipe {
namespace {

constexpr int STAGES = 3;

// NWV waves of 32 queries each.
template <int DP, int NWV>
__global__ __launch_bounds__(64 * NWV, 2) void causal_fwd_kernel(CausalArgs p) {
  using T = Tile<DP>;
  constexpr int SL = T::SLOTS, DT = T::DT;
  __shared__ uint4 ks[STAGES][SL], vs[STAGES][SL];
  constexpr int ROWS = 32 * NWV;
  const AttnPlace a = attn_place(p, p.group, ROWS);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int c = l & 31, h = l >> 5;
  const bool late = NWV == 8 && w >= NWV / 2;   // the group that runs a phase behind
  const int head = a.head_k * p.group + a.gq, shift = a.k_len - a.q_len;
  const int q0 = a.r0 + 32 * w, row = min(q0 + c, a.q_len - 1);
  const int last_key = row + shift;                            // that the lane's query sees
  const int wave_keys = q0 < a.q_len ? min(q0 + 31, a.q_len - 1) + shift + 1 : 0;
  const int first_cut = (q0 + shift + 1) & ~63;                // keys from here on some query misses
  const int keys = min(a.r0 + ROWS - 1, a.q_len - 1) + shift + 1;
  const int nt = keys > 0 ? (keys + 63) / 64 : 0;
  const bf16* K = head_of(p.k, a.head_k, a.k_row);
  const bf16* V = head_of(p.v, a.head_k, a.k_row);
  const float sl2 = p.scale * kLog2e;
  constexpr float kSlack = 8.0f;

  const uint32_t ks0 = lds_at(ks), vs0 = lds_at(vs);
  constexpr int AHEAD = T::KF < 4 ? 2 * T::KF : 8;   // reads of K before their products begin

  float m, sum;
  f32x16 o[DT];
  auto walk = [&](auto by_pairs) __attribute__((always_inline)) {
    // (of each walk its own: over both they would have to leave the registers)
    RowOp<DP> q;
    load_row<DP>(q, head_of(p.q, head, a.q_row + row), p.d, h);
    PairCopy<DP, NWV> copy;
    copy.init(w, l, p.k.row, p.v.row, p.d);
    RowReads<DP> kread;
    kread.init(c, h);
    ColReads<DP> vread;
    vread.init(l);
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    // pair t: tile t of K and tile t - 1 of V, in a stage of the ring
    Feed kf, vf;
    kf.start(K, p.k.row, 0, min(a.k_len, 64 * nt), p.d);
    vf.start(V, p.v.row, 0, min(a.k_len, 64 * nt), p.d);
    auto issue = [&](uint32_t stage) __attribute__((always_inline)) {
      copy.copy(w, ks0 + stage, vs0 + stage, kf.next(), vf.next());
    };
    f32x16 s[2];
    bf16x8 pb[4];
    bf16x8 first[AHEAD];
    // the first operands of a tile of K, and its scores
    auto fetch = [&](uint32_t stage) __attribute__((always_inline)) {
#pragma unroll
      for (int f = 0; f < AHEAD / 2; ++f) {
        const uint32_t at = kread.base(ks0 + stage, f);
        first[2 * f] = kread.get(at, 0);
        first[2 * f + 1] = kread.get(at, 32);
      }
    };
    auto scores = [&](uint32_t stage) __attribute__((always_inline)) {
      s[0] = s[1] = zero16();
#pragma unroll
      for (int f = 0; f < AHEAD / 2; ++f)
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) s[k2] = mfma(first[2 * f + k2], q.f[f], s[k2]);
#pragma unroll
      for (int f = AHEAD / 2; f < T::KF; ++f) {
        const uint32_t at = kread.base(ks0 + stage, f);
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) s[k2] = mfma(kread.get(at, 32 * k2), q.f[f], s[k2]);
      }
    };
    auto softmax = [&](int t) __attribute__((always_inline)) {
      if (64 * t >= wave_keys) return;
      if (64 * t >= first_cut) {
        const int lim = last_key - 64 * t - 4 * h;
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[k2][i] = 32 * k2 + acc_row(i, 0) <= lim ? s[k2][i] : -INFINITY;
      }
      float mx = s[0][0];
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[k2][i]);
      mx = max_halves(mx);
      const float mt = mx * sl2;
      if (__any(mt > m + kSlack)) {
        const float mn = mt > m + kSlack ? mt : m;
        const float alpha = m == -INFINITY ? 0.f : exp2_fast(m - mn);
        m = mn;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
        sum *= alpha;
      }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = exp2_fast(fmaf(s[k2][i], sl2, -ref));
          s[k2][i] = e;
          sum += e;
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) pb[j] = pack8(s[j >> 1], j & 1);
    };
    // products of tile t from `stage`, pair t + 3 into `then`
    auto products = [&](int t, uint32_t stage, uint32_t then) __attribute__((always_inline)) {
      if (64 * t >= wave_keys) {
        issue(then);
        return;
      }
      scores(stage);   // (past the wave's last tile: of whatever the stage holds, for nobody)
      issue(then);
      if (by_pairs.value && 64 * t >= first_cut) {
        add_pairs<DP, 64>(o, pb, &vs[0][0] + stage / 16, l, [&](int r) { return 64 * t + r <= last_key; });
        return;
      }
      const auto at = vread.base(vs0 + stage);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = mfma(vread.get(at, 16 * j, dt), pb[j], o[dt]);
      if constexpr (!by_pairs.value) {
        // 2 KF products of scores, the first AHEAD of them fetched; 8 DT half reads and 4 DT
        // products of values
        constexpr int REST = 2 * T::KF - AHEAD, LATER = 8 * DT - 2 * AHEAD;
        order_step<REST, 1>();
        order_step<AHEAD, 2>();
        order_step<LATER / 2, 2>();
        order_step<4 * DT - LATER / 2, 0>();
      }
    };
    // In a slot the early group takes its softmax of tile t while the late group multiplies (tile
    // t - 1), in the next one the other way round: the matrix and the vector units work at once.
    // Products of tile t are the scores of tile t + 1 and the values of tile t, both in pair t + 1.
    // A pair is sent for three tiles ahead, in the products' slot, where the stage's last reader was a
    // slot before, and has arrived a tile before its first reader.
    Ring ring;
    ring.start(SL * 16);
    copy.copy(w, ks0 + ring.c, vs0 + ring.c, kf.next(), buffer_t{0, 0, 0, 0x00027000u});
    issue(ring.a);
    issue(ring.b);
    wait_copies<0>();
    lds_barrier();
    if (wave_keys > 0) {
      fetch(ring.c);
      scores(ring.c);
    }
    if (late) bare_barrier();
    for (int t = 0; t < nt; ++t) {
      softmax(t);
      fetch(ring.a);
      wait_copies<0>();
      bare_barrier();
      __builtin_amdgcn_s_setprio(1);
      products(t, ring.a, ring.c);
      __builtin_amdgcn_s_setprio(0);
      bare_barrier();
      ring.next();
    }
    if (NWV == 8 && !late) bare_barrier();
  };
  walk(std::false_type());
  // what a query does not see must not reach it: see add_pairs
  if (__syncthreads_or(!finite16(o))) walk(std::true_type());
  sum = add_halves(sum);
  if (q0 + c >= a.q_len) return;
  const float inv = last_key < 0 ? 0.f : 1.0f / sum;
  store_row<DP>(out_of(p.o, head, a.q_row + row), o, inv, p.d, h);
  if (h == 0 && p.lse) p.lse[head * p.ld_lse + a.q_row + row] = (m + log2f(sum)) * kLn2;
}

template <int DP, int NWV> hipError_t launch(const CausalArgs& a, int items, hipStream_t s) {
  static_assert(64 * NWV <= kAttnThreads, "threads of a grid");
  hipLaunchKernelGGL((causal_fwd_kernel<DP, NWV>), dim3((unsigned)items * a.heads_k * a.group),
                     dim3(64 * NWV), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t causal_bf16_fwd(const CausalArgs& a, int items, hipStream_t s) {
  switch (causal_width(a.d)) {
    case 32: return launch<32, 4>(a, items, s);
    case 64: return launch<64, 4>(a, items, s);
    case 96: return launch<96, 4>(a, items, s);
    default: return a.q_waves == 4 ? launch<128, 4>(a, items, s) : launch<128, 8>(a, items, s);
  }
}

}  // namespace mpipe
