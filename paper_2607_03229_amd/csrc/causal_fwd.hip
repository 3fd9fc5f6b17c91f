// Causal attention forward, bf16.
#include <type_traits>

#include "causal_bf16.h"

namespace mpipe {
namespace {

constexpr int NWV = 8;              // waves of a block, 32 queries each
constexpr int ROWS = kForwardRows;
static_assert(ROWS == 32 * NWV, "32 queries a wave");
constexpr int STAGES = 3;

template <int DP>
__global__ __launch_bounds__(64 * NWV, 2) void causal_fwd_kernel(CausalArgs p) {
  using T = Tile<DP>;
  constexpr int SL = T::SLOTS, DT = T::DT;
  __shared__ uint4 ks[STAGES][SL], vs[STAGES][SL];
  const AttnPlace a = attn_place(p, p.group, ROWS);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int c = l & 31, h = l >> 5;
  const bool late = w >= NWV / 2;   // the group that runs a phase behind
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

  RowOp<DP> q;
  load_row<DP>(q, head_of(p.q, head, a.q_row + row), p.d, h);
  PairCopy<DP, NWV> copy;
  copy.init(w, l, p.k.row, p.v.row);
  RowReads<DP> kread;
  kread.init(c, h);
  ColReads<DP> vread;
  vread.init(l);
  const uint32_t ks0 = lds_at(ks), vs0 = lds_at(vs);
  // pair t: tile t of K and tile t - 1 of V, in stage t mod 3
  auto issue = [&](int t) __attribute__((always_inline)) {
    const uint32_t stage = stage_of<STAGES>(t) * (SL * 16);
#pragma unroll
    for (int i = 0; i < PairCopy<DP, NWV>::N; ++i) {
      const bool of_k = copy.of_x(i, w);
      const int tt = of_k ? t : t - 1;
      if (tt >= 0 && tt < nt)
        copy.copy(i, w, l, (of_k ? ks0 : vs0) + stage, (of_k ? K : V) + 64 * tt * (of_k ? p.k.row : p.v.row),
                  a.k_len - 64 * tt, p.d);
    }
  };

  float m, sum;
  f32x16 o[DT];
  auto walk = [&](auto by_pairs) __attribute__((always_inline)) {
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = zero16();
    f32x16 s[2];
    bf16x8 pb[4];
    auto scores = [&](int t) __attribute__((always_inline)) {
      if (64 * t >= wave_keys) return;
      const uint32_t kt = ks0 + stage_of<STAGES>(t) * (SL * 16);
      s[0] = s[1] = zero16();
#pragma unroll
      for (int f = 0; f < T::KF; ++f) {
        const uint32_t at = kread.base(kt, f);
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
      mx = fmaxf(mx, __shfl_xor(mx, 32));
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
    auto values = [&](int t) __attribute__((always_inline)) {
      if (64 * t >= wave_keys) return;
      const uint32_t stage = stage_of<STAGES>(t + 1);
      if (by_pairs.value && 64 * t >= first_cut) {
        add_pairs<DP, 64>(o, pb, vs[stage], l, [&](int r) { return 64 * t + r <= last_key; });
        return;
      }
      const auto at = vread.base(vs0 + stage * (SL * 16));
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = mfma(vread.get(at, 16 * j, dt), pb[j], o[dt]);
    };
    // The early group's softmax of tile t meets the late group's products of tile t - 1 in a
    // slot, and the other way round in the next: the matrix and the vector units work at once.
    // Products of tile t are the scores of tile t + 1 and the values of tile t, both in pair
    // t + 1.  It was sent for two slots before the early group reads it; its stage's last reader is the
    // late group, one slot before that.
    issue(0);
    issue(1);
    wait_copies<0>();
    lds_barrier();
    scores(0);
    if (late) lds_barrier();
    for (int t = 0; t < nt; ++t) {
      issue(t + 2);
      softmax(t);
      if (!late) {   // pair t + 1 is there; t + 2, where it is a whole one, may be under way
        if (t + 2 < nt) wait_copies<PairCopy<DP, NWV>::N>();
        else wait_copies<0>();
      }
      lds_barrier();
      __builtin_amdgcn_s_setprio(1);
      if (t + 1 < nt) scores(t + 1);
      values(t);
      __builtin_amdgcn_s_setprio(0);
      if (late) wait_copies<0>();
      lds_barrier();
    }
    if (!late) lds_barrier();
  };
  walk(std::false_type());
  // what a query does not see must not reach it: see add_pairs
  if (__syncthreads_or(!finite16(o))) walk(std::true_type());
  sum += __shfl_xor(sum, 32);
  if (q0 + c >= a.q_len) return;
  const float inv = last_key < 0 ? 0.f : 1.0f / sum;
  store_row<DP>(out_of(p.o, head, a.q_row + row), o, inv, p.d, h);
  if (h == 0 && p.lse) p.lse[head * p.ld_lse + a.q_row + row] = (m + log2f(sum)) * kLn2;
}

template <int DP> hipError_t launch(const CausalArgs& a, int items, hipStream_t s) {
  hipLaunchKernelGGL(causal_fwd_kernel<DP>, dim3((unsigned)items * a.heads_k * a.group),
                     dim3(64 * NWV), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t causal_bf16_fwd(const CausalArgs& a, int items, hipStream_t s) {
  return a.d <= 32 ? launch<32>(a, items, s) : a.d <= 64 ? launch<64>(a, items, s)
         : a.d <= 96 ? launch<96>(a, items, s) : launch<128>(a, items, s);
}

}  // namespace mpipe
