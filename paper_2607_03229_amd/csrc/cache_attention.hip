// Attention of one new token of every sequence over a paged cache (mpipe_op_cache_attention).
//
// Every key and value is read once for 16 query heads of its group, so HBM is the bound up to there (64
// sequences of up to 8192, heads of 128 to one key head, bf16: 16 of them 47 us, 64 of them 131); the
// products (up to 16 heads against 16 keys) take a small part of the bf16 MFMA rate, and half of the
// fp32 one.  The work is one line of units, TILE tokens of one (sequence, key head) each, sequences one
// behind the other; of U units each block takes ceil(U / blocks) in turn, so that every block reads as
// much whatever the lengths.  U comes from the device's lengths: every block adds them up itself, and
// nothing has to be known on the host.  A block that covers a head's whole length writes its output;
// otherwise it leaves (maximum, sum, weighted values) of its part, and a second kernel joins a head's
// parts in order.  A block has at most two such parts: where it starts and where it ends.  The second
// kernel has blocks for every sequence, so it takes the units before one from the first, which leaves
// them in scratch (16384 sequences of up to 100, 8/8 heads of 128: 0.18 ms of join beside 1.7, where it
// took 10.5 with every block adding all lengths up again).
//
// In a block a wave takes 32 of a unit's tokens: S^T = K Q^T with a query head per column, so that
// maxima and sums are lane exchanges within a column, and P^T is already the operand of
// O^T += V^T P^T.  K comes from memory in operand order; V goes through LDS, from which the
// transposing reads take it.  The next tokens' loads are in flight meanwhile.
//
// Scores, maxima, sums and outputs are fp32; the weights of a bf16 query are rounded to bf16 (half a
// step of 2^-8) for the matrix unit.  Measured on MI355X: 64 sequences of up to 16384, 32/8 heads of
// 128, bf16, pages of 32: 410 us, 5.8 TB/s, and 6 us to join (first kernel 730); four of up to
// 131072, 28/4 heads, e4m3: 98 us, 4.8 TB/s, and 7 (first 320); eight of up to 1000: 11 us, a chain
// of loads (length, page, keys), and 5 (first 27).
#include <type_traits>

#include "cache_places.h"

namespace mpipe {
namespace {

constexpr int NW = 4, TILE = 32 * NW;   // waves of a block, tokens of a unit
static_assert(TILE == kCacheUnit, "units");
constexpr int QG = 16;                  // query heads of a column block
constexpr int MAX_BLOCKS = 768;          // of any variant: three a CU

struct Args {
  const void *k, *v;
  const uint8_t *sk, *sv;
  CachePlaces at;   // table, ld_table, n_seq, width, n_pages, heads, d, shift
  AttnView q, o;
  const int32_t* lens;
  float* lse;
  float* part;      // [2 * blocks][QG][DP + 2]: weighted values, maximum, sum
  int64_t* before;  // [n_seq + 1]: units before every sequence, and all, which one kernel leaves to the other
  int64_t ld_lse;
  float scale;
  int group, col_blocks, blocks;   // query heads per key head, in blocks of QG
};

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Sequence s's tokens that can be read, and whether that is all of them.
__device__ __forceinline__ int tokens_of(const Args& p, int s, bool& all) {
  const int n = max(p.lens[s], 0);
  const int64_t most = (int64_t)p.at.width << p.at.shift;
  all = n <= most;
  return all ? n : (int)most;
}
__device__ __forceinline__ int units_of(const Args& p, int s) {
  bool all;
  return cache_units(tokens_of(p, s, all));
}

// Units before every sequence, by the whole block: thread t adds up a run of sequences.  Calls
// `found(s, units before s, all units)` for each, on the thread whose run holds it.  Returns all units.
template <class Found>
__device__ __forceinline__ int64_t scan_units(const Args& p, int64_t* sums, Found found) {
  const int t = threadIdx.x, n = p.at.n_seq, per = (n + 255) / 256;
  const int lo = min(t * per, n), hi = min(lo + per, n);
  int64_t mine = 0;
  for (int s = lo; s < hi; ++s) mine += units_of(p, s);
  int64_t x = mine;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int64_t y = __shfl_up(x, o);
    if ((t & 63) >= o) x += y;
  }
  if ((t & 63) == 63) sums[t >> 6] = x;
  __syncthreads();
  int64_t before = x - mine, all = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < (t >> 6)) before += sums[i];
    all += sums[i];
  }
  for (int s = lo; s < hi; ++s) {
    found(s, before, all);
    before += units_of(p, s);
  }
  return all;
}

// v_exp_f32: one ulp; results below the normal range become 0, which no fp32 sum of weights up
// to 1 notices
__device__ __forceinline__ float exp2_any(float x) { return __builtin_amdgcn_exp2f(x); }

// Units of a block.
__device__ __forceinline__ int64_t units_each(int64_t units, int blocks) {
  const int64_t n = units + blocks - 1;
  return n >> 32 ? n / blocks : (int64_t)((uint32_t)n / (uint32_t)blocks);
}
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

template <int DP> struct PartOf {
  static constexpr int ROW = DP + 2;   // floats
};

// The queries as the products' column operand, and the products themselves: bf16 in steps of 32
// columns, fp32 in steps of 16 (four MFMAs each).
// (8-bit keys: in the order in which lanes hold 16 of them at once, see fetch)
template <class T, int DP, bool F8> struct Query;
template <int DP, bool F8> struct Query<bf16, DP, F8> {
  bf16x8 f[DP / 32];
  __device__ __forceinline__ void load(const bf16* Q, int d, int g) {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = F8 ? 64 * (i / 2) + 16 * g + 8 * (i % 2) + e : 32 * i + 8 * g + e;
        f[i][e] = c < d ? Q[c] : (bf16)0.f;
      }
  }
};
template <int DP, bool F8> struct Query<float, DP, F8> {
  f32x4 f[DP / 16];
  __device__ __forceinline__ void load(const float* Q, int d, int g) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = F8 ? 64 * (i / 4) + 16 * g + 4 * (i % 4) + e : 16 * i + 4 * g + e;
        f[i][e] = c < d ? Q[c] : 0.f;
      }
  }
};
// Sixteen 8-bit values, columns c .. of d; EXACT: all there and aligned.
template <bool EXACT> __device__ __forceinline__ uint4 load_e4m3x16(const uint8_t* x, int c, int d) {
  if constexpr (EXACT) return *reinterpret_cast<const uint4*>(x + c);
  uint2 a = make_uint2(0, 0), b = a;
  if (c < d) a = *reinterpret_cast<const uint2*>(x + c);
  if (c + 8 < d) b = *reinterpret_cast<const uint2*>(x + c + 8);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// A bf16 wave's 32 rows of V in LDS: 16-byte chunk c of row R at c ^ mix(R), so that the transposing
// reads (8 rows x 32 bytes at a time) and the writes of whole rows meet no bank twice.  (Values of 8 bits
// are written two or four chunks a lane, which do meet: for 6 % of the time in bf16, 19 % in fp32.)
template <int DP> __device__ __forceinline__ int mix(int row) {
  return DP == 64 ? (row >> 1 & 3) << 1 : (row & 7) << 1;
}

// Where the 32 tokens from k0 of a sequence lie, for one key head: the row of d values of token
// k0 + i (tokens past the last: the last one's).  SMALL pages: lane i knows row i.  Otherwise a
// page holds all 32 and `first` is the row of k0, the same for every lane.
template <bool SMALL> struct Rows32 {
  int32_t page;    // as read, of lane l's token (SMALL) or of all
  int64_t first;
  int last;
  __device__ __forceinline__ void look(const CachePlaces& at, const int32_t* table, int k0, int len, int l) {
    last = min(31, len - 1 - k0);
    page = table[(SMALL ? k0 + min(l & 31, last) : k0) >> at.shift];
  }
  __device__ __forceinline__ void find(const CachePlaces& at, int k0, int head, int l, bool& bad) {
    const bool out = (uint32_t)page >= (uint32_t)at.n_pages;
    bad |= out;
    first = at.in_page(out ? 0 : page, SMALL ? k0 + min(l & 31, last) : k0, head);
    if constexpr (!SMALL)
      first = (int64_t)__builtin_amdgcn_readfirstlane((int)first) & 0xffffffffll |
              (int64_t)__builtin_amdgcn_readfirstlane((int)(first >> 32)) << 32;
  }
  // where row i of d values is, FULL: all 32 tokens are there
  template <bool FULL> __device__ __forceinline__ int64_t at(int i, int d) const {
    if constexpr (SMALL) return __shfl(first, i) * d;
    else return first * d + (FULL ? i : min(i, last)) * d;
  }
};

// Blocks that share a CU: eight bits leave half as many bytes under way in a wave, and take fewer
// registers.  Measured on MI355X, two -> three blocks a CU (768 in all): four sequences of up to
// 131072, 4 key heads of 128, e4m3: 146 -> 129 us; 64 of 8192, 8 of 64: 138 -> 118; bf16, 64 of up
// to 16384, 8 of 128: 426 -> 445.
constexpr int blocks_per_cu(int width, bool eight, bool bf) {
  return width == 256 ? 1 : eight && (bf || width == 64) ? 3 : 2;
}

template <class T, int DP, bool F8, bool SMALL>
__global__ __launch_bounds__(256, (blocks_per_cu(DP, F8, sizeof(T) == 2))) void cache_attn_kernel(Args p) {
  constexpr bool BF = sizeof(T) == 2;
  // V's rows in LDS: NC chunks of 16 bytes, PC apart (fp32: so that four rows four apart, which
  // a read takes at once, lie in different banks)
  constexpr int NDT = DP / 16, NF = BF ? DP / 32 : DP / 16;
  constexpr int NC = BF ? DP / 8 : DP / 4, PC = BF ? NC : NC + 1;
  __shared__ uint4 vt[NW][32 * PC];
  __shared__ float ml[NW][2][QG];
  __shared__ int64_t sums[4];
  __shared__ int start_seq;
  __shared__ int64_t start_before;
  const int tid = threadIdx.x, l = tid & 63, g = l >> 4, r = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d = p.at.d, heads_v = p.at.heads * p.col_blocks;   // (key head, column block) pairs
  // the sequence that holds the block's first unit (of heads_v * the sequence's units)
  const int64_t units = heads_v * scan_units(p, sums, [&](int s, int64_t before, int64_t all) {
    const int64_t u0 = blockIdx.x * units_each(heads_v * all, p.blocks);
    const int64_t lo = heads_v * before, hi = lo + (int64_t)heads_v * units_of(p, s);
    if (u0 >= lo && u0 < hi) {
      start_seq = s;
      start_before = lo;
    }
    if (blockIdx.x == 0) {
      p.before[s] = before;
      if (s == 0) p.before[p.at.n_seq] = all;
    }
  });
  __syncthreads();
  const int64_t each = units_each(units, p.blocks);
  int64_t u = blockIdx.x * each;
  const int64_t u_end = min(u + each, units);
  if (u >= u_end) return;
  int seq = __builtin_amdgcn_readfirstlane(start_seq);
  int64_t seq_u0 = start_before;
  const float sl2 = p.scale * kLog2e;

  while (u < u_end) {
    bool all_there;
    const int len = __builtin_amdgcn_readfirstlane(tokens_of(p, seq, all_there)), nt = cache_units(len);
    if (nt == 0) {   // (a sequence without tokens has no units)
      ++seq;
      continue;
    }
    const int hv = __builtin_amdgcn_readfirstlane((int)quotient(u - seq_u0, nt));
    const int tile0 = __builtin_amdgcn_readfirstlane((int)(u - seq_u0 - (int64_t)hv * nt));
    const int tile1 = __builtin_amdgcn_readfirstlane((int)min((int64_t)nt, tile0 + (u_end - u)));
    const int head_k = hv / p.col_blocks, col = hv % p.col_blocks;
    const int nq = min(QG, p.group - QG * col);
    const int head_q = head_k * p.group + QG * col;
    const int32_t* table = p.at.table + seq * p.at.ld_table;
    bool bad = !all_there;

    // one tile's keys as the products' row operand, and its values as they lie
    Rows32<SMALL> rows, ahead;   // of the tile under way, and of the one after it
    // (of 8 bits, a lane holds 16 values of a row at once: 64 f + 16 g .. of its key)
    constexpr int NK = F8 ? DP / 64 : NF, NV = F8 ? DP / 32 : NC / 2, VE = F8 ? 16 : BF ? 8 : 4;
    constexpr int VS = DP / VE;                     // slots of V's rows
    uint4 kr[2][NK], vr[NV];
    uint8_t scale_k = 0, scale_v = 0;               // of token l % 32, as stored
    auto fetch_as = [&](auto exact, auto full) __attribute__((always_inline)) {
      constexpr bool EXACT = exact.value, FULL = full.value;
      if constexpr (F8) {
        const int64_t row = SMALL ? rows.first : rows.first + min(l & 31, rows.last);
        scale_k = p.sk[row];
        scale_v = p.sv[row];
      }
#pragma unroll
      for (int kq = 0; kq < 2; ++kq) {
        const int64_t at = rows.template at<FULL>(16 * kq + r, d);
#pragma unroll
        for (int f = 0; f < NK; ++f) {
          if constexpr (F8) {
            kr[kq][f] = load_e4m3x16<EXACT>(reinterpret_cast<const uint8_t*>(p.k) + at, 64 * f + 16 * g, d);
          } else {
            const int c = BF ? 32 * f + 8 * g : 16 * f + 4 * g;
            if (!EXACT) kr[kq][f] = make_uint4(0, 0, 0, 0);
            if (EXACT || c < d) kr[kq][f] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.k) + at + c);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int slot = 64 * i + l, c = slot % VS * VE;
        const int64_t at = rows.template at<FULL>(slot / VS, d);
        if constexpr (F8) {
          vr[i] = load_e4m3x16<EXACT>(reinterpret_cast<const uint8_t*>(p.v) + at, c, d);
        } else {
          if (!EXACT) vr[i] = make_uint4(0, 0, 0, 0);
          if (EXACT || c < d) vr[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.v) + at + c);
        }
      }
    };
    auto fetch = [&]() __attribute__((always_inline)) {
      // (plain fp32 has no registers for a second form)
      if ((!BF && !F8) || d < DP || rows.last < 31) fetch_as(std::false_type(), std::false_type());
      else fetch_as(std::true_type(), std::true_type());
    };
    // wave w's tokens of tile t, of 0 .. tile1 - 1: below 2^31
    auto start = [&](int t) { return t * TILE + 32 * w; };
    auto there = [&](int t) { return t < tile1 && start(t) < len; };
    if (there(tile0)) {
      rows.look(p.at, table, start(tile0), len, l);
      if (there(tile0 + 1)) ahead.look(p.at, table, start(tile0 + 1), len, l);
      rows.find(p.at, start(tile0), head_k, l, bad);
      fetch();
    }
    Query<T, DP, F8> q;
    q.load(reinterpret_cast<const T*>(p.q.p) + p.q.row * seq + p.q.head * (head_q + min(r, nq - 1)), d, g);
    float m = -INFINITY, sum = 0.f;
    f32x4 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int t = tile0; t < tile1; ++t) {
      const int k0 = start(t);
      if (k0 >= len) break;
      const uint32_t ku = k0, end = len;   // (k0 plus a row may be 2^31 and more)
      const float scale_kt = F8 ? e8m0(scale_k) : 1.f, scale_vt = F8 ? e8m0(scale_v) : 1.f;
      f32x4 s[2];
#pragma unroll
      for (int kq = 0; kq < 2; ++kq) {
        s[kq] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float scale = F8 ? __shfl(scale_kt, 16 * kq + r) : 1.f;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const uint32_t* word = reinterpret_cast<const uint32_t*>(&kr[kq][F8 ? (BF ? f / 2 : f / 4) : f]);
          if constexpr (BF) {
            bf16x8 kf;
            if constexpr (F8) kf = bf16_of_e4m3(make_uint2(word[2 * (f % 2)], word[2 * (f % 2) + 1]), scale);
            else kf = *reinterpret_cast<const bf16x8*>(word);
            s[kq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q.f[f], s[kq], 0, 0, 0);
          } else {
            f32x4 kf;
            if constexpr (F8) kf = f32_of_e4m3(word[f % 4], scale);
            else kf = *reinterpret_cast<const f32x4*>(word);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[kq] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q.f[f][e], s[kq], 0, 0, 0);
          }
        }
      }
      if (ku + 32 > end) {   // rows past the last token: 0 times the last one again could be NaN
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (ku + (64 * i + l) / VS >= end) vr[i] = make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int slot = 64 * i + l, row = slot / VS;
        const float scale = F8 ? __shfl(scale_vt, row) : 1.f;
        const uint32_t word[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
#pragma unroll
        for (int j = 0; j < (F8 ? (BF ? 2 : 4) : 1); ++j) {
          uint4 x = vr[i];
          if constexpr (F8 && BF) {
            const bf16x8 y = bf16_of_e4m3(make_uint2(word[2 * j], word[2 * j + 1]), scale);
            x = *reinterpret_cast<const uint4*>(&y);
          } else if constexpr (F8) {
            const f32x4 y = f32_of_e4m3(word[j], scale);
            x = *reinterpret_cast<const uint4*>(&y);
          }
          const int chunk = slot % VS * (F8 ? (BF ? 2 : 4) : 1) + j;
          vt[w][row * PC + (BF ? chunk ^ mix<DP>(row) : chunk)] = x;
        }
      }
      if (there(t + 1)) {   // the next tile's bytes on their way, and where the one after it lies
        rows = ahead;
        rows.find(p.at, start(t + 1), head_k, l, bad);
        if (there(t + 2)) ahead.look(p.at, table, start(t + 2), len, l);
        fetch();
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kq = 0; kq < 2; ++kq)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = ku + 16 * kq + 4 * g + e < end ? s[kq][e] * sl2 : -INFINITY;
          s[kq][e] = x;
          mx = fmaxf(mx, x);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn, c = exp2_any(m - ref);
      m = mn;
      sum *= c;
#pragma unroll
      for (int kq = 0; kq < 2; ++kq)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[kq][e] = exp2_any(s[kq][e] - ref);
          sum += s[kq][e];
        }
      if (__any(c != 1.f)) {   // a new maximum somewhere
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] *= c;
      }
      if constexpr (BF) {
        bf16x8 pb;
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[e] = (bf16)s[e / 4][e % 4];
        const char* base = reinterpret_cast<const char*>(vt[w]);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          // V^T: column 16 dt + r, tokens 4g .. 4g + 3 and 16 + 4g ..
          bf16x8 a;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 16 * i + 4 * g + (r >> 2), chunk = 2 * dt + ((r & 3) >> 1);
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4*)(base + (row * NC + (chunk ^ mix<DP>(row))) * 16 + (r & 1) * 8));
            const bf16* y = reinterpret_cast<const bf16*>(&x);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[4 * i + e] = y[e];
          }
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb, o[dt], 0, 0, 0);
        }
      } else {
        const float* base = reinterpret_cast<const float*>(vt[w]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const float a = base[(16 * (i / 4) + 4 * g + i % 4) * (4 * PC) + 16 * dt + r];
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[i / 4][i % 4], o[dt], 0, 0, 0);
          }
      }
    }
    // the block's four waves, in order
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (__any(bad)) sum = NAN;
    if (g == 0) {
      ml[w][0][r] = m;
      ml[w][1][r] = sum;
    }
    __syncthreads();
    float M = -INFINITY, tot = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) M = fmaxf(M, ml[i][0][r]);
    const float ref = M == -INFINITY ? 0.f : M, mine = exp2_any(m - ref);
#pragma unroll
    for (int i = 0; i < NW; ++i) tot += ml[i][1][r] * exp2_any(ml[i][0][r] - ref);
    float* red = reinterpret_cast<float*>(vt);   // a wave's [QG][DP + 4]
    constexpr int RP = DP + 4;
    static_assert(QG * RP * sizeof(float) <= sizeof(vt) / 2, "two waves' values");
    // two waves at a time
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (w / 2 == half) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          f32x4 x = m == -INFINITY ? f32x4{0.f, 0.f, 0.f, 0.f} : o[dt] * mine;
          f32x4* at = reinterpret_cast<f32x4*>(red + ((w & 1) * QG + r) * RP + 16 * dt + 4 * g);
          if (half) x += *at;
          *at = x;
        }
      }
      __syncthreads();
    }
    const bool whole = tile0 == 0 && tile1 == nt;
    float* part = p.part + (int64_t)(2 * blockIdx.x + (tile0 == 0 ? 1 : 0)) * QG * PartOf<DP>::ROW;
    if (whole) {
      // (M and tot are of this lane's column; the outputs go by rows)
      if (w == 0 && g == 0) {
        ml[0][0][r] = M;
        ml[0][1][r] = tot;
      }
      __syncthreads();
      for (int i = tid; i < nq * DP; i += 256) {
        const int h = i / DP, c = i % DP;
        T* O = reinterpret_cast<T*>(const_cast<void*>(p.o.p)) + p.o.row * seq + p.o.head * (head_q + h);
        if (c < d) O[c] = (T)((red[h * RP + c] + red[(QG + h) * RP + c]) / ml[0][1][h]);
      }
      if (p.lse && tid < nq)
        p.lse[(head_q + tid) * p.ld_lse + seq] = (ml[0][0][tid] + log2f(ml[0][1][tid])) * kLn2;
    } else {
      for (int i = tid; i < nq * DP; i += 256) {
        const int h = i / DP, c = i % DP;
        part[h * PartOf<DP>::ROW + c] = red[h * RP + c] + red[(QG + h) * RP + c];
      }
      if (w == 0 && g == 0 && r < nq) {
        part[r * PartOf<DP>::ROW + DP] = M;
        part[r * PartOf<DP>::ROW + DP + 1] = tot;
      }
    }
    __syncthreads();
    u += tile1 - tile0;
    if (u - seq_u0 == (int64_t)heads_v * nt) {
      ++seq;
      seq_u0 = u;
    }
  }
}

// One query head's parts of n blocks from b0 on: part i is block b0 + i's; the first block's begins the
// head, the others' begin the block.  h: the head's place in its column block.
template <int DP> __device__ __forceinline__ const float* part_of(const Args& p, int b0, int i, int h) {
  return p.part + ((int64_t)(2 * (b0 + i) + (i == 0 ? 1 : 0)) * QG + h) * PartOf<DP>::ROW;
}

// Joins them with a block.
template <class T, int DP>
__device__ __forceinline__ void join_by_block(const Args& p, int seq, int head, int h, int b0, int n) {
  constexpr int LANES = 256 / DP;   // threads to a column
  __shared__ float weight[MAX_BLOCKS], top[4], total[4], cols[256];
  const int tid = threadIdx.x;
  float m = -INFINITY;
  for (int i = tid; i < n; i += 256) {
    weight[i] = part_of<DP>(p, b0, i, h)[DP];
    m = fmaxf(m, weight[i]);
  }
  m = warp_max(m);
  if (tid % 64 == 0) top[tid / 64] = m;
  __syncthreads();
  const float M = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), ref = M == -INFINITY ? 0.f : M;
  float tot = 0.f;
  for (int i = tid; i < n; i += 256) {
    weight[i] = exp2_any(weight[i] - ref);
    tot += part_of<DP>(p, b0, i, h)[DP + 1] * weight[i];
  }
  tot = warp_sum(tot);
  if (tid % 64 == 0) total[tid / 64] = tot;
  __syncthreads();
  tot = total[0] + total[1] + total[2] + total[3];
  const int c = tid % DP;
  float x = 0.f;
#pragma unroll 8
  for (int i = tid / DP; i < n; i += LANES) x = fmaf(part_of<DP>(p, b0, i, h)[c], weight[i], x);
  if constexpr (LANES > 1) {
    cols[tid] = x;
    __syncthreads();
    if (tid >= DP) return;
#pragma unroll
    for (int i = 1; i < LANES; ++i) x += cols[i * DP + c];
  }
  if (c < p.at.d) reinterpret_cast<T*>(const_cast<void*>(p.o.p))[p.o.row * seq + p.o.head * head + c] = (T)(x / tot);
  if (p.lse && tid == 0) p.lse[head * p.ld_lse + seq] = (M + log2f(tot)) * kLn2;
}

// Joins the parts of one (sequence, query head) with a block, or (ALL) of the query heads of a column
// block with a wave each; sequences without tokens get their outputs here.
//
// A wave adds a head's parts one by one, and a column block has up to four heads for each, so (ALL)
// heads of more than LONG parts get a block each all the same: those behind the column blocks'.  More
// than LONG parts are LONG blocks at least that begin inside the head, one of which has a number that is a
// multiple of LONG, so every such number is looked at.  Measured on MI355X, us of the join, heads of 128,
// without these blocks -> with them: one sequence of 131072 tokens among 255 of 100, 16/1 heads, 108 -> 15
// (beside 39 of the attention), among 63, 28/4 heads, 22 -> 8.  With them 256 sequences of up to 512, 28/4
// heads, none of them long, take 6.1 us, and of up to 200, 8/8 heads, 5.1.
constexpr int LONG = 16;

template <class T, int DP, bool ALL>
__global__ __launch_bounds__(256) void join_kernel(Args p) {
  __shared__ int long_seq;
  const int tid = threadIdx.x, heads_v = p.at.heads * p.col_blocks, d = p.at.d;
  const int items = ALL ? heads_v : p.at.heads * p.group;   // of a sequence
  const int of_long = ALL ? (int)blockIdx.x - p.at.n_seq * items : -1;
  if (ALL && of_long >= 0) {
    const int width = min(QG, p.group), b = (of_long / width + 1) * LONG, h = of_long % width;
    const int64_t each = units_each(heads_v * p.before[p.at.n_seq], p.blocks), u = b * each;
    if (tid == 0) long_seq = -1;
    __syncthreads();
    // the sequence that holds block b's first unit
    for (int s = tid; s < p.at.n_seq; s += 256)
      if (heads_v * p.before[s] <= u && u < heads_v * p.before[s + 1]) long_seq = s;
    __syncthreads();
    const int seq = long_seq;
    if (seq < 0) return;   // no such unit
    const int nt = units_of(p, seq);
    const int64_t seq_u0 = heads_v * p.before[seq];
    const int hv = (int)quotient(u - seq_u0, nt);
    const int64_t u0 = seq_u0 + (int64_t)hv * nt;
    const int b0 = (int)quotient(u0, each), n = (int)quotient(u0 + nt - 1, each) - b0 + 1;
    const int first = hv % p.col_blocks * QG;
    // (the first such number inside the head joins it)
    if (n <= LONG || b - LONG > b0 || b == b0 || first + h >= p.group) return;
    join_by_block<T, DP>(p, seq, hv / p.col_blocks * p.group + first + h, h, b0, n);
    return;
  }
  const int seq = blockIdx.x / items, item = blockIdx.x % items;
  const int head_k = item / (ALL ? p.col_blocks : p.group);
  const int first = ALL ? item % p.col_blocks * QG : item % p.group;   // of the key head's
  const int count = ALL ? min(QG, p.group - first) : 1, col = first / QG;
  bool all_there;
  const int len = tokens_of(p, seq, all_there), nt = cache_units(len);
  int b0 = 0, n = 0;
  if (nt > 0) {   // (without any unit nobody wrote `before`)
    const int64_t each = units_each(heads_v * p.before[p.at.n_seq], p.blocks);
    const int64_t u0 = heads_v * p.before[seq] + (int64_t)(head_k * p.col_blocks + col) * nt;
    b0 = (int)quotient(u0, each);
    n = (int)quotient(u0 + nt - 1, each) - b0 + 1;
  }
  if (n == 1 || (ALL && n > LONG)) return;   // written by its block, or joined by those behind
  auto out_of = [&](int head) {
    return reinterpret_cast<T*>(const_cast<void*>(p.o.p)) + p.o.row * seq + p.o.head * head;
  };
  const int head0 = head_k * p.group + first;
  if (nt == 0) {
    const float x = all_there ? 0.f : NAN;
    for (int i = tid; i < count * d; i += 256) out_of(head0 + i / d)[i % d] = (T)x;
    if (p.lse && tid < count) p.lse[(head0 + tid) * p.ld_lse + seq] = all_there ? -INFINITY : NAN;
    return;
  }
  if constexpr (ALL) {
    const int l = tid & 63;
    for (int h = tid >> 6; h < count; h += 4) {
      const float m = l < n ? part_of<DP>(p, b0, l, h)[DP] : -INFINITY;
      const float M = warp_max(m), ref = M == -INFINITY ? 0.f : M;
      float tot = 0.f, x[DP / 64];
#pragma unroll
      for (int j = 0; j < DP / 64; ++j) x[j] = 0.f;
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const float* part = part_of<DP>(p, b0, i, h);
        const float weight = exp2_any(part[DP] - ref);
        tot += part[DP + 1] * weight;
#pragma unroll
        for (int j = 0; j < DP / 64; ++j) x[j] = fmaf(part[64 * j + l], weight, x[j]);
      }
      T* O = out_of(head0 + h);
#pragma unroll
      for (int j = 0; j < DP / 64; ++j)
        if (64 * j + l < d) O[64 * j + l] = (T)(x[j] / tot);
      if (p.lse && l == 0) p.lse[(head0 + h) * p.ld_lse + seq] = (M + log2f(tot)) * kLn2;
    }
  } else {
    join_by_block<T, DP>(p, seq, head0, first % QG, b0, n);
  }
}

template <class T, int DP, bool F8, bool SMALL>
hipError_t launch(Args& a, int64_t units, hipStream_t s) {
  a.blocks = (int)(units < 256 * blocks_per_cu(DP, F8, sizeof(T) == 2) ? units : 256 * blocks_per_cu(DP, F8, sizeof(T) == 2));
  static_assert(256 * blocks_per_cu(DP, F8, sizeof(T) == 2) <= MAX_BLOCKS, "parts and weights");
  if (a.blocks > 0) {
    hipLaunchKernelGGL((cache_attn_kernel<T, DP, F8, SMALL>), dim3(a.blocks), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  // A query head has a block of its own, or, from 256 column blocks on (one for every CU), a wave.
  // Measured on MI355X, us of the join, 28/4 heads of 128, block -> wave: 256 sequences of up to 512
  // 16.3 -> 7.1, 100 of up to 30000 12.6 -> 8.8, 64 of up to 1000 7.0 -> 6.5; 8 of up to 1000 5.7 -> 7.1,
  // four of up to 131072 7.3 -> 17.  (All of them some 1 us more than now: each block added the lengths up.)
  const int columns = a.at.n_seq * a.at.heads * a.col_blocks;
  if (columns >= 256)
    hipLaunchKernelGGL((join_kernel<T, DP, true>),
                       dim3(columns + (a.blocks - 1) / LONG * (a.group < QG ? a.group : QG)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((join_kernel<T, DP, false>), dim3(a.at.n_seq * a.at.heads * a.group), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <class T, bool F8, bool SMALL>
hipError_t by_width(Args& a, int64_t units, hipStream_t s) {
  return a.at.d <= 64    ? launch<T, 64, F8, SMALL>(a, units, s)
         : a.at.d <= 128 ? launch<T, 128, F8, SMALL>(a, units, s)
                         : launch<T, 256, F8, SMALL>(a, units, s);
}
template <class T, bool F8> hipError_t by_page(Args& a, int64_t units, hipStream_t s) {
  return a.at.shift < 5 ? by_width<T, F8, true>(a, units, s) : by_width<T, F8, false>(a, units, s);
}

int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

}  // namespace

// two parts a block, and the units before every sequence; up to 4095 of them the size is one, so that
// a batch may grow in it
static size_t part_bytes(int head_dim) {
  return (size_t)2 * MAX_BLOCKS * QG * (padded(head_dim) + 2) * sizeof(float);
}
size_t cache_attention_scratch(int n_seq, int head_dim) {
  return part_bytes(head_dim) + (n_seq < 4096 ? 4096 : (size_t)n_seq + 1) * sizeof(int64_t);
}

hipError_t cache_attention(const CacheAttention& p, hipStream_t s) {
  Args a;
  a.k = p.cache.k;
  a.v = p.cache.v;
  a.sk = p.cache.k_scale;
  a.sv = p.cache.v_scale;
  a.at = cache_places(p.cache, p.table, p.ld_table, p.n_seq, p.width, nullptr, nullptr);
  a.q = {p.q.p, p.q.row, p.q.head};
  a.o = {p.o.p, p.o.row, p.o.head};
  a.lens = p.lens;
  a.lse = p.lse;
  a.part = p.scratch;
  a.before = reinterpret_cast<int64_t*>((char*)p.scratch + part_bytes(p.cache.head_dim));
  a.ld_lse = p.ld_lse;
  a.scale = p.scale;
  a.group = p.q.heads / p.cache.heads;
  a.col_blocks = (a.group + QG - 1) / QG;
  // (no more blocks than units there can be)
  const int64_t units = ((int64_t)p.width * p.cache.page + TILE - 1) / TILE * p.cache.heads * a.col_blocks * p.n_seq;
  const bool f8 = p.cache.dtype == MPIPE_E4M3;
  if (p.dtype == DT_BF16) return f8 ? by_page<bf16, true>(a, units, s) : by_page<bf16, false>(a, units, s);
  return f8 ? by_page<float, true>(a, units, s) : by_page<float, false>(a, units, s);
}

}  // namespace mpipe
