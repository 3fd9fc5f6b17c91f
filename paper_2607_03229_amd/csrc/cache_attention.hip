// Attention of one new token of every sequence over a paged cache (mpipe_op_cache_attention).
//
// Every key and value is read once, so HBM is the bound; the products (a group's query heads, up
// to 16 at a time, against 16 keys) take a small part of the MFMA rate.  The work is one line of
// units, TILE tokens of one (sequence, key head) each, sequences one behind the other; block b of
// W takes the units [U b / W, U (b + 1) / W), so that every block reads as much whatever the
// lengths.  U comes from the device's lengths: every block adds them up itself, and nothing has to
// be known on the host.  A block that covers a head's whole length writes its output; otherwise
// it leaves (maximum, sum, weighted values) of its part, and a second kernel joins a head's
// parts in order.  A block has at most two such parts: where it starts and where it ends.
//
// In a block a wave takes 32 of a unit's tokens: S^T = K Q^T with a query head per column, so that
// maxima and sums are lane exchanges within a column, and P^T is already the operand of
// O^T += V^T P^T.  K comes from memory in operand order; V goes through LDS, from which the
// transposing reads take it.  The next tokens' loads are in flight meanwhile.
#include "cache_places.h"

namespace mpipe {
namespace {

constexpr int NW = 4, TILE = 32 * NW;   // waves of a block, tokens of a unit
constexpr int QG = 16;                  // query heads of a column block
constexpr int MAX_BLOCKS = 512;

struct Args {
  const void *k, *v;
  const uint8_t *sk, *sv;
  CachePlaces at;   // table, ld_table, n_seq, width, n_pages, heads, d, shift
  AttnView q, o;
  const int32_t* lens;
  float* lse;
  float* part;      // [2 * blocks][QG][DP + 2]: weighted values, maximum, sum
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
  return (tokens_of(p, s, all) + TILE - 1) / TILE;
}

// Units before every sequence, by the whole block: thread t adds up a run of sequences.  Calls
// `found(s, units before s)` on the threads whose run holds unit u.  Returns all units.
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

// Where a part begins: the first unit of block b.
__device__ __forceinline__ int64_t first_unit(int64_t units, int b, int blocks) {
  return units * b / blocks;
}

template <int DP> struct PartOf {
  static constexpr int ROW = DP + 2;   // floats
};

// The queries as the products' column operand, and the products themselves: bf16 in steps of 32
// columns, fp32 in steps of 16 (four MFMAs each).
template <class T, int DP> struct Query;
template <int DP> struct Query<bf16, DP> {
  bf16x8 f[DP / 32];
  __device__ __forceinline__ void load(const bf16* Q, int d, int g) {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = 32 * i + 8 * g + e;
        f[i][e] = c < d ? Q[c] : (bf16)0.f;
      }
  }
};
template <int DP> struct Query<float, DP> {
  f32x4 f[DP / 16];
  __device__ __forceinline__ void load(const float* Q, int d, int g) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 16 * i + 4 * g + e;
        f[i][e] = c < d ? Q[c] : 0.f;
      }
  }
};

template <class T, int DP, bool F8>
__global__ __launch_bounds__(256) void cache_attn_kernel(Args p) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NDT = DP / 16, NC = DP / 8;
  __shared__ uint4 vt[NW][32 * NC];   // bf16: a wave's 32 rows of V
  __shared__ float ml[NW][2][QG];
  __shared__ int64_t sums[4];
  __shared__ int start_seq;
  __shared__ int64_t start_before;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, g = l >> 4, r = l & 15;
  const int d = p.at.d, heads_v = p.at.heads * p.col_blocks;   // (key head, column block) pairs
  if (tid == 0) start_seq = -1;
  __syncthreads();
  // the sequence that holds the block's first unit (of heads_v * the sequence's units)
  const int64_t units = heads_v * scan_units(p, sums, [&](int s, int64_t before, int64_t all) {
    const int64_t u0 = first_unit(heads_v * all, blockIdx.x, p.blocks);
    const int64_t lo = heads_v * before, hi = lo + (int64_t)heads_v * units_of(p, s);
    if (u0 >= lo && u0 < hi) {
      start_seq = s;
      start_before = lo;
    }
  });
  __syncthreads();
  int64_t u = first_unit(units, blockIdx.x, p.blocks);
  const int64_t u_end = first_unit(units, blockIdx.x + 1, p.blocks);
  if (u >= u_end) return;
  int seq = start_seq;
  int64_t seq_u0 = start_before;
  const float sl2 = p.scale * kLog2e;

  while (u < u_end) {
    bool all_there;
    const int len = tokens_of(p, seq, all_there), nt = (len + TILE - 1) / TILE;
    if (nt == 0) {   // (a sequence without tokens has no units)
      ++seq;
      continue;
    }
    const int hv = (int)((u - seq_u0) / nt), tile0 = (int)((u - seq_u0) % nt);
    const int tile1 = (int)min((int64_t)nt, tile0 + (u_end - u));
    const int head_k = hv / p.col_blocks, col = hv % p.col_blocks;
    const int nq = min(QG, p.group - QG * col);
    const int head_q = head_k * p.group + QG * col;
    // queries: column r of the products
    Query<T, DP> q;
    q.load(reinterpret_cast<const T*>(p.q.p) + p.q.row * seq + p.q.head * (head_q + min(r, nq - 1)), d, g);
    const int32_t* table = p.at.table + seq * p.at.ld_table;
    float m = -INFINITY, sum = 0.f;
    bool bad = !all_there;
    f32x4 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (int t = tile0; t < tile1; ++t) {
      const int k0 = t * TILE + 32 * w;
      if (k0 >= len) break;
      // lane l < 32 (and l + 32 again) knows where token k0 + l lies
      int64_t place;
      {
        const int tok = min(k0 + (l & 31), len - 1);
        int32_t page = table[tok >> p.at.shift];
        if ((uint32_t)page >= (uint32_t)p.at.n_pages) {
          bad = true;
          page = 0;
        }
        place = p.at.in_page(page, tok, head_k);
      }
      f32x4 s[2];
#pragma unroll
      for (int kq = 0; kq < 2; ++kq) {
        const int64_t row = __shfl(place, 16 * kq + r);
        s[kq] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (!BF) {
#pragma unroll
          for (int f = 0; f < DP / 16; ++f) {
            const int c = 16 * f + 4 * g;
            f32x4 kf = {0.f, 0.f, 0.f, 0.f};
            if (c < d) {
              if constexpr (F8) kf = load4_e4m3(reinterpret_cast<const uint8_t*>(p.k) + row * d + c, e8m0(p.sk[row]));
              else kf = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p.k) + row * d + c);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[kq] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q.f[f][e], s[kq], 0, 0, 0);
          }
        } else
#pragma unroll
        for (int f = 0; f < DP / 32; ++f) {
          const int c = 32 * f + 8 * g;
          bf16x8 kf;
#pragma unroll
          for (int e = 0; e < 8; ++e) kf[e] = (bf16)0.f;
          if (c < d) {
            if constexpr (F8) {
              float x[8];
              load8_e4m3(reinterpret_cast<const uint8_t*>(p.k) + row * d + c, e8m0(p.sk[row]), x);
#pragma unroll
              for (int e = 0; e < 8; ++e) kf[e] = (bf16)x[e];
            } else {
              kf = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const bf16*>(p.k) + row * d + c);
            }
          }
          s[kq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q.f[f], s[kq], 0, 0, 0);
        }
      }
      // V rows into LDS
      if constexpr (BF)
#pragma unroll
      for (int i = 0; i < 32 * NC / 64; ++i) {
        const int slot = 64 * i + l, vr = slot / NC, c = slot % NC;
        const int64_t row = __shfl(place, vr);
        uint4 x = make_uint4(0, 0, 0, 0);
        if (8 * c < d && k0 + vr < len) {
          if constexpr (F8) {
            float y[8];
            load8_e4m3(reinterpret_cast<const uint8_t*>(p.v) + row * d + 8 * c, e8m0(p.sv[row]), y);
            bf16x8 z;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (bf16)y[e];
            x = *reinterpret_cast<uint4*>(&z);
          } else {
            x = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.v) + row * d + 8 * c);
          }
        }
        vt[w][slot] = x;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kq = 0; kq < 2; ++kq)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = k0 + 16 * kq + 4 * g + e < len ? s[kq][e] * sl2 : -INFINITY;
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
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) o[dt] *= c;
      if constexpr (BF) {
        bf16x8 pb;
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[e] = (bf16)s[e / 4][e % 4];
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          // V^T: column 16 dt + r, tokens 4g .. 4g + 3 and 16 + 4g ..
          bf16x8 a;
          const bf16* base = reinterpret_cast<const bf16*>(vt[w]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a[e] = base[(4 * g + e) * DP + 16 * dt + r];
            a[4 + e] = base[(16 + 4 * g + e) * DP + 16 * dt + r];
          }
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb, o[dt], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int vr = 16 * (i / 4) + 4 * g + i % 4;
          const int64_t row = __shfl(place, vr);
          const float scale = F8 ? e8m0(p.sv[row]) : 1.f;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const int col_v = 16 * dt + r;
            float a = 0.f;
            if (col_v < d && k0 + vr < len) {
              if constexpr (F8)
                a = scale * __builtin_amdgcn_cvt_f32_fp8(reinterpret_cast<const uint8_t*>(p.v)[row * d + col_v], 0);
              else
                a = reinterpret_cast<const float*>(p.v)[row * d + col_v];
            }
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[i / 4][i % 4], o[dt], 0, 0, 0);
          }
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
    float* red = reinterpret_cast<float*>(vt);   // [QG][DP], a wave at a time
    for (int i = 0; i < NW; ++i) {
      if (w == i) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = m == -INFINITY ? 0.f : o[dt][e] * mine;
            float* at = red + r * DP + 16 * dt + 4 * g + e;
            *at = i == 0 ? x : *at + x;
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
      for (int i = tid; i < nq * d; i += 256) {
        const int h = i / d, c = i % d;
        T* O = reinterpret_cast<T*>(const_cast<void*>(p.o.p)) + p.o.row * seq + p.o.head * (head_q + h);
        O[c] = (T)(red[h * DP + c] / ml[0][1][h]);
      }
      if (p.lse && tid < nq)
        p.lse[(head_q + tid) * p.ld_lse + seq] = (ml[0][0][tid] + log2f(ml[0][1][tid])) * kLn2;
    } else {
      for (int i = tid; i < nq * DP; i += 256) part[i / DP * PartOf<DP>::ROW + i % DP] = red[i];
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

// Joins the parts of one (sequence, query head); sequences without tokens get their outputs here.
template <class T, int DP>
__global__ __launch_bounds__(256) void join_kernel(Args p) {
  __shared__ int64_t sums[4];
  __shared__ int64_t before_s;
  const int heads_q = p.at.heads * p.group, heads_v = p.at.heads * p.col_blocks, d = p.at.d;
  const int seq = blockIdx.x / heads_q, head = blockIdx.x % heads_q;
  const int head_k = head / p.group, col = head % p.group / QG, h = head % p.group % QG;
  const int64_t units = heads_v * scan_units(p, sums, [&](int s, int64_t before, int64_t) {
    if (s == seq) before_s = heads_v * before;
  });
  __syncthreads();
  bool all_there;
  const int len = tokens_of(p, seq, all_there), nt = (len + TILE - 1) / TILE;
  T* O = reinterpret_cast<T*>(const_cast<void*>(p.o.p)) + p.o.row * seq + p.o.head * head;
  if (nt == 0) {
    const float x = all_there ? 0.f : NAN;
    for (int c = threadIdx.x; c < d; c += 256) O[c] = (T)x;
    if (p.lse && threadIdx.x == 0) p.lse[head * p.ld_lse + seq] = all_there ? -INFINITY : NAN;
    return;
  }
  const int64_t u0 = before_s + (int64_t)(head_k * p.col_blocks + col) * nt, u1 = u0 + nt;
  // the block of a unit: the largest b with first_unit(b) <= u
  auto block_of = [&](int64_t x) {
    int64_t b = (x * p.blocks) / units;
    while (b + 1 < p.blocks && first_unit(units, (int)b + 1, p.blocks) <= x) ++b;
    while (first_unit(units, (int)b, p.blocks) > x) --b;
    return (int)b;
  };
  const int b0 = block_of(u0), b1 = block_of(u1 - 1);
  if (b0 == b1) return;   // written by that block
  auto part_of = [&](int b) {
    return p.part + ((int64_t)(2 * b + (b == b0 ? 1 : 0)) * QG + h) * PartOf<DP>::ROW;
  };
  float M = -INFINITY, tot = 0.f;
  for (int b = b0; b <= b1; ++b)
    if (first_unit(units, b, p.blocks) < first_unit(units, b + 1, p.blocks)) M = fmaxf(M, part_of(b)[DP]);
  const float ref = M == -INFINITY ? 0.f : M;
  for (int c = threadIdx.x; c < DP; c += 256) {
    float x = 0.f;
    tot = 0.f;
    for (int b = b0; b <= b1; ++b) {
      if (first_unit(units, b, p.blocks) == first_unit(units, b + 1, p.blocks)) continue;
      const float* a = part_of(b);
      const float wt = exp2_any(a[DP] - ref);
      tot += a[DP + 1] * wt;
      x += a[c] * wt;
    }
    if (c < d) O[c] = (T)(x / tot);
  }
  if (p.lse && threadIdx.x == 0) p.lse[head * p.ld_lse + seq] = (M + log2f(tot)) * kLn2;
}

template <class T, int DP, bool F8>
hipError_t launch(const Args& a, int n_blocks, int joins, hipStream_t s) {
  if (n_blocks > 0) {
    hipLaunchKernelGGL((cache_attn_kernel<T, DP, F8>), dim3(n_blocks), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL((join_kernel<T, DP>), dim3(joins), dim3(256), 0, s, a);
  return hipGetLastError();
}

int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

}  // namespace

size_t cache_attention_scratch(int n_seq, int heads_q, int heads_k, int head_dim) {
  return (size_t)2 * MAX_BLOCKS * QG * (padded(head_dim) + 2) * sizeof(float);
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
  a.ld_lse = p.ld_lse;
  a.scale = p.scale;
  a.group = p.q.heads / p.cache.heads;
  a.col_blocks = (a.group + QG - 1) / QG;
  // no more blocks than units there can be
  const int64_t units = ((int64_t)p.width * p.cache.page + TILE - 1) / TILE * p.cache.heads * a.col_blocks;
  a.blocks = (int)(units >= MAX_BLOCKS ? MAX_BLOCKS : units * p.n_seq >= MAX_BLOCKS ? MAX_BLOCKS : units * p.n_seq);
  const int joins = p.n_seq * p.q.heads;
#define MPIPE_DECODE(T, F8)                                                          \
  (p.cache.head_dim <= 64    ? launch<T, 64, F8>(a, a.blocks, joins, s)              \
   : p.cache.head_dim <= 128 ? launch<T, 128, F8>(a, a.blocks, joins, s)             \
                             : launch<T, 256, F8>(a, a.blocks, joins, s))
  const bool f8 = p.cache.dtype == MPIPE_E4M3;
  if (p.dtype == DT_BF16) return f8 ? MPIPE_DECODE(bf16, true) : MPIPE_DECODE(bf16, false);
  return f8 ? MPIPE_DECODE(float, true) : MPIPE_DECODE(float, false);
#undef MPIPE_DECODE
}

}  // namespace mpipe
