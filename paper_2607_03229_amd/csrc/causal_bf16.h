// Shared pieces of the bf16 kernels of causal attention (causal_fwd.hip, causal_bwd.hip).
//
// A tile is 64 rows of one head, DP columns wide (32, 64, 96 or 128; columns past head_dim and
// rows past the sequence are zeros), row-major in LDS in chunks of 16 bytes, chunk c of row R at
// c ^ swz(R).  It is filled by 16-byte global-to-LDS copies, whose lane l writes slot base + l,
// so each lane picks the source of its slot.  Two kinds of reads take MFMA operands from it:
//   rows        16 bytes of row l % 32: sixteen rows at a time fall on sixteen different chunks
//   transposed  (ds_read_b64_tr_b16) four rows x 64 bytes at a time: swz moves rows of one such
//               group to four different groups of four chunks
// so neither meets a bank twice.
//
// MFMA operands (v_mfma_f32_32x32x16_bf16), lane l = 32 h + c: A holds row c, B column c, both the
// eight reduction indices 8h .. 8h + 7; the accumulator's element i is row 8 (i / 4) + 4h + i % 4
// of column c.
#pragma once
#include "attn_kernels.h"
#include "common.h"

namespace mpipe {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <int DP> struct Tile {
  static constexpr int NC = DP / 8;         // chunks of a row
  static constexpr int SLOTS = 64 * NC;
  static constexpr int KF = DP / 16;        // 16-wide steps over the columns
  static constexpr int DT = DP / 32;        // 32-wide output tiles
};

template <int DP> __device__ __forceinline__ int swz(int row) {
  const int lo = (row >> 2) & 3;
  if constexpr (DP == 128) return lo | (row & 3) << 2;
  if constexpr (DP == 64) return lo | ((row >> 1) & 1) << 2;
  return lo;
}
// A lane's places in a tile, bytes from its start, once a kernel; a read adds the tile's LDS
// address, and what is a multiple of 16 rows is part of the instruction.
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
template <int DP> struct RowReads {   // rows r0 + c (r0 a multiple of 32), columns 16f + 8h ..
  uint32_t at[Tile<DP>::KF];
  __device__ __forceinline__ void init(int c, int h) {
#pragma unroll
    for (int f = 0; f < Tile<DP>::KF; ++f) at[f] = (c * Tile<DP>::NC + ((2 * f + h) ^ swz<DP>(c))) * 16;
  }
  // The place of step f in a tile, kept whole: left to itself the compiler keeps the sums of `at`
  // and every constant over the loop, in registers that the kernels do not have.
  __device__ __forceinline__ uint32_t base(uint32_t tile, int f) const {
    uint32_t b = tile + at[f];
    asm("" : "+v"(b));
    return b;
  }
  __device__ __forceinline__ static bf16x8 get(uint32_t base, int r0) {
    typedef __attribute__((address_space(3))) const char lds_char;
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
    return *reinterpret_cast<lds_bf16x8*>(reinterpret_cast<lds_char*>(base) + r0 * Tile<DP>::NC * 16);
  }
};
// Transposed: column 32 dt + c, rows k0 + 4h .. + 3 and k0 + 8 + 4h .. + 3 (k0 a multiple of
// 16): the rows whose scores an accumulator's elements 8j .. 8j + 7 hold.
template <int DP> struct ColReads {
  uint32_t at[Tile<DP>::DT][2];
  __device__ __forceinline__ void init(int l) {
    const int h = l >> 5, r = l & 15;
#pragma unroll
    for (int dt = 0; dt < Tile<DP>::DT; ++dt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = 4 * h + (r >> 2) + 8 * i;    // of k0's sixteen
        const int chunk = 4 * dt + 2 * ((l >> 4) & 1) + ((r & 3) >> 1);
        at[dt][i] = (row * Tile<DP>::NC + (chunk ^ swz<DP>(row))) * 16 + (r & 1) * 8;
      }
  }
  struct Base {
    uint32_t b[Tile<DP>::DT][2];
  };
  __device__ __forceinline__ Base base(uint32_t tile) const {
    Base x;
#pragma unroll
    for (int dt = 0; dt < Tile<DP>::DT; ++dt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x.b[dt][i] = tile + at[dt][i];
        asm("" : "+v"(x.b[dt][i]));
      }
    return x;
  }
  __device__ __forceinline__ static bf16x8 get(const Base& x, int k0, int dt) {
    typedef __attribute__((address_space(3))) char lds_char;
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(
          reinterpret_cast<lds_char*>(x.b[dt][i]) + k0 * Tile<DP>::NC * 16));
      const bf16* p = reinterpret_cast<const bf16*>(&a);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * i + e] = p[e];
    }
    return v;
  }
};
__device__ __forceinline__ f32x16 mfma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// row of an accumulator's element i
__device__ __forceinline__ int acc_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// Registers' operand of one row from memory, as B (or A) over the columns.
template <int DP> struct RowOp {
  bf16x8 f[Tile<DP>::KF];
};
template <int DP>
__device__ __forceinline__ void load_row(RowOp<DP>& R, const bf16* row, int d, int h) {
#pragma unroll
  for (int f = 0; f < Tile<DP>::KF; ++f) {
    const int col = 16 * f + 8 * h;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (col < d) v = *reinterpret_cast<const uint4*>(row + col);
    R.f[f] = *reinterpret_cast<bf16x8*>(&v);
  }
}

// Places of the three stages of a ring, bytes: of tile t + 1, t + 2 and t + 3 (which is t's).
// (t mod 3 in sight of the reads would be spread into their addresses: more registers than there
// are.)
struct Ring {
  uint32_t a, b, c;
  __device__ __forceinline__ void start(uint32_t bytes) {
    a = bytes;
    b = 2 * bytes;
    c = 0;
    asm("" : "+s"(a), "+s"(b), "+s"(c));
  }
  __device__ __forceinline__ void next() {
    const uint32_t x = a;
    a = b;
    b = c;
    c = x;
  }
};
// The larger of the values that lanes l and l ^ 32 hold, and their sum: one exchange of the
// halves of a wave in the vector unit.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The tiles of one tensor's rows in order, as buffers: what lies past a tensor's last row, and a
// place that no buffer has (kNowhere), are read as zeros, and a tile past the last as nothing else.
typedef __attribute__((ext_vector_type(4))) uint32_t buffer_t;
constexpr uint32_t kNowhere = 0x80000000u;
struct Feed {
  uint64_t base, step;   // the next tile's first row, and from tile to tile
  uint32_t tail;         // bytes of the last tile
  int left;              // tiles, from the next one to the last
  __device__ __forceinline__ void start(const bf16* X, int64_t ld, int first, int rows, int d) {
    base = (uint64_t)(X + 64 * first * ld);
    step = 128 * (uint64_t)ld;
    left = (rows + 63) / 64 - first;
    tail = (uint32_t)(2 * ((rows - 1) % 64 * ld + d));
  }
  __device__ __forceinline__ buffer_t next() {
    const buffer_t b = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffff,
                        left > 1 ? 0x7fffffffu : left == 1 ? tail : 0u, 0x00027000u};
    base += step;
    --left;
    return b;
  }
};

// Copies from a buffer into LDS (lane l's 16 bytes to `to` + 16 l), under way until wait_copies.
// An instruction of its own rather than the builtin: for the builtin's copies the compiler puts
// a wait before every transposing read, whose LDS it cannot tell from theirs.  It writes no
// register but m0, and reads its own as it is issued.  The compiler does not look into it for hazards:
// gfx9 wants five wait states between a vector instruction that writes a scalar register (a lane's
// read, as of a spilled one) and a memory instruction that reads it.  s_mov is one, s_nop 3 four.
__device__ __forceinline__ void copy16(uint32_t to, uint32_t off, const buffer_t& from) {
  uint32_t m0;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
               : "={m0}"(m0) : "s"(to), "v"(off), "s"(from));
}
__device__ __forceinline__ void copy4(uint32_t to, uint32_t off, const buffer_t& from) {
  uint32_t m0;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tbuffer_load_dword %2, %3, 0 offen lds"
               : "={m0}"(m0) : "s"(to), "v"(off), "s"(from));
}

// Wave w of NWV waves copies its share of a pair of tiles (x, then y): wave instruction j = w,
// NWV + w, ... of 2 NC, each 64 slots.  64 rows of a view are less than 2^31 bytes.
template <int DP, int NWV> struct PairCopy {
  static constexpr int NC = Tile<DP>::NC, N = 2 * NC / NWV;
  static_assert(2 * NC % NWV == 0, "whole instructions for every wave");
  uint32_t off[N];   // of the lane's slot in each, bytes from the tile's first row
  __device__ __forceinline__ static bool of_x(int i, int w) {
    if constexpr (NC % NWV == 0) return i < NC / NWV;
    else return i * NWV + w < NC;
  }
  __device__ __forceinline__ static int slot(int i, int w) {
    const int j = i * NWV + w;
    return (of_x(i, w) ? j : j - NC) * 64;
  }
  __device__ __forceinline__ void init(int w, int l, int64_t ld_x, int64_t ld_y, int d) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = slot(i, w) + l, row = s / NC, col = 8 * (s % NC ^ swz<DP>(row));
      off[i] = col < d ? 2 * (uint32_t)(row * (of_x(i, w) ? ld_x : ld_y) + col) : kNowhere;
    }
  }
  __device__ __forceinline__ void copy(int w, uint32_t x, uint32_t y, const buffer_t& from_x, const buffer_t& from_y) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      copy16((of_x(i, w) ? x : y) + 16 * slot(i, w), off[i], of_x(i, w) ? from_x : from_y);
  }
};

// Wait until at most n of the wave's memory operations are under way (s_waitcnt: vmcnt in bits
// 3:0 and 15:14; expcnt and lgkmcnt at their largest).
template <int n> __device__ __forceinline__ void wait_copies() {
  static_assert(n >= 0 && n < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (15 << 8) | (((n >> 4) & 3) << 14));
}
// The same, and until at most m of its LDS operations are.
template <int n, int m> __device__ __forceinline__ void wait_copies_and_writes() {
  static_assert(n >= 0 && n < 64 && m >= 0 && m < 16, "vmcnt, lgkmcnt");
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (m << 8) | (((n >> 4) & 3) << 14));
}
// A barrier that waits for nothing of the wave's own.
__device__ __forceinline__ void bare_barrier() { asm volatile("s_barrier" ::: "memory"); }
// A barrier that waits for the wave's LDS reads and writes, not for copies under way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
  asm volatile("s_barrier" ::: "memory");
}

// 2^x (v_exp_f32): results below the normal range become 0, which no bf16 weight notices.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ bf16x8 pack8(const f32x16& s, int j) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16)s[8 * j + e];
  return r;
}
// Order of a stretch of products whose operands come from LDS, the first of them read before: with
// each product the reads of one that is some reads later.  One wave of a SIMD reads at a time and a
// read takes a few hundred cycles, so the compiler's own order, a few reads ahead, left the
// matrix unit idle half of the time.
template <int N, int READS> __device__ __forceinline__ void order_step() {
  if constexpr (N > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);              // MFMA
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);   // LDS reads
    order_step<N - 1, READS>();
  }
}

template <int N> __device__ __forceinline__ bool finite16(const f32x16 (&acc)[N]) {
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) z = fmaf(acc[i][e], 0.f, z);
  return __all(z == 0.f);
}

// The block's sequence, first row and head; the key head is the fastest index: blocks go round
// the eight XCDs, so those that read the same keys share an L2.
struct AttnPlace {
  int q_row, q_len, k_row, k_len, r0, head_k, gq;
};
__device__ __forceinline__ AttnPlace attn_place(const CausalArgs& p, int per_head, int rows) {
  AttnPlace a;
  int b = blockIdx.x;
  a.head_k = b % p.heads_k;
  b /= p.heads_k;
  a.gq = b % per_head;
  b /= per_head;
  const uint32_t it = (uint32_t)p.pool.word[kAttnWords - 1 - b];
  const int32_t* s = p.pool.word + 4 * (it & 255);
  a.q_row = s[0];
  a.q_len = s[1];
  a.k_row = s[2];
  a.k_len = s[3];
  a.r0 = (int)(it >> 8) * rows;
  return a;
}
__device__ __forceinline__ const bf16* head_of(const AttnView& v, int head, int row) {
  return reinterpret_cast<const bf16*>(v.p) + v.head * head + v.row * row;
}
__device__ __forceinline__ bf16* out_of(const AttnView& v, int head, int row) {
  return const_cast<bf16*>(head_of(v, head, row));
}

// acc += the products of a cut tile of N rows pair by pair: weights w (elements as the
// accumulators' of its rows), `tile` the other operand's rows in LDS, seen(row) whether the pair
// counts.  A pair that does not has weight 0, but 0 times an infinity or a NaN would still reach
// a sum of products.  Only cut tiles hold such pairs, and only a result that is not finite can
// be touched: the kernels look at their results, and where one is not finite the block goes
// over its tiles again this way.
template <int DP, int N, class Seen>
__device__ __forceinline__ void add_pairs(f32x16 (&acc)[Tile<DP>::DT], const bf16x8 (&w)[N / 16],
                                          const uint4* tile, int l, Seen seen) {
  const int c = l & 31, h = l >> 5;
  const uint32_t* word = reinterpret_cast<const uint32_t*>(w);   // two weights each
#pragma nounroll
  for (int row = 0; row < N; ++row) {
    const int half = row >> 5, i = ((row & 31) >> 3) * 4 + (row & 3), src = (row >> 2) & 1;
    uint32_t pair = 0;
#pragma unroll
    for (int n = 0; n < N / 4; ++n) pair = n == 8 * half + (i >> 1) ? word[n] : pair;
    float x = __uint_as_float(i & 1 ? pair & 0xffff0000u : pair << 16);
    x = __shfl(x, c + 32 * src);
    const bool in = seen(row);
#pragma unroll
    for (int dt = 0; dt < Tile<DP>::DT; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q) {     // columns 32 dt + 8q + 4h ..
        const uint4* chunk = tile + row * Tile<DP>::NC + ((4 * dt + q) ^ swz<DP>(row));
        const bf16* y = reinterpret_cast<const bf16*>(chunk) + 4 * h;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[dt][4 * q + e] = in ? fmaf(x, (float)y[e], acc[dt][4 * q + e]) : acc[dt][4 * q + e];
        asm volatile("" ::: "memory");   // one read at a time: speed is not wanted, registers are
      }
  }
}

// Columns 32 dt .. 32 dt + 31 of row c of an output from an accumulator that holds them as rows,
// times f.
__device__ __forceinline__ void store_columns(bf16* row, const f32x16& acc, float f, int dt, int d, int h) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (32 * dt + 8 * i >= d) continue;
    bf16 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (bf16)(acc[4 * i + e] * f);
    *reinterpret_cast<uint2*>(row + 32 * dt + 8 * i + 4 * h) = *reinterpret_cast<uint2*>(x);
  }
}
template <int DP>
__device__ __forceinline__ void store_row(bf16* row, const f32x16 (&acc)[Tile<DP>::DT], float f, int d, int h) {
#pragma unroll
  for (int dt = 0; dt < Tile<DP>::DT; ++dt) store_columns(row, acc[dt], f, dt, d, h);
}
// Values 4 i .. 4 i + 3 of an accumulator.
__device__ __forceinline__ f32x4 f32x4_of(const f32x16& acc, int i) {
  return f32x4{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
}

}  // namespace mpipe
