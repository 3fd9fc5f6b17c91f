// Launch interface of the first LLM layer's attention (causal_attention.hip,
// causal_general.hip, cache_attention.hip, kv_cache.hip); arguments are checked by attn_ops.cpp.
#pragma once
#include <hip/hip_runtime.h>

#include "attn_plan.h"
#include "internal.h"

namespace mpipe {

struct CausalProblem {
  int dtype = 0, head_dim = 0;
  int64_t rows_q = 0, rows_k = 0;
  HeadView q, k, v, o, d_o, dq, dk, dv;
  float* lse = nullptr;
  int64_t ld_lse = 0;
  float* scratch = nullptr;
  float scale = 0.f;
  std::vector<AttnSeq> seqs;
};
hipError_t causal_attention_fwd(const CausalProblem& p, hipStream_t s);
hipError_t causal_attention_bwd(const CausalProblem& p, hipStream_t s);
size_t causal_attention_scratch(int64_t rows_q, int heads_q, int64_t rows_k, int heads_k,
                                int head_dim);

// What a kernel of causal attention takes; all of it stays below 4 KB.
struct AttnView {
  const void* p;
  int64_t row, head;
};
struct CausalArgs {
  AttnPool pool;
  AttnView q, k, v, o, d_o, dq, dk, dv;
  float* lse;
  float* delta;   // backward: [2][heads][rows_q] of what one kernel leaves to the next
  float* partial;   // dkdv in parts: [blocks][2][width][keys of a block] as the lanes hold them
  int64_t ld_lse, rows_q;
  float scale;
  int d, heads_k, group;
  int sub;       // 16-row blocks of an item, causal_general.hip
  int q_waves;   // of a block of 32 queries each, fwd and dq
  int parts;     // parts: blocks that share a key tile's queries, of dkdv
};
static_assert(sizeof(CausalArgs) <= 4000, "a launch's arguments");
// Any dtype, alignment and head_dim of at most 256 (causal_general.hip): items of 16 * sub rows.
hipError_t causal_general_fwd(int dtype, const CausalArgs& a, int items, hipStream_t s);
hipError_t causal_general_dq(int dtype, const CausalArgs& a, int items, hipStream_t s);
hipError_t causal_general_dkdv(int dtype, const CausalArgs& a, int items, hipStream_t s);

// bf16, 16-byte aligned views, head_dim of at most 128 (causal_fwd.hip, causal_bwd.hip): items of 32
// queries a wave, and for dkdv of 16 keys a wave.  dq writes to
// `delta` what dkdv reads of each query.
hipError_t causal_bf16_fwd(const CausalArgs& a, int items, hipStream_t s);
hipError_t causal_bf16_dq(const CausalArgs& a, int items, hipStream_t s);
hipError_t causal_bf16_dkdv(const CausalArgs& a, int items, hipStream_t s);
// The width a head is padded to in the tiles.
constexpr int causal_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : 256; }
// Waves of a block: four where the tiles' LDS lets two blocks share a CU (one's start and end then
// meet the other's work, and half as many rows pad a sequence's last block), else eight, whose
// two halves share the SIMDs.  Measured on MI355X, us with 8 -> 4 waves: forward, four sequences
// of 8192, 8 heads of 64: 357 -> 309; 64 of 200, 16 heads of 80: 62 -> 53; 32 of 1024, 28/4 heads
// of 128 (one block of either): 390 -> 585.  dK and dV (with dQ): 1158 -> 1096 at 64, 188 -> 232 at
// 80, 1149 -> 1300 at 128.
constexpr int causal_q_waves(int width) { return width <= 96 ? 4 : 8; }
constexpr int causal_k_waves(int width) { return width <= 64 ? 4 : 8; }

struct CacheRows {   // rows on their way into or out of a cache
  mpipe_kv_cache cache;
  int dtype = 0;
  int64_t rows = 0;
  HeadView k, v;
  const int32_t* table = nullptr;
  int64_t ld_table = 0;
  int32_t n_seq = 0, width = 0;
  const int32_t* seq = nullptr;
  const int32_t* pos = nullptr;
  int32_t* status = nullptr;
};
hipError_t cache_write(const CacheRows& p, hipStream_t s);
hipError_t cache_read(const CacheRows& p, hipStream_t s);

struct CacheAttention {
  mpipe_kv_cache cache;
  int dtype = 0;
  int32_t n_seq = 0, width = 0;
  HeadView q, o;
  const int32_t* table = nullptr;
  int64_t ld_table = 0;
  const int32_t* lens = nullptr;
  float scale = 0.f;
  float* lse = nullptr;
  int64_t ld_lse = 0;
  float* scratch = nullptr;
};
hipError_t cache_attention(const CacheAttention& p, hipStream_t s);
size_t cache_attention_scratch(int n_seq, int head_dim);

}  // namespace mpipe
