// Causal attention with grouped heads over sequences (mpipe_op_causal_attention_fwd / _bwd):
// the launches.
#include <algorithm>
#include <initializer_list>

#include "attn_kernels.h"
#include "common.h"

namespace mpipe {
namespace {

AttnView view(const HeadView& v) { return {v.p, v.row, v.head}; }

// Waves of a block of fwd and dq.  A width of 96 at most: see causal_q_waves.  At 128 a CU has one
// block of either kind, so four waves pay only where even blocks of eight leave most CUs idle.
// Measured on MI355X, us of forward and dQ, one sequence, 28/4 heads of 128, 8 -> 4 waves: 256 rows
// (28 blocks) 17 -> 15 and 23 -> 18; 512 rows 22 -> 21 and 31 -> 26; 1024 rows (112 blocks) 34 -> 35
// and 45 -> 41; 2048 rows 59 -> 70 and 79 -> 85.
constexpr int64_t kFewBlocks = 64;
int q_waves(const CausalProblem& p) {
  const int most = causal_q_waves(causal_width(p.head_dim));
  if (most == 4) return 4;
  int64_t blocks = 0;
  for (const AttnSeq& q : p.seqs) blocks += (q.q_len + 255) / 256 * p.q.heads;
  return blocks > kFewBlocks ? most : 4;
}

CausalArgs args_of(const CausalProblem& p) {
  CausalArgs a;
  a.q = view(p.q);
  a.k = view(p.k);
  a.v = view(p.v);
  a.o = view(p.o);
  a.d_o = view(p.d_o);
  a.dq = view(p.dq);
  a.dk = view(p.dk);
  a.dv = view(p.dv);
  a.lse = p.lse;
  a.ld_lse = p.ld_lse;
  a.delta = p.scratch;
  a.partial = nullptr;
  a.parts = 1;
  a.sub = 1;
  a.q_waves = q_waves(p);
  a.rows_q = p.rows_q;
  a.scale = p.scale;
  a.d = p.head_dim;
  a.heads_k = p.k.heads;
  a.group = p.q.heads / p.k.heads;
  return a;
}

// Blocks of dK and dV in parts, at most, and query tiles of a part, at least: few key tiles (single
// or short sequences, few key heads) leave CUs without one, so the queries of a key tile, of all
// heads of its group, are cut and the parts' sums joined.  Measured on MI355X, us of a whole
// backward without parts, with 256, 512 and 1024 blocks, one sequence, 28/4 heads of 128: 1024
// rows 194, 85, 91, 120; 4096 rows 734, 516, 440, 460; 8192 rows 1866, 1862, 1494, 1506.  Two to
// twelve tiles: within 10 %.
constexpr int64_t kSplitBlocks = 512, kPartTiles = 4;
int64_t split_blocks(int64_t rows_q, int heads_q, int64_t rows_k, int heads_k, int d) {
  if (heads_k == 0 || d > 128) return 0;
  const int rows = 16 * causal_k_waves(causal_width(d));
  const int64_t parts = (rows_q + 63) / 64 * (heads_q / heads_k) / kPartTiles;
  const int64_t tiles = (rows_k + rows - 1) / rows * heads_k;
  return parts < 2 || tiles > kSplitBlocks / 2 ? 0 : std::min(kSplitBlocks, parts * tiles);
}
// The same for the general kernels, whose tiles have 16 rows and whose four waves cut a part again.
// Without parts, with 1024, 2048 and 4096 blocks, fp32, one sequence of 2048: 8/1 heads of 64 686,
// 255, 248, 275; 16/1 of 128 2626, 1032, 1066, 1153; four of 500, 28/4 of 128 586, 599, 615, 681.
constexpr int64_t kGeneralSplit = 1024, kGeneralPartTiles = 16;
int64_t general_split_blocks(int64_t rows_q, int heads_q, int64_t rows_k, int heads_k) {
  if (heads_k == 0) return 0;
  const int64_t parts = (rows_q + 15) / 16 * (heads_q / heads_k) / kGeneralPartTiles;
  const int64_t tiles = (rows_k + 15) / 16 * heads_k;
  return parts < 2 || tiles > kGeneralSplit / 2 ? 0 : std::min(kGeneralSplit, parts * tiles);
}
// Parts of every key tile, so that they are `blocks` in all, of `least` query tiles at least.
int parts_of(const CausalProblem& p, int key_rows, int query_rows, int64_t blocks, int64_t least) {
  int64_t tiles = 0, longest = 0;
  for (const AttnSeq& q : p.seqs) {
    tiles += (q.k_len + key_rows - 1) / key_rows * (int64_t)p.k.heads;
    longest = std::max<int64_t>(longest, (q.q_len + query_rows - 1) / query_rows * (int64_t)(p.q.heads / p.k.heads));
  }
  return tiles == 0 ? 1 : (int)std::max<int64_t>(1, std::min(blocks / tiles, longest / least));
}
int64_t delta_bytes(int64_t rows_q, int heads_q) { return (rows_q * heads_q * 8 + 31) / 16 * 16; }

// Blocks of 16 rows to an item of the general kernels: eight, so that a launch's arguments hold long
// sequences, or as many as the longest has (223 fp32 sequences of 10 rows, 12/4 heads of 48, forward
// and backward: 254 us with eight, 95 with one).
int general_sub(const CausalProblem& p, bool by_keys) {
  int longest = 0;
  for (const AttnSeq& q : p.seqs) longest = std::max(longest, by_keys ? q.k_len : q.q_len);
  return std::max(1, std::min(8, (longest + 15) / 16));
}

// All items, as many to a launch as its arguments and its grid hold.
template <class Launch>
hipError_t in_pieces(const CausalProblem& p, CausalArgs& a, bool by_keys, int rows,
                     int64_t blocks_per_item, Launch one) {
  std::vector<AttnItem> items;
  attn_items(p.seqs, by_keys, rows, items);
  const int64_t most = attn_launch_items(blocks_per_item);
  for (size_t at = 0; at < items.size();) {
    const int n = attn_pack(p.seqs, items, at, most, a.pool);
    if (hipError_t e = one(a, n)) return e;
    at += n;
  }
  return hipSuccess;
}

// Whether the bf16 kernels can read and write these views: 16-byte pieces at 16-byte places, and a
// tile's 64 rows less than 2^31 bytes apart.
bool tiled(const CausalProblem& p, std::initializer_list<const HeadView*> views) {
  if (p.dtype != DT_BF16 || p.head_dim > 128) return false;
  for (const HeadView* v : views)
    if ((uintptr_t)v->p % 16 || v->row % 8 || v->head % 8 || v->row > (1 << 23)) return false;
  return true;
}

}  // namespace

hipError_t causal_attention_fwd(const CausalProblem& p, hipStream_t s) {
  CausalArgs a = args_of(p);
  if (tiled(p, {&p.q, &p.k, &p.v, &p.o})) {
    return in_pieces(p, a, false, 32 * a.q_waves, p.q.heads, [&](const CausalArgs& b, int n) {
      return causal_bf16_fwd(b, n, s);
    });
  }
  a.sub = general_sub(p, false);
  return in_pieces(p, a, false, 16 * a.sub, a.sub * p.q.heads, [&](const CausalArgs& b, int n) {
    return causal_general_fwd(p.dtype, b, n, s);
  });
}

size_t causal_attention_scratch(int64_t rows_q, int heads_q, int64_t rows_k, int heads_k,
                                int head_dim) {
  const int width = causal_width(head_dim);
  const int64_t tiled = split_blocks(rows_q, heads_q, rows_k, heads_k, head_dim) * 16 * causal_k_waves(width);
  const int64_t general = general_split_blocks(rows_q, heads_q, rows_k, heads_k) * 16;
  return (size_t)(delta_bytes(rows_q, heads_q) + std::max(tiled, general) * 2 * width * 4);
}

hipError_t causal_attention_bwd(const CausalProblem& p, hipStream_t s) {
  CausalArgs a = args_of(p);
  a.partial = p.scratch + delta_bytes(p.rows_q, p.q.heads) / 4;
  if (tiled(p, {&p.q, &p.k, &p.v, &p.o, &p.d_o, &p.dq, &p.dk, &p.dv})) {
    const int width = causal_width(p.head_dim);
    if (hipError_t e = in_pieces(p, a, false, 32 * a.q_waves, p.q.heads,
                                 [&](const CausalArgs& b, int n) { return causal_bf16_dq(b, n, s); }))
      return e;
    const int rows = 16 * causal_k_waves(width);
    a.parts = parts_of(p, rows, 64, split_blocks(p.rows_q, p.q.heads, p.rows_k, p.k.heads, p.head_dim), kPartTiles);
    return in_pieces(p, a, true, rows, p.k.heads * a.parts,
                     [&](const CausalArgs& b, int n) { return causal_bf16_dkdv(b, n, s); });
  }
  a.sub = general_sub(p, false);
  if (hipError_t e = in_pieces(p, a, false, 16 * a.sub, a.sub * p.q.heads, [&](const CausalArgs& b, int n) {
        return causal_general_dq(p.dtype, b, n, s);
      }))
    return e;
  a.sub = general_sub(p, true);
  a.parts = parts_of(p, 16 * a.sub, 16, general_split_blocks(p.rows_q, p.q.heads, p.rows_k, p.k.heads) / a.sub,
                     kGeneralPartTiles);
  return in_pieces(p, a, true, 16 * a.sub, a.sub * p.k.heads * a.parts, [&](const CausalArgs& b, int n) {
    return causal_general_dkdv(p.dtype, b, n, s);
  });
}

}  // namespace mpipe
