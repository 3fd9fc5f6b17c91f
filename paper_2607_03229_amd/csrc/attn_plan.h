// Host-only planning of the first LLM layer's attention (mpipe_ops.h): sequence checks, work
// items, and the checks of a paged cache's arguments.  No HIP: the sanitizer tests build it
// with g++.
#pragma once
#include <cstdint>
#include <string>
#include <vector>

#include "layer_plan.h"

namespace mpipe {

// ---- causal attention ---------------------------------------------------------------------
// One sequence: its rows in the tensors of q and of k; query i sees keys 0 .. i + k_len - q_len.
struct AttnSeq {
  int32_t q_row, q_len, k_row, k_len;
};
// The sequences, checked: inside the tensors, queries apart; `keys_apart` (a backward): no key
// row in two sequences.  key_row / key_len null: the queries' own rows.
mpipe_status attn_sequences(const int64_t* seq_row, const int64_t* seq_len, const int64_t* key_row,
                            const int64_t* key_len, int32_t n_seq, int64_t rows_q, int64_t rows_k,
                            bool keys_apart, std::vector<AttnSeq>& seqs, std::string& why);

// A work item: a tile of rows (queries, or keys) of one sequence.
struct AttnItem {
  int32_t seq, tile;
};
// Items of `rows` query (by_keys: key) rows each, the longest walks over the other side first, so
// that what starts last ends soon.
void attn_items(const std::vector<AttnSeq>& seqs, bool by_keys, int rows,
                std::vector<AttnItem>& items);

// Items of `blocks` blocks each to a launch, at least one (heads end at 65536): a grid has fewer than
// 2^32 threads, and a block of causal attention at most kAttnThreads of them.
constexpr int kAttnThreads = 512;
constexpr int64_t attn_launch_items(int64_t blocks) {
  return ((int64_t(1) << 32) / kAttnThreads - 1) / blocks;
}

// What one launch carries in its arguments: sequences from the front (four words each), items
// from the back (a word: sequence in 8 bits, tile in 24).
constexpr int kAttnWords = 900;
struct AttnPool {
  int32_t word[kAttnWords];
};
// Fills `pool` with items [at, ...) and returns how many it holds (at most `most`).
int attn_pack(const std::vector<AttnSeq>& seqs, const std::vector<AttnItem>& items, size_t at,
              int64_t most, AttnPool& pool);

// ---- paged cache --------------------------------------------------------------------------
// Tokens of a page are a power of two of at most 2^16; a pool has at most 2^31 - 1 pages.
mpipe_status cache_ok(const mpipe_kv_cache* c, std::string& why);
// Whether a range shares a byte with the cache's pages or scales.
bool cache_meets(const mpipe_kv_cache& c, const void* p, size_t bytes);
bool cache_meets(const mpipe_kv_cache& c, const HeadView& v, int64_t rows, int esz);
int64_t cache_page_values(const mpipe_kv_cache& c);   // of k or v, in one page
// The attention over a cache takes a sequence's tokens in units; its units, of 0 .. 2^31 - 1 tokens.
constexpr int kCacheUnit = 128;
constexpr int cache_units(int tokens) {
  return (int)(((uint32_t)tokens + kCacheUnit - 1) / kCacheUnit);
}

}  // namespace mpipe
