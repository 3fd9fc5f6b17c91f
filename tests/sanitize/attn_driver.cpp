// The host planning of the first LLM layer's attention under AddressSanitizer and
// UndefinedBehaviorSanitizer: sequence checks, work items against a plain count, their packing
// into launches, and a cache's checks, on valid and invalid inputs from a fixed-seed generator.
// Built and run by tests/test_attention_sanitize.py with g++.
#include <algorithm>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <memory>
#include <set>

#include "../../paper_2607_03229_amd/csrc/attn_plan.h"

using namespace mpipe;

namespace {

uint64_t g_state = 0x9E3779B97F4A7C15ull;
uint32_t next_u32() {   // xorshift64*
  g_state ^= g_state >> 12;
  g_state ^= g_state << 25;
  g_state ^= g_state >> 27;
  return (uint32_t)((g_state * 0x2545F4914F6CDD1Dull) >> 32);
}
int uniform(int lo, int hi) { return lo + (int)(next_u32() % (uint32_t)(hi - lo + 1)); }

int failures = 0;
void expect(bool ok, const char* what, int k) {
  if (!ok) {
    std::fprintf(stderr, "FAILED: %s (case %d)\n", what, k);
    ++failures;
  }
}

void check_sequences() {
  for (int k = 0; k < 600; ++k) {
    const int n = uniform(0, 12);
    const int64_t rq = uniform(0, 60), rk = uniform(0, 60);
    std::vector<int64_t> a, la, b, lb;
    for (int s = 0; s < n; ++s) {
      a.push_back(uniform(-1, 60));
      la.push_back(uniform(-1, 12));
      b.push_back(uniform(0, 60));
      lb.push_back(uniform(0, 20));
    }
    const bool own = uniform(0, 1), apart = uniform(0, 1);
    bool ok = true;
    std::map<int64_t, int> of_q, of_k;
    for (int s = 0; s < n; ++s) {
      const int64_t kr = own ? a[s] : b[s], kl = own ? la[s] : lb[s];
      ok = ok && la[s] >= 0 && kl >= 0 && a[s] >= 0 && a[s] + la[s] <= rq && kr >= 0 && kr + kl <= rk;
      for (int64_t i = 0; i < la[s]; ++i) ++of_q[a[s] + i];
      for (int64_t i = 0; i < kl; ++i) ++of_k[kr + i];
    }
    for (auto& x : of_q) ok = ok && x.second == 1;
    if (apart)
      for (auto& x : of_k) ok = ok && x.second == 1;
    std::vector<AttnSeq> seqs;
    std::string why;
    const mpipe_status st = attn_sequences(a.data(), la.data(), own ? nullptr : b.data(),
                                           own ? nullptr : lb.data(), n, rq, rk, apart, seqs, why);
    expect((st == MPIPE_OK) == ok, "sequences", k);
    if (st != MPIPE_OK) {
      expect(!why.empty(), "a reason", k);
      continue;
    }
    expect((int)seqs.size() == n, "number of sequences", k);
  }
  std::vector<AttnSeq> seqs;
  std::string why;
  const int64_t big[1] = {INT64_MAX}, one[1] = {1}, zero[1] = {0};
  expect(attn_sequences(big, one, nullptr, nullptr, 1, 8, 8, true, seqs, why) != MPIPE_OK, "a far row", 0);
  expect(attn_sequences(one, big, nullptr, nullptr, 1, 8, 8, true, seqs, why) != MPIPE_OK, "a long one", 0);
  expect(attn_sequences(zero, one, big, big, 1, 8, 8, true, seqs, why) != MPIPE_OK, "far keys", 0);
  expect(attn_sequences(zero, one, one, nullptr, 1, 8, 8, true, seqs, why) != MPIPE_OK, "half of the keys", 0);
  expect(attn_sequences(nullptr, nullptr, nullptr, nullptr, -1, 8, 8, true, seqs, why) != MPIPE_OK, "a negative count", 0);
  expect(attn_sequences(nullptr, nullptr, nullptr, nullptr, 1, 8, 8, true, seqs, why) != MPIPE_OK, "no lists", 0);
}

// Every tile of every sequence once, the longest walks first, whatever a launch holds.
void check_items() {
  for (int k = 0; k < 60; ++k) {
    const int n = k == 0 ? 0 : uniform(1, k % 3 ? 40 : 1200), rows = 64 << uniform(0, 2);
    const bool by_keys = uniform(0, 1);
    std::vector<AttnSeq> seqs;
    std::set<std::pair<int, int>> want;
    for (int s = 0; s < n; ++s) {
      const AttnSeq x = {s, uniform(0, 900), s, uniform(0, 900)};
      seqs.push_back(x);
      for (int t = 0; t * rows < (by_keys ? x.k_len : x.q_len); ++t) want.insert({s, t});
    }
    std::vector<AttnItem> items;
    attn_items(seqs, by_keys, rows, items);
    std::set<std::pair<int, int>> got;
    int64_t before = INT64_MAX;
    for (const AttnItem& it : items) {
      expect(got.insert({it.seq, it.tile}).second, "an item twice", k);
      const AttnSeq& x = seqs[it.seq];
      const int64_t walk = by_keys ? std::min<int64_t>(x.q_len, x.k_len - it.tile * rows)
                                   : std::min<int64_t>(x.k_len, (it.tile + 1) * rows + x.k_len - x.q_len);
      expect(walk <= before, "order of items", k);
      before = walk;
    }
    expect(got == want, "all items", k);
    auto pool = std::make_unique<AttnPool>();
    const int64_t most = k % 2 ? 1 << 20 : uniform(1, 300);
    size_t at = 0;
    while (at < items.size()) {
      const int m = attn_pack(seqs, items, at, most, *pool);
      expect(m > 0 && m <= most && at + m <= items.size(), "a launch's items", k);
      if (m <= 0) break;
      for (int i = 0; i < m; ++i) {
        const uint32_t word = (uint32_t)pool->word[kAttnWords - 1 - i];
        const int32_t* s = pool->word + 4 * (word & 255);
        expect(s + 4 <= pool->word + kAttnWords - m, "sequences below the items", k);
        const AttnSeq& x = seqs[items[at + i].seq];
        expect((int)(word >> 8) == items[at + i].tile && s[0] == x.q_row && s[1] == x.q_len &&
                   s[2] == x.k_row && s[3] == x.k_len, "a packed item", k);
      }
      at += m;
    }
  }
  // the last tile of the longest sequence, and a query tile without keys
  std::vector<AttnSeq> seqs = {{0, 1 << 30, 0, 64}};
  std::vector<AttnItem> one = {{0, (1 << 24) - 1}};
  auto pool = std::make_unique<AttnPool>();
  expect(attn_pack(seqs, one, 0, 1, *pool) == 1, "a far tile", 0);
  expect((uint32_t)pool->word[kAttnWords - 1] >> 8 == (1u << 24) - 1, "a far tile's word", 0);
}

void check_cache() {
  alignas(16) static char k[4096], v[4096];
  static uint8_t ks[64], vs[64];
  std::string why;
  auto make = [&](int32_t dtype) {
    mpipe_kv_cache c = {k, v, nullptr, nullptr, 2, 2, 4, 16, dtype};   // 256 values each
    if (dtype == MPIPE_E4M3) c.k_scale = ks, c.v_scale = vs;
    return c;
  };
  for (int32_t dtype : std::vector<int32_t>{MPIPE_F32, MPIPE_BF16, MPIPE_E4M3}) {
    const mpipe_kv_cache good = make(dtype);
    expect(cache_ok(&good, why) == MPIPE_OK, "a cache", dtype);
    const int esz = dtype == MPIPE_F32 ? 4 : dtype == MPIPE_BF16 ? 2 : 1;
    expect(cache_meets(good, k + 256 * esz - 1, 1), "the last byte", dtype);
    expect(!cache_meets(good, k + 256 * esz, 1), "past the last byte", dtype);
    expect(cache_meets(good, ks, 1) == (dtype == MPIPE_E4M3), "scales", dtype);
    HeadView view;
    view.p = k + 256 * esz;
    view.row = 32;
    view.head = 16;
    view.heads = 2;
    expect(!cache_meets(good, view, 1, 2), "rows behind", dtype);
    view.p = k;
    expect(cache_meets(good, view, 1, 2), "rows in it", dtype);
    for (int i = 0; i < 13; ++i) {
      mpipe_kv_cache c = good;
      switch (i) {
        case 0: c.page = 3; break;
        case 1: c.page = 0; break;
        case 2: c.page = 1 << 17; break;
        case 3: c.head_dim = 12; break;
        case 4: c.head_dim = 264; break;
        case 5: c.heads = 0; break;
        case 6: c.heads = 65537; break;
        case 7: c.n_pages = -1; break;
        case 8: c.n_pages = INT64_MAX; break;
        case 9: c.k = k + 8; break;
        case 10: c.v = nullptr; break;
        case 11: c.v = k; break;
        default: c.k_scale = dtype == MPIPE_E4M3 ? nullptr : ks; break;
      }
      expect(cache_ok(&c, why) != MPIPE_OK, "a bad cache", 100 * dtype + i);
    }
    mpipe_kv_cache c = good;   // sizes whose product does not fit 64 bits
    c.n_pages = INT32_MAX;
    c.heads = 65536;
    c.page = 1 << 16;
    c.head_dim = 256;
    expect(cache_ok(&c, why) != MPIPE_OK, "a product past 64 bits", dtype);
    c.n_pages = 0;
    expect(cache_ok(&c, why) == MPIPE_OK, "no pages", dtype);
  }
  expect(cache_ok(nullptr, why) != MPIPE_OK, "no cache", 0);
}

}  // namespace

int main() {
  check_sequences();
  check_items();
  check_cache();
  if (failures) return 1;
  std::printf("attention checks passed\n");
  return 0;
}
