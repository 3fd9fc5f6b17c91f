// Ranges and views of the operators around the first LLM layer against sets of their elements,
// under AddressSanitizer and UndefinedBehaviorSanitizer.  Built and run by
// tests/test_layer_memory_sanitize.py with g++.
#include <climits>
#include <cstdio>
#include <set>

#include "../../paper_2607_03229_amd/csrc/layer_plan.h"

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

std::set<uintptr_t> elements(const HeadView& v, int64_t rows, int d, int esz) {
  std::set<uintptr_t> at;
  for (int64_t r = 0; r < rows; ++r)
    for (int h = 0; h < v.heads; ++h)
      for (int c = 0; c < d; ++c)
        for (int b = 0; b < esz; ++b)
          at.insert((uintptr_t)v.p + (uintptr_t)((r * v.row + h * v.head + c) * esz + b));
  return at;
}

void check_ranges() {
  int meet = 0;
  for (int k = 0; k < 20000; ++k) {
    const int d = 8, esz = 2, rows = uniform(0, 5);
    HeadView v;
    v.heads = uniform(0, 4);
    v.head = uniform(0, 1) ? 8 : uniform(0, 60);
    v.row = uniform(0, 1) ? 40 : uniform(0, 200);
    v.p = (const void*)(uintptr_t)(4096 + 2 * uniform(0, 60));
    const uintptr_t lo = 3800 + uniform(0, 2400);
    const size_t bytes = uniform(0, 3) ? uniform(0, 40) : uniform(0, 2000);
    bool share = false;
    for (uintptr_t e : elements(v, rows, d, esz)) share |= e >= lo && e < lo + bytes;
    expect(range_meets((const void*)lo, bytes, v, rows, d, esz) == share, "a range and a view", k);
    meet += share;
  }
  std::printf("%d of 20000 ranges meet\n", meet);
  expect(meet > 1000 && meet < 19000, "both kinds of ranges", 0);
  // strides over one row or one head may be anything
  HeadView v;
  v.p = (const void*)4096;
  v.heads = 1;
  v.head = v.row = INT64_MAX;
  expect(range_meets((const void*)4100, 4, v, 1, 8, 2), "one head of one row", 0);
  expect(!range_meets((const void*)4112, 4, v, 1, 8, 2), "behind one head of one row", 0);
}

// Views of one product in any order of rows, heads and q | k | v: exactly; any others: never
// apart where they meet.
void check_views() {
  int said_apart = 0, meet = 0, close = 0;
  for (int k = 0; k < 40000; ++k) {
    const int d = 8, esz = 2, rows = uniform(1, 6);
    const bool one_row = uniform(0, 3) > 0, one_head = uniform(0, 3) > 0;
    HeadView v[2];
    for (int z = 0; z < 2; ++z) {
      v[z].heads = uniform(1, 4);
      v[z].row = z && one_row ? v[0].row : uniform(0, 1) ? 8 * uniform(1, 20) : uniform(0, 120);
      v[z].head = z && one_head ? v[0].head : uniform(0, 1) ? 8 * uniform(1, 20) : uniform(0, 120);
      v[z].p = (const void*)(uintptr_t)(4096 + (uniform(0, 1) ? 16 * uniform(0, 20) : 2 * uniform(0, 160)));
    }
    const std::set<uintptr_t> a = elements(v[0], rows, d, esz), b = elements(v[1], rows, d, esz);
    bool share = false;
    for (uintptr_t e : a) share |= b.count(e) > 0;
    const bool said = views_meet(v[0], v[1], rows, d, esz);
    expect(said == views_meet(v[1], v[0], rows, d, esz), "either way round", k);
    expect(said || !share, "views that meet", k);
    const bool row = rows == 1 || v[0].row == v[1].row,
               head = v[0].heads == 1 || v[1].heads == 1 || v[0].head == v[1].head;
    if (row && head) expect(said == share, "views of one product", k);
    said_apart += !said;
    meet += share;
    close += !said && *a.begin() < *b.rbegin() && *b.begin() < *a.rbegin();
  }
  std::printf("%d of 40000 pairs meet, %d said apart, %d of them within each other\n", meet, said_apart, close);
  expect(meet > 4000 && said_apart > 4000 && close > 1000, "every kind of views", 0);
  // [rows][heads][q | k | v][d], and [heads][rows][q | k | v][d]
  for (int order = 0; order < 2; ++order)
    for (int z = 0; z < 9; ++z) {
      const HeadView a = {(const void*)(uintptr_t)(4096 + 256 * (z / 3)), order ? 384 : 32 * 384,
                          order ? 1000 * 384 : 384, 32},
                     b = {(const void*)(uintptr_t)(4096 + 256 * (z % 3)), a.row, a.head, 32};
      expect(views_meet(a, b, 1000, 128, 2) == (z / 3 == z % 3), "q, k and v head by head", z);
    }
  // q, k, q, v of groups of two heads: strides of 2 d and 4 d; k reaches into a row's last q
  const HeadView q = {(const void*)4096, 2048, 256, 8}, k = {(const void*)(4096 + 256), 2048, 512, 4},
                 over = {(const void*)(4096 + 260), 2048, 512, 4};
  expect(!views_meet(q, k, 100, 128, 2) && views_meet(q, over, 100, 128, 2), "groups", 0);
  // strides over one row or one head may be anything
  HeadView w = {(const void*)4096, INT64_MAX, INT64_MAX, 1};
  expect(views_meet(w, w, 1, 8, 2), "one head of one row", 0);
}

}  // namespace

int main() {
  check_ranges();
  check_views();
  if (failures) return 1;
  std::puts("memory checks passed");
  return 0;
}
