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

}  // namespace

int main() {
  check_ranges();
  if (failures) return 1;
  std::puts("memory checks passed");
  return 0;
}
