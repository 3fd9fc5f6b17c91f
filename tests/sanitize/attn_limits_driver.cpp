// The largest sizes that the first LLM layer's attention takes, in its host-side arithmetic, under
// UndefinedBehaviorSanitizer.  Built and run by tests/test_attention_limits.py with g++.
#include <climits>
#include <cstdio>

#include "../../paper_2607_03229_amd/csrc/attn_plan.h"

using namespace mpipe;

namespace {

int failures = 0;
void expect(bool ok, const char* what, int64_t k) {
  if (!ok) {
    std::fprintf(stderr, "FAILED: %s (%lld)\n", what, (long long)k);
    ++failures;
  }
}

void check_units() {
  for (int64_t n : {int64_t(0), int64_t(1), int64_t(127), int64_t(128), int64_t(129), int64_t(65536),
                    INT32_MAX - int64_t(256), INT32_MAX - int64_t(128), INT32_MAX - int64_t(127),
                    INT32_MAX - int64_t(1), int64_t(INT32_MAX)}) {
    const int64_t want = (n + kCacheUnit - 1) / kCacheUnit;
    expect(cache_units((int)n) == want, "units of tokens", n);
    // a place in the last unit's last quarter is still below 2^31
    if (n) expect((want - 1) * kCacheUnit + 3 * kCacheUnit / 4 <= INT32_MAX, "the last unit's waves", n);
  }
}

// A grid's threads stay below 2^32 whatever an item's blocks, in launches as full as that allows.
void check_launches() {
  for (int64_t blocks : {int64_t(1), int64_t(28), int64_t(512), int64_t(65535), int64_t(65536), int64_t(8) * 65536}) {
    const int64_t items = attn_launch_items(blocks);
    expect(items >= 1, "an item", blocks);
    expect(items * blocks * kAttnThreads < int64_t(1) << 32, "threads of a grid", blocks);
    expect((items + 1) * blocks * kAttnThreads >= int64_t(1) << 32, "a full grid", blocks);
  }
}

}  // namespace

int main() {
  check_units();
  check_launches();
  if (failures) return 1;
  std::printf("attention limits passed\n");
  return 0;
}
