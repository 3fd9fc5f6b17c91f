// The host planning of the operators around the first LLM layer under AddressSanitizer and
// UndefinedBehaviorSanitizer: position spans against a plain walk over the rows, rotary
// tables, views that meet against every element, gradient lists, on valid and invalid inputs
// from a fixed-seed generator.  Built and run by tests/test_layer_sanitize.py with g++.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <limits>
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

void check_positions() {
  for (int k = 0; k < 400; ++k) {
    std::vector<int64_t> sr, sl, sp, ir;
    std::vector<int32_t> g, st;
    int64_t row = 0;
    const int n_seq = uniform(0, 5);
    for (int s = 0; s < n_seq; ++s) {
      row += uniform(0, 9);
      const int64_t len = uniform(0, 120);
      sr.push_back(row);
      sl.push_back(len);
      sp.push_back(uniform(0, 50));
      int64_t at = row + uniform(0, 5);
      while (uniform(0, 3)) {
        const int t = uniform(1, 3), h = uniform(1, 4), w = uniform(1, 4);
        if (at + t * h * w > row + len) break;
        ir.push_back(at);
        g.insert(g.end(), {t, 2 * h, 2 * w});
        st.push_back(uniform(0, 3));
        at += t * h * w + uniform(0, 4);
      }
      row += len;
    }
    const int64_t n_rows = row + uniform(0, 9);
    // a shuffled order of sequences and items
    for (size_t i = sr.size(); i > 1; --i) {
      const size_t j = next_u32() % i;
      std::swap(sr[i - 1], sr[j]);
      std::swap(sl[i - 1], sl[j]);
      std::swap(sp[i - 1], sp[j]);
    }
    std::vector<PosSpan> spans;
    std::vector<int64_t> next(n_seq, -1);
    std::string why;
    int64_t end = 0;
    const mpipe_status st_ = position_spans(sr.data(), sl.data(), sp.data(), n_seq, ir.data(),
                                            g.data(), st.data(), (int32_t)ir.size(), n_rows,
                                            next.data(), spans, end, why);
    expect(st_ == MPIPE_OK, "valid positions", k);
    // the spans, expanded
    std::vector<int64_t> got(3 * n_rows, -1), want(3 * n_rows, -1);
    for (size_t i = 0; i < spans.size(); ++i) {
      const PosSpan& s = spans[i];
      const int64_t stop = i + 1 < spans.size() ? spans[i + 1].row : end;
      expect(stop > s.row && stop <= n_rows, "spans in order", k);
      for (int64_t r = s.row; r < stop && s.w >= 0; ++r) {
        const int64_t q = r - s.row;
        got[3 * r] = s.pos + (s.w ? q / s.hw * s.step : q);
        got[3 * r + 1] = s.pos + (s.w ? q % s.hw / s.w : q);
        got[3 * r + 2] = s.pos + (s.w ? q % s.hw % s.w : q);
      }
    }
    for (int s = 0; s < n_seq; ++s) {
      int64_t p = sp[s];
      for (int64_t r = sr[s]; r < sr[s] + sl[s];) {
        size_t it = 0;
        while (it < ir.size() && ir[it] != r) ++it;
        if (it == ir.size()) {
          for (int a = 0; a < 3; ++a) want[3 * r + a] = p;
          ++r;
          ++p;
          continue;
        }
        const int t = g[3 * it], h = g[3 * it + 1] / 2, w = g[3 * it + 2] / 2;
        for (int e = 0; e < t * h * w; ++e, ++r) {
          want[3 * r] = p + (int64_t)(e / (h * w)) * st[it];
          want[3 * r + 1] = p + e / w % h;
          want[3 * r + 2] = p + e % w;
        }
        p += std::max({(int64_t)(t - 1) * st[it] + 1, (int64_t)h, (int64_t)w});
      }
      expect(next[s] == p, "next position", k);
    }
    expect(got == want, "positions", k);
    // anything at all: a status, no report
    std::vector<int64_t> wild(ir.size());
    for (int64_t& v : wild) v = (int64_t)(next_u32() % 400) - 100;
    for (int32_t& v : g) v = uniform(-2, 40);
    position_spans(sr.data(), sl.data(), sp.data(), n_seq, wild.data(), g.data(), st.data(),
                   (int32_t)wild.size(), n_rows, nullptr, spans, end, why);
  }
  const int64_t big[2] = {INT64_MAX, INT64_MIN}, one[1] = {0}, len[1] = {int64_t(1) << 40};
  const int32_t huge[3] = {INT32_MAX, 32768, 32768}, step[1] = {INT32_MAX};
  std::vector<PosSpan> spans;
  std::string why;
  int64_t end;
  expect(position_spans(big, big, big, 2, nullptr, nullptr, nullptr, 0, INT64_MAX, nullptr, spans,
                        end, why) != MPIPE_OK, "extreme sequences", 0);
  expect(position_spans(one, len, nullptr, 1, one, huge, step, 1, int64_t(1) << 40, nullptr, spans,
                        end, why) != MPIPE_OK, "extreme item", 0);
  // text longer than a piece is cut
  const int64_t gib[1] = {int64_t(1) << 30};
  expect(position_spans(one, gib, nullptr, 1, nullptr, nullptr, nullptr, 0, gib[0], nullptr, spans,
                        end, why) == MPIPE_OK && spans.size() == 4 && spans[3].pos == 3 << 28,
         "long text", 0);
}

void check_tables() {
  for (int k = 0; k < 2000; ++k) {
    mpipe_rope_cfg c = {};
    c.head_dim = 8 * uniform(-1, 34);
    c.rot_dim = 8 * uniform(-1, 34);
    c.axes = uniform(-1, 5);
    int left = c.rot_dim / 2;
    for (int a = 0; a < 4; ++a) {
      c.section[a] = a == c.axes - 1 ? left : uniform(0, std::max(0, left));
      left -= c.section[a];
    }
    if (uniform(0, 9) == 0) c.section[0] = uniform(-100000, 100000);
    c.order = uniform(0, 1);
    c.spectrum = uniform(0, 1);
    c.pairing = uniform(0, 1);
    c.theta = uniform(0, 20) ? 1.0 + uniform(1, 1000000) : std::numeric_limits<double>::max();
    RopeTable t;
    std::string why;
    if (rope_axes_table(&c, t, why) != MPIPE_OK) continue;
    int seen[4] = {0, 0, 0, 0};
    for (int i = 0; i < c.rot_dim / 2; ++i) {
      const int a = t.axis[i];
      expect(a < c.axes, "axis", k);
      const double e = c.spectrum ? (double)seen[a] / c.section[a] : (double)i / (c.rot_dim / 2);
      const double f = std::pow(c.theta, -e) / 6.283185307179586477;
      expect(std::fabs(std::ldexp((double)t.turn[i], -64) - f) <= 1e-13 * f + 1e-19, "frequency", k);
      ++seen[a];
    }
    for (int a = 0; a < c.axes; ++a) expect(seen[a] == c.section[a], "sections", k);
  }
}

void check_views() {
  int apart = 0, meet = 0;
  for (int k = 0; k < 20000; ++k) {
    const int d = 8, rows = uniform(1, 4);
    HeadView v[2];
    std::set<uintptr_t> at[2];
    bool ok[2];
    for (int z = 0; z < 2; ++z) {
      v[z].heads = uniform(1, 3);
      v[z].head = uniform(0, 1) ? 8 : uniform(0, 40);
      v[z].row = uniform(0, 1) ? 64 : uniform(0, 90);
      v[z].p = (const void*)(uintptr_t)(4096 + 2 * uniform(0, 120));
      std::string why;
      ok[z] = view_ok(v[z], rows, d, 2, true, why);
      size_t n = 0;
      for (int r = 0; r < rows; ++r)
        for (int h = 0; h < v[z].heads; ++h)
          for (int c = 0; c < d; ++c, ++n)
            at[z].insert((uintptr_t)v[z].p + 2 * (r * v[z].row + h * v[z].head + c));
      if (ok[z]) expect(at[z].size() == n, "an accepted output has distinct elements", k);
    }
    bool share = false;
    for (uintptr_t e : at[0]) share |= at[1].count(e) > 0;
    const bool said = views_meet(v[0], v[1], rows, d, 2);
    if (share) expect(said, "views that meet", k);
    if (!said) ++apart;
    if (share) ++meet;
  }
  expect(apart > 1000 && meet > 1000, "both kinds of views", 0);
  HeadView v;
  std::string why;
  v.p = (const void*)4096;
  v.heads = INT32_MAX;
  v.head = INT64_MAX;
  v.row = INT64_MAX;
  expect(!view_ok(v, 1 << 30, 256, 4, false, why), "strides too large", 0);
}

void check_gradients() {
  for (int k = 0; k < 2000; ++k) {
    const int n = uniform(0, 6);
    std::vector<mpipe_grad_tensor> in(n), out(n);
    uintptr_t at = 4096;
    for (int i = 0; i < n; ++i) {
      in[i].dtype = uniform(0, 1);
      in[i].n = uniform(0, 3) ? uniform(0, 9000) : 0;
      in[i].data = (void*)at;
      at += in[i].n * (in[i].dtype ? 2 : 4) + 4 * uniform(0, 2);
      at = (at + 3) / 4 * 4;
      out[i] = in[i];
      if (uniform(0, 1)) {
        out[i].dtype = uniform(0, 1);
        out[i].data = (void*)(uintptr_t)(uniform(0, 1) ? 1 << 24 : 4096 + 4 * uniform(0, 9000));
      }
    }
    GradPlan p;
    std::string why;
    expect(grad_plan(in.data(), n, p, why) == MPIPE_OK, "valid list", k);
    int64_t chunks = 0;
    for (const auto& t : in) chunks += std::max<int64_t>(1, (t.n + p.chunk - 1) / p.chunk);
    expect(chunks == p.chunks, "chunks", k);
    bool bad = false;
    auto bytes = [](const mpipe_grad_tensor& t) { return (uintptr_t)t.n * (t.dtype ? 2 : 4); };
    auto share = [&](const mpipe_grad_tensor& a, const mpipe_grad_tensor& b) {
      return a.n && b.n && (uintptr_t)a.data < (uintptr_t)b.data + bytes(b) &&
             (uintptr_t)b.data < (uintptr_t)a.data + bytes(a);
    };
    for (int i = 0; i < n; ++i)
      for (int j = 0; j < n; ++j) {
        if (j < i) bad |= share(out[i], out[j]);
        const bool own = i == j && out[i].data == in[i].data && out[i].dtype == in[i].dtype;
        bad |= !own && share(out[i], in[j]);
      }
    expect((grad_outputs_ok(in.data(), out.data(), n, why) != MPIPE_OK) == bad, "outputs", k);
  }
  mpipe_grad_tensor t = {(void*)4096, INT64_MAX, 0, 0};
  GradPlan p;
  std::string why;
  expect(grad_plan(&t, 1, p, why) != MPIPE_OK, "too long", 0);
}

}  // namespace

int main() {
  check_positions();
  check_tables();
  check_views();
  check_gradients();
  if (failures) return 1;
  std::puts("layer checks passed");
  return 0;
}
