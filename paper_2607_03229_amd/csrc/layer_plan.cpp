// Host-only planning of the operators around the first LLM layer (layer_plan.h).
#include "layer_plan.h"

#include <algorithm>
#include <climits>
#include <cmath>

namespace mpipe {

namespace {
mpipe_status fail(std::string& why, mpipe_status s, const char* text) {
  why = text;
  return s;
}
}  // namespace

// ---- positions ----------------------------------------------------------------------------

mpipe_status position_spans(const int64_t* seq_row, const int64_t* seq_len,
                            const int64_t* seq_pos, int32_t n_seq, const int64_t* item_row,
                            const int32_t* grid_thw, const int32_t* time_step, int32_t n_items,
                            int64_t n_rows, int64_t* next, std::vector<PosSpan>& spans,
                            int64_t& end, std::string& why) {
  constexpr int64_t kPiece = int64_t(1) << 28;
  spans.clear();
  end = 0;
  if (n_seq < 0 || n_items < 0 || n_rows < 0)
    return fail(why, MPIPE_ERR_INVALID_ARG, "negative count");
  if ((n_seq > 0 && (!seq_row || !seq_len)) || (n_items > 0 && (!item_row || !grid_thw)))
    return fail(why, MPIPE_ERR_INVALID_ARG, "null host array");
  std::vector<int32_t> seqs, items(n_items);
  for (int32_t i = 0; i < n_seq; ++i) {
    if (seq_len[i] < 0 || seq_row[i] < 0 || seq_row[i] > n_rows || seq_len[i] > n_rows - seq_row[i])
      return fail(why, MPIPE_ERR_BAD_METADATA, "a sequence outside the rows");
    if (seq_pos && (seq_pos[i] < 0 || seq_pos[i] > INT32_MAX))
      return fail(why, MPIPE_ERR_BAD_METADATA, "a first position outside [0, 2^31)");
    if (seq_len[i] > 0) seqs.push_back(i);
  }
  for (int32_t i = 0; i < n_items; ++i) {
    const int32_t* g = grid_thw + 3 * (int64_t)i;
    if (g[0] <= 0 || g[1] <= 0 || g[2] <= 0 || g[1] % 2 || g[2] % 2 || g[1] > 32768 || g[2] > 32768)
      return fail(why, MPIPE_ERR_BAD_METADATA, "bad grid");
    if ((int64_t)g[0] * (g[1] / 2) * (g[2] / 2) > kPiece)
      return fail(why, MPIPE_ERR_UNSUPPORTED, "an item of more than 2^28 rows");
    if (time_step && time_step[i] < 0)
      return fail(why, MPIPE_ERR_BAD_METADATA, "negative time step");
    if (item_row[i] < 0) return fail(why, MPIPE_ERR_BAD_METADATA, "an item outside the sequences");
    items[i] = i;
  }
  std::sort(seqs.begin(), seqs.end(),
            [&](int32_t a, int32_t b) { return seq_row[a] < seq_row[b]; });
  std::sort(items.begin(), items.end(),
            [&](int32_t a, int32_t b) { return item_row[a] < item_row[b]; });
  auto text = [&](int64_t row, int64_t n, int64_t pos, int32_t w) {
    for (; n > 0; row += kPiece, pos += kPiece, n -= kPiece)
      spans.push_back({row, w < 0 ? 0 : (int32_t)pos, 1, 1, w});
  };
  std::vector<int64_t> last(n_seq);
  for (int32_t i = 0; i < n_seq; ++i) last[i] = seq_pos ? seq_pos[i] : 0;
  size_t it = 0;
  for (int32_t s : seqs) {
    const int64_t stop = seq_row[s] + seq_len[s];
    int64_t at = seq_row[s], p = last[s];
    if (!spans.empty()) {
      if (at < end) return fail(why, MPIPE_ERR_BAD_METADATA, "sequences overlap");
      text(end, at - end, 0, -1);
    }
    if (it < items.size() && item_row[items[it]] < at)
      return fail(why, MPIPE_ERR_BAD_METADATA, "an item outside the sequences, or two that overlap");
    for (; it < items.size() && item_row[items[it]] < stop; ++it) {
      const int32_t i = items[it];
      const int64_t t = grid_thw[3 * (int64_t)i], h = grid_thw[3 * (int64_t)i + 1] / 2,
                    w = grid_thw[3 * (int64_t)i + 2] / 2, step = time_step ? time_step[i] : 1;
      const int64_t n = t * h * w, gap = item_row[i] - at;
      if (gap < 0 || n > stop - item_row[i])
        return fail(why, MPIPE_ERR_BAD_METADATA, "an item across a sequence's end, or two that overlap");
      const int64_t extent = std::max((t - 1) * step + 1, std::max(h, w));
      if (p + gap + extent - 1 > INT32_MAX)
        return fail(why, MPIPE_ERR_UNSUPPORTED, "a position of 2^31 or more");
      text(at, gap, p, 0);
      p += gap;
      spans.push_back({item_row[i], (int32_t)p, (int32_t)step, (int32_t)(h * w), (int32_t)w});
      p += extent;
      at = item_row[i] + n;
    }
    if (p + (stop - at) - 1 > INT32_MAX)
      return fail(why, MPIPE_ERR_UNSUPPORTED, "a position of 2^31 or more");
    text(at, stop - at, p, 0);
    last[s] = p + (stop - at);
    end = stop;
  }
  if (it < items.size()) return fail(why, MPIPE_ERR_BAD_METADATA, "an item outside the sequences");
  if (next) std::copy(last.begin(), last.end(), next);
  return MPIPE_OK;
}

// ---- rotary tables ------------------------------------------------------------------------

mpipe_status rope_axes_table(const mpipe_rope_cfg* c, RopeTable& t, std::string& why) {
  if (!c) return fail(why, MPIPE_ERR_INVALID_ARG, "null rotary configuration");
  if (c->head_dim < 8 || c->head_dim > kMaxHeadDim || c->head_dim % 8 || c->rot_dim < 8 ||
      c->rot_dim > c->head_dim || c->rot_dim % 8)
    return fail(why, MPIPE_ERR_UNSUPPORTED,
                "head_dim and rot_dim must be multiples of 8, 8 <= rot_dim <= head_dim <= 256");
  if (c->axes < 1 || c->axes > MPIPE_ROPE_MAX_AXES)
    return fail(why, MPIPE_ERR_INVALID_ARG, "axes must be 1 to 4");
  if (c->order < 0 || c->order > 1 || c->spectrum < 0 || c->spectrum > 1 || c->pairing < 0 ||
      c->pairing > 1)
    return fail(why, MPIPE_ERR_INVALID_ARG, "bad order, spectrum or pairing");
  if (!(c->theta > 1.0) || !std::isfinite(c->theta))
    return fail(why, MPIPE_ERR_INVALID_ARG, "theta must be finite and above 1");
  const int half = c->rot_dim / 2;
  int64_t sum = 0;
  for (int a = 0; a < c->axes; ++a) {
    if (c->section[a] < 0) return fail(why, MPIPE_ERR_INVALID_ARG, "negative section");
    sum += c->section[a];
  }
  if (sum != half)
    return fail(why, MPIPE_ERR_INVALID_ARG, "the sections must sum to rot_dim / 2");
  int count[MPIPE_ROPE_MAX_AXES] = {0, 0, 0, 0};
  int block = 0;
  // Frequencies as running products of one ratio per axis, in 64-bit mantissas: off by less
  // than 2^-57 of themselves after 128 products, which 2^31 positions turn into 2^-26 of a
  // radian; fp64 would leave 2^-20.
  const bool each = c->spectrum == MPIPE_ROPE_AXIS_SPECTRA;
  long double ratio[MPIPE_ROPE_MAX_AXES], next[MPIPE_ROPE_MAX_AXES];
  for (int a = 0; a < (each ? c->axes : 1); ++a) {
    const int n = each ? c->section[a] : half;
    ratio[a] = n > 0 ? std::pow((long double)c->theta, -1.0L / n) : 1.0L;
    next[a] = 18446744073709551616.0L / 6.283185307179586476925286766559L;   // 2^64 / (2 pi)
  }
  for (int i = 0; i < half; ++i) {
    int a;
    if (c->order == MPIPE_ROPE_INTERLEAVED) {
      a = i % c->axes;
      if (i / c->axes >= c->section[a]) a = 0;
    } else {
      while (count[block] == c->section[block]) ++block;
      a = block;
    }
    ++count[a];
    if (count[a] > c->section[a])
      return fail(why, MPIPE_ERR_INVALID_ARG, "the sections do not fit the interleaved order");
    long double& f = next[each ? a : 0];
    t.turn[i] = (uint64_t)std::llround(f);   // below 2^62
    f *= ratio[each ? a : 0];
    t.axis[i] = (uint8_t)a;
  }
  for (int i = half; i < kMaxPairs; ++i) {
    t.turn[i] = 0;
    t.axis[i] = 0;
  }
  return MPIPE_OK;
}

// ---- views of heads -----------------------------------------------------------------------

namespace {
// elements from the first to one past the last; false on overflow
bool extent(const HeadView& v, int64_t rows, int32_t d, int64_t& n) {
  int64_t a, b;
  if (__builtin_mul_overflow(rows - 1, v.row, &a) ||
      __builtin_mul_overflow((int64_t)v.heads - 1, v.head, &b) || __builtin_add_overflow(a, b, &n) ||
      __builtin_add_overflow(n, (int64_t)d, &n))
    return false;
  return n <= INT64_MAX / 8;
}
}  // namespace

bool view_ok(const HeadView& v, int64_t rows, int32_t d, int esz, bool written, std::string& why) {
  if (v.heads < 0) return why = "negative head count", false;
  if (v.heads == 0 || rows == 0) return true;
  if (!v.p) return why = "null device buffer", false;
  if ((uintptr_t)v.p % esz) return why = "a buffer not aligned to its elements", false;
  if (v.row < 0 || v.head < 0) return why = "negative stride", false;
  int64_t n;
  if (!extent(v, rows, d, n)) return why = "strides too large", false;
  if (written) {
    const int64_t w = (v.heads - 1) * v.head + d, t = (rows - 1) * v.row + d;
    const bool heads_ok = v.heads == 1 || v.head >= d, rows_ok = rows == 1 || v.row >= d;
    if (!heads_ok || !rows_ok || (rows > 1 && v.heads > 1 && v.row < w && v.head < t))
      return why = "an output whose heads or rows overlap", false;
  }
  return true;
}

bool same_view(const HeadView& a, const HeadView& b, int64_t rows) {
  return a.p == b.p && a.heads == b.heads && (a.row == b.row || rows == 1) &&
         (a.head == b.head || a.heads == 1);
}

namespace {
// Whether x + c * step comes within (-d, d) for a whole c of [lo, hi].
bool comes_near(int64_t x, int64_t step, int64_t lo, int64_t hi, int32_t d) {
  // the last c that leaves it at or below zero, and the next
  const int64_t last = step == 0 ? lo : x > 0 ? -((x - 1) / step) - 1 : -x / step;
  for (int64_t c : {last, last + 1}) {
    const int64_t y = x + std::max(lo, std::min(hi, c)) * step;
    if (y > -d && y < d) return true;
  }
  return false;
}
}  // namespace

bool views_meet(const HeadView& a, const HeadView& b, int64_t rows, int32_t d, int esz) {
  if (a.heads == 0 || b.heads == 0 || rows == 0) return false;
  if (b.heads > a.heads) return views_meet(b, a, rows, d, esz);
  int64_t na, nb;
  extent(a, rows, d, na);
  extent(b, rows, d, nb);
  if (!ranges_meet(a.p, (size_t)na * esz, b.p, (size_t)nb * esz)) return false;
  if (rows > 1 && a.row != b.row) return true;
  const int64_t row = rows > 1 ? a.row : 0, head_a = a.heads > 1 ? a.head : 0,
                head_b = b.heads > 1 ? b.head : head_a;
  const int64_t off = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p) / esz;
  const int64_t wa = (a.heads - 1) * head_a + d, wb = (b.heads - 1) * head_b + d;
  const bool whole = row > 0 && wa <= row && wb <= row;   // a row holds each of them
  const int64_t in_row = whole ? (off % row + row) % row : 0;
  if (whole && in_row >= wa && in_row + wb <= row) return false;   // side by side
  // Heads of one stride, too: the distances of two heads are off + i * row + j * head for all
  // i and j between the rows' and the heads' differences.
  if (head_a == head_b) {
    if (a.heads + (int64_t)b.heads < 2 * rows) {
      for (int64_t j = 1 - a.heads; j < b.heads; ++j)
        if (comes_near(off + j * head_a, row, 1 - rows, rows - 1, d)) return true;
    } else {
      for (int64_t i = 1 - rows; i < rows; ++i)
        if (comes_near(off + i * row, head_a, 1 - a.heads, b.heads - 1, d)) return true;
    }
    return false;
  }
  // Otherwise b's heads one by one against a's of the same row and, where a head runs on into
  // the next, of that one; which rows come first and last is not looked at.
  if (row > 0 && !whole) return true;
  for (int64_t j = 0; j < b.heads; ++j) {
    int64_t x = off + j * head_b;
    if (row > 0) {
      x = (x % row + row) % row;
      if (comes_near(row - x, head_a, 0, a.heads - 1, d)) return true;
    }
    if (comes_near(-x, head_a, 0, a.heads - 1, d)) return true;
  }
  return false;
}

bool ranges_meet(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  return a_bytes > 0 && b_bytes > 0 && pa < pb + b_bytes && pb < pa + a_bytes;
}

bool range_meets(const void* p, size_t bytes, const HeadView& v, int64_t rows, int32_t d, int esz) {
  if (v.heads == 0 || rows == 0) return false;
  int64_t n;
  extent(v, rows, d, n);
  if (!ranges_meet(p, bytes, v.p, (size_t)n * esz)) return false;
  // the range as [lo, hi) from the view's start; the shorter side of the view is walked, and
  // on the other the first run of columns that ends behind lo starts before hi or none does
  const int64_t lo = (int64_t)((uintptr_t)p - (uintptr_t)v.p), hi = lo + (int64_t)bytes;
  const bool by_head = v.heads <= rows;
  const int64_t s_row = rows > 1 ? v.row * esz : 0, s_head = v.heads > 1 ? v.head * esz : 0;
  const int64_t n_out = by_head ? v.heads : rows, n_in = by_head ? rows : v.heads;
  const int64_t s_out = by_head ? s_head : s_row, s_in = by_head ? s_row : s_head;
  for (int64_t o = 0; o < n_out; ++o) {
    const int64_t behind = lo - o * s_out - (int64_t)d * esz;   // the run's offset is above it
    int64_t i = 0;
    if (behind >= 0) {
      if (s_in == 0) continue;
      i = behind / s_in + 1;
    }
    if (i < n_in && o * s_out + i * s_in < hi) return true;
  }
  return false;
}

// ---- gradient lists -------------------------------------------------------------------------

int64_t grad_chunk(int64_t total) {
  int64_t c = 4096;
  while (c < 32768 && c * 2048 < total) c *= 2;
  return c;
}

namespace {

int esz_of(int32_t dtype) { return dtype == MPIPE_BF16 ? 2 : 4; }

// every tensor valid: type, length, pointer
mpipe_status tensors_ok(const mpipe_grad_tensor* t, int32_t n, int64_t& total, std::string& why) {
  if (n < 0) return fail(why, MPIPE_ERR_INVALID_ARG, "negative tensor count");
  if (n > 0 && !t) return fail(why, MPIPE_ERR_INVALID_ARG, "null tensor list");
  total = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].dtype != MPIPE_F32 && t[i].dtype != MPIPE_BF16)
      return fail(why, MPIPE_ERR_INVALID_ARG, "bad dtype");
    if (t[i].n < 0 || t[i].n > (int64_t(1) << 44))
      return fail(why, MPIPE_ERR_INVALID_ARG, "a tensor of fewer than 0 or more than 2^44 elements");
    if (t[i].n > 0 && (!t[i].data || (uintptr_t)t[i].data % esz_of(t[i].dtype)))
      return fail(why, MPIPE_ERR_INVALID_ARG, "a null tensor, or one not aligned to its elements");
    if ((uintptr_t)t[i].data >> 48)   // the kernels' lists keep 48 bits of it
      return fail(why, MPIPE_ERR_INVALID_ARG, "an address of more than 48 bits");
    total += t[i].n;
    if (total > (int64_t(1) << 44))
      return fail(why, MPIPE_ERR_INVALID_ARG, "more than 2^44 elements in all");
  }
  return MPIPE_OK;
}

struct Range {
  uintptr_t lo, hi;
  int32_t owner;
};
void ranges_of(const mpipe_grad_tensor* t, int32_t n, std::vector<Range>& r) {
  for (int32_t i = 0; i < n; ++i)
    if (t[i].n > 0)
      r.push_back({(uintptr_t)t[i].data, (uintptr_t)t[i].data + (uintptr_t)t[i].n * esz_of(t[i].dtype), i});
}
void sort_ranges(std::vector<Range>& r) {
  auto less = [](const Range& a, const Range& b) { return a.lo < b.lo; };
  if (!std::is_sorted(r.begin(), r.end(), less)) std::sort(r.begin(), r.end(), less);
}
bool apart(const std::vector<Range>& r) {   // sorted
  for (size_t i = 1; i < r.size(); ++i)
    if (r[i].lo < r[i - 1].hi) return false;
  return true;
}

}  // namespace

mpipe_status grad_plan(const mpipe_grad_tensor* t, int32_t n, GradPlan& p, std::string& why) {
  mpipe_status st = tensors_ok(t, n, p.total, why);
  if (st) return st;
  std::vector<Range> r;
  r.reserve(n);
  ranges_of(t, n, r);
  sort_ranges(r);
  if (!apart(r)) return fail(why, MPIPE_ERR_INVALID_ARG, "two tensors of the list share memory");
  p.chunk = grad_chunk(p.total);
  p.chunks = 0;
  for (int32_t i = 0; i < n; ++i) p.chunks += std::max<int64_t>(1, (t[i].n + p.chunk - 1) / p.chunk);
  if (p.chunks > (1 << 23))   // blocks of a launch: 2^32 threads in all
    return fail(why, MPIPE_ERR_UNSUPPORTED, "too many tensors or elements");
  return MPIPE_OK;
}

mpipe_status grad_outputs_ok(const mpipe_grad_tensor* in, const mpipe_grad_tensor* out, int32_t n,
                             std::string& why) {
  int64_t total;
  mpipe_status st = tensors_ok(out, n, total, why);
  if (st) return st;
  for (int32_t i = 0; i < n; ++i)
    if (in[i].n != out[i].n)
      return fail(why, MPIPE_ERR_INVALID_ARG, "an output of another length than its input");
  std::vector<Range> a, b;
  a.reserve(n);
  b.reserve(n);
  ranges_of(in, n, a);
  ranges_of(out, n, b);
  sort_ranges(a);
  sort_ranges(b);
  if (!apart(b)) return fail(why, MPIPE_ERR_INVALID_ARG, "two outputs share memory");
  // both sorted and apart within themselves: one sweep finds every pair that meets
  for (size_t i = 0, j = 0; i < a.size() && j < b.size();) {
    if (a[i].hi <= b[j].lo) {
      ++i;
    } else if (b[j].hi <= a[i].lo) {
      ++j;
    } else {
      if (a[i].owner != b[j].owner || a[i].lo != b[j].lo || a[i].hi != b[j].hi)
        return fail(why, MPIPE_ERR_INVALID_ARG, "an output that meets an input other than its own");
      ++i;
      ++j;
    }
  }
  return MPIPE_OK;
}

bool list_meets(const mpipe_grad_tensor* t, int32_t n, const void* p, size_t bytes) {
  for (int32_t i = 0; i < n; ++i)
    if (ranges_meet(p, bytes, t[i].data, (size_t)t[i].n * esz_of(t[i].dtype))) return true;
  return false;
}

}  // namespace mpipe
