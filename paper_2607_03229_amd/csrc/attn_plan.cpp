// Host-only planning of the first LLM layer's attention; see attn_plan.h.
#include "attn_plan.h"

#include <algorithm>

namespace mpipe {
namespace {

mpipe_status fail(std::string& why, mpipe_status s, const char* m) {
  why = m;
  return s;
}

bool apart(std::vector<std::pair<int64_t, int64_t>>& r) {
  auto less = [](const auto& a, const auto& b) { return a.first < b.first; };
  if (!std::is_sorted(r.begin(), r.end(), less)) std::sort(r.begin(), r.end(), less);
  for (size_t i = 1; i < r.size(); ++i)
    if (r[i].first < r[i - 1].second) return false;
  return true;
}

}  // namespace

mpipe_status attn_sequences(const int64_t* seq_row, const int64_t* seq_len, const int64_t* key_row,
                            const int64_t* key_len, int32_t n_seq, int64_t rows_q, int64_t rows_k,
                            bool keys_apart, std::vector<AttnSeq>& seqs, std::string& why) {
  if (rows_q < 0 || rows_k < 0) return fail(why, MPIPE_ERR_INVALID_ARG, "negative row count");
  if (rows_q > (1 << 30) || rows_k > (1 << 30))
    return fail(why, MPIPE_ERR_UNSUPPORTED, "more than 2^30 rows");
  if (n_seq < 0) return fail(why, MPIPE_ERR_INVALID_ARG, "negative sequence count");
  if (n_seq > 0 && (!seq_row || !seq_len))
    return fail(why, MPIPE_ERR_INVALID_ARG, "null sequence list");
  if (!key_row != !key_len)
    return fail(why, MPIPE_ERR_INVALID_ARG, "key_row and key_len go together");
  if (!key_row) {
    key_row = seq_row;
    key_len = seq_len;
  }
  std::vector<std::pair<int64_t, int64_t>> q, k;
  q.reserve(n_seq);
  k.reserve(n_seq);
  seqs.reserve(n_seq);
  for (int32_t i = 0; i < n_seq; ++i) {
    const int64_t a = seq_row[i], n = seq_len[i], b = key_row[i], m = key_len[i];
    if (n < 0 || m < 0) return fail(why, MPIPE_ERR_INVALID_ARG, "negative sequence length");
    if (a < 0 || a > rows_q || n > rows_q - a || b < 0 || b > rows_k || m > rows_k - b)
      return fail(why, MPIPE_ERR_INVALID_ARG, "a sequence outside the rows");
    if (n > 0) q.push_back({a, a + n});
    if (m > 0) k.push_back({b, b + m});
    seqs.push_back({(int32_t)a, (int32_t)n, (int32_t)b, (int32_t)m});
  }
  if (!apart(q)) return fail(why, MPIPE_ERR_INVALID_ARG, "two sequences share a row");
  if (keys_apart && !apart(k))
    return fail(why, MPIPE_ERR_INVALID_ARG, "two sequences share a key row, whose gradient would be theirs both");
  return MPIPE_OK;
}

void attn_items(const std::vector<AttnSeq>& seqs, bool by_keys, int rows,
                std::vector<AttnItem>& items) {
  struct Order {
    int64_t walk;
    AttnItem item;
  };
  std::vector<Order> order;
  for (size_t s = 0; s < seqs.size(); ++s) {
    const int64_t nq = seqs[s].q_len, nk = seqs[s].k_len, n = by_keys ? nk : nq;
    for (int64_t t = 0; t * rows < n; ++t) {
      // keys the item's last query sees, or queries that see the item's first key
      const int64_t walk = by_keys ? std::min(nq, nk - t * rows)
                                   : std::min(nk, (t + 1) * rows + nk - nq);
      order.push_back({walk, {(int32_t)s, (int32_t)t}});
    }
  }
  std::stable_sort(order.begin(), order.end(),
                   [](const Order& a, const Order& b) { return a.walk > b.walk; });
  items.reserve(order.size());
  for (const Order& o : order) items.push_back(o.item);
}

int attn_pack(const std::vector<AttnSeq>& seqs, const std::vector<AttnItem>& items, size_t at,
              int64_t most, AttnPool& pool) {
  int n = 0, n_seq = 0;
  int32_t slot_of[256];   // the sequence in each slot of this launch
  for (; at + n < items.size() && n < most; ++n) {
    const AttnItem& it = items[at + n];
    int slot = n_seq - 1;
    while (slot >= 0 && slot_of[slot] != it.seq) --slot;
    const int more = slot < 0 ? 1 : 0;
    if (4 * (n_seq + more) + n + 1 > kAttnWords || n_seq + more > 256) break;
    if (more) {
      slot = n_seq++;
      slot_of[slot] = it.seq;
      const AttnSeq& s = seqs[it.seq];
      const int32_t w[4] = {s.q_row, s.q_len, s.k_row, s.k_len};
      std::copy(w, w + 4, pool.word + 4 * slot);
    }
    pool.word[kAttnWords - 1 - n] = (int32_t)((uint32_t)it.tile << 8 | (uint32_t)slot);
  }
  return n;
}

// ---- paged cache --------------------------------------------------------------------------

namespace {
int cache_esz(int32_t dtype) { return dtype == MPIPE_F32 ? 4 : dtype == MPIPE_BF16 ? 2 : 1; }
}  // namespace

int64_t cache_page_values(const mpipe_kv_cache& c) {
  return (int64_t)c.heads * c.page * c.head_dim;
}

mpipe_status cache_ok(const mpipe_kv_cache* c, std::string& why) {
  if (!c) return fail(why, MPIPE_ERR_INVALID_ARG, "null cache");
  if (c->dtype != MPIPE_F32 && c->dtype != MPIPE_BF16 && c->dtype != MPIPE_E4M3)
    return fail(why, MPIPE_ERR_INVALID_ARG, "bad dtype of the cache");
  if (c->head_dim < 8 || c->head_dim > kMaxHeadDim || c->head_dim % 8)
    return fail(why, MPIPE_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 of at most 256");
  if (c->heads < 1) return fail(why, MPIPE_ERR_INVALID_ARG, "a cache of no heads");
  if (c->heads > 65536) return fail(why, MPIPE_ERR_UNSUPPORTED, "more than 65536 heads");
  if (c->page < 1 || (c->page & (c->page - 1)) || c->page > (1 << 16))
    return fail(why, MPIPE_ERR_UNSUPPORTED, "a page's tokens must be a power of two of at most 2^16");
  if (c->n_pages < 0 || c->n_pages > INT32_MAX)
    return fail(why, MPIPE_ERR_INVALID_ARG, "page count out of range");
  if (c->n_pages == 0) return MPIPE_OK;
  int64_t n;
  if (__builtin_mul_overflow(cache_page_values(*c), c->n_pages, &n) || n > INT64_MAX / 8)
    return fail(why, MPIPE_ERR_INVALID_ARG, "a cache too large");
  if (!c->k || !c->v || (uintptr_t)c->k % 16 || (uintptr_t)c->v % 16)
    return fail(why, MPIPE_ERR_INVALID_ARG, "null pages, or pages not aligned to 16 bytes");
  const bool scaled = c->dtype == MPIPE_E4M3;
  if (scaled != (c->k_scale != nullptr) || scaled != (c->v_scale != nullptr))
    return fail(why, MPIPE_ERR_INVALID_ARG, "scales go with 8-bit pages, and only with them");
  const size_t bytes = (size_t)n * cache_esz(c->dtype), sb = scaled ? (size_t)(n / c->head_dim) : 0;
  const struct {
    const void* p;
    size_t bytes;
  } part[4] = {{c->k, bytes}, {c->v, bytes}, {c->k_scale, sb}, {c->v_scale, sb}};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (ranges_meet(part[i].p, part[i].bytes, part[j].p, part[j].bytes))
        return fail(why, MPIPE_ERR_INVALID_ARG, "the cache's parts share memory");
  return MPIPE_OK;
}

bool cache_meets(const mpipe_kv_cache& c, const void* p, size_t bytes) {
  const size_t n = (size_t)(cache_page_values(c) * c.n_pages), nb = n * cache_esz(c.dtype);
  const size_t sb = c.dtype == MPIPE_E4M3 ? n / c.head_dim : 0;
  return ranges_meet(p, bytes, c.k, nb) || ranges_meet(p, bytes, c.v, nb) ||
         ranges_meet(p, bytes, c.k_scale, sb) || ranges_meet(p, bytes, c.v_scale, sb);
}

bool cache_meets(const mpipe_kv_cache& c, const HeadView& v, int64_t rows, int esz) {
  const size_t n = (size_t)(cache_page_values(c) * c.n_pages), nb = n * cache_esz(c.dtype);
  const size_t sb = c.dtype == MPIPE_E4M3 ? n / c.head_dim : 0;
  const int d = c.head_dim;
  return range_meets(c.k, nb, v, rows, d, esz) || range_meets(c.v, nb, v, rows, d, esz) ||
         (sb && (range_meets(c.k_scale, sb, v, rows, d, esz) ||
                 range_meets(c.v_scale, sb, v, rows, d, esz)));
}

}  // namespace mpipe
