// Entry points of the first LLM layer's attention (include/mpipe_ops.h): every check on the
// host, then the launches.
#include <cmath>
#include <exception>
#include <string>

#include "attn_kernels.h"

using namespace mpipe;

namespace mpipe {
mpipe_status set_error(mpipe_status s, const std::string& m);
}

namespace {

mpipe_status hip_status(hipError_t e) {
  if (e == hipSuccess) return MPIPE_OK;
  return set_error(MPIPE_ERR_HIP, std::string("launch: ") + hipGetErrorString(e));
}

// no exception (host memory running out) leaves a C entry
template <class F>
mpipe_status guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return set_error(MPIPE_ERR_INVALID_ARG, e.what());
  }
}

mpipe_status invalid(const char* m) { return set_error(MPIPE_ERR_INVALID_ARG, m); }

int esz_of(int32_t dtype) { return dtype == MPIPE_BF16 ? 2 : 4; }

bool dim_ok(int32_t d) { return d >= 8 && d <= kMaxHeadDim && d % 8 == 0; }
constexpr const char* kBadDim = "head_dim must be a multiple of 8 of at most 256";

// A view with its rows.
struct Side {
  HeadView v;
  int64_t rows = 0;
  bool written = false;
};
Side side_of(const mpipe_heads* h, int64_t rows, bool written) {
  Side s;
  if (h) {
    s.v.p = h->p;
    s.v.row = h->row_stride;
    s.v.head = h->head_stride;
    s.v.heads = h->heads;
  }
  s.rows = rows;
  s.written = written;
  return s;
}
bool sides_meet(const Side& a, const Side& b, int32_t d, int esz) {
  if (a.rows == 0 || b.rows == 0) return false;
  if (a.rows == b.rows) return views_meet(a.v, b.v, a.rows, d, esz);
  // of other row counts: apart as far as both would reach with the rows of the longer, or by
  // their own ranges
  const Side &s = a.rows < b.rows ? a : b, &t = a.rows < b.rows ? b : a;
  const size_t bytes = ((s.rows - 1) * s.v.row + (s.v.heads - 1) * s.v.head + d) * (size_t)esz;
  if (!range_meets(s.v.p, bytes, t.v, t.rows, d, esz)) return false;
  HeadView longer = s.v;
  std::string why;
  return !view_ok(longer, t.rows, d, esz, false, why) || views_meet(longer, t.v, t.rows, d, esz);
}

// Valid views, and every written one apart from all others.
mpipe_status sides_ok(const Side* s, int n, int32_t d, int esz) {
  std::string why;
  for (int i = 0; i < n; ++i)
    if (!view_ok(s[i].v, s[i].rows, d, esz, s[i].written, why))
      return set_error(MPIPE_ERR_INVALID_ARG, why);
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if ((s[i].written || s[j].written) && sides_meet(s[i], s[j], d, esz))
        return invalid("an output shares memory with another view");
  return MPIPE_OK;
}
bool sides_meet_range(const Side* s, int n, const void* p, size_t bytes, int32_t d, int esz) {
  for (int i = 0; i < n; ++i)
    if (range_meets(p, bytes, s[i].v, s[i].rows, d, esz)) return true;
  return false;
}

mpipe_status heads_ok(int32_t heads_q, int32_t heads_k) {
  if (heads_q < 0 || heads_k < 0) return invalid("negative head count");
  if (heads_q > 65536) return set_error(MPIPE_ERR_UNSUPPORTED, "more than 65536 heads");
  if (heads_q > 0 && (heads_k == 0 || heads_q % heads_k))
    return invalid("the heads of q must be a multiple of those of k");
  if (heads_q == 0 && heads_k > 0) return invalid("heads of k without heads of q");
  return MPIPE_OK;
}

// [heads][ld] of statistics: null, or aligned and long enough; bytes it spans
mpipe_status stats_ok(const float* lse, int64_t ld, int64_t rows, int32_t heads, size_t& bytes) {
  bytes = 0;
  if (!lse || rows == 0 || heads == 0) return MPIPE_OK;
  if ((uintptr_t)lse % 4) return invalid("lse misaligned");
  if (ld < rows || ld > (int64_t(1) << 40)) return invalid("ld_lse must be at least the rows");
  bytes = ((size_t)(heads - 1) * ld + rows) * sizeof(float);
  return MPIPE_OK;
}

bool scale_ok(float s) { return std::isfinite(s) && s > 0.f; }

mpipe_status check_causal(CausalProblem& p, int32_t dtype, int32_t head_dim, int64_t rows_q,
                          int64_t rows_k, const mpipe_heads* const in[5],
                          const mpipe_heads* const out[3], bool bwd, const int64_t* seq_row,
                          const int64_t* seq_len, const int64_t* key_row, const int64_t* key_len,
                          int32_t n_seq, float scale, float* lse, int64_t ld_lse, void* scratch,
                          size_t scratch_bytes) {
  if (dtype != MPIPE_F32 && dtype != MPIPE_BF16) return invalid("bad dtype");
  if (!dim_ok(head_dim)) return set_error(MPIPE_ERR_UNSUPPORTED, kBadDim);
  if (!scale_ok(scale)) return invalid("scale must be positive and finite");
  std::string why;
  if (mpipe_status st = attn_sequences(seq_row, seq_len, key_row, key_len, n_seq, rows_q, rows_k,
                                       bwd, p.seqs, why))
    return set_error(st, why);
  const int esz = esz_of(dtype), d = head_dim;
  // in: q, k, v, and for a backward o and d_o; out: o, or dq, dk, dv
  Side s[8] = {side_of(in[0], rows_q, false), side_of(in[1], rows_k, false),
               side_of(in[2], rows_k, false)};
  int n = 3;
  if (bwd) {
    s[n++] = side_of(in[3], rows_q, false);
    s[n++] = side_of(in[4], rows_q, false);
    s[n++] = side_of(out[0], rows_q, true);
    s[n++] = side_of(out[1], rows_k, true);
    s[n++] = side_of(out[2], rows_k, true);
  } else {
    s[n++] = side_of(out[0], rows_q, true);
  }
  const int hq = s[0].v.heads, hk = s[1].v.heads;
  if (mpipe_status st = heads_ok(hq, hk)) return st;
  for (int i = 0; i < n; ++i) {
    const bool of_k = i == 1 || i == 2 || (bwd && i >= 6);
    if (s[i].v.heads != (of_k ? hk : hq)) return invalid("inputs and outputs of different head counts");
  }
  if (mpipe_status st = sides_ok(s, n, d, esz)) return st;
  p.dtype = dtype;
  p.head_dim = d;
  p.rows_q = rows_q;
  p.rows_k = rows_k;
  p.q = s[0].v;
  p.k = s[1].v;
  p.v = s[2].v;
  p.o = s[3].v;
  p.scale = scale;
  p.lse = lse;
  p.ld_lse = ld_lse;
  size_t lse_bytes = 0;
  if (mpipe_status st = stats_ok(lse, ld_lse, rows_q, hq, lse_bytes)) return st;
  if (!bwd) {
    if (sides_meet_range(s, n, lse, lse_bytes, d, esz)) return invalid("lse shares memory with a view");
    return MPIPE_OK;
  }
  p.d_o = s[4].v;
  p.dq = s[5].v;
  p.dk = s[6].v;
  p.dv = s[7].v;
  if (!lse && rows_q > 0 && hq > 0) return invalid("null lse");
  if (sides_meet_range(s + 5, 3, lse, lse_bytes, d, esz)) return invalid("an output shares memory with lse");
  if (hq == 0 || p.seqs.empty()) return MPIPE_OK;
  const size_t need = causal_attention_scratch(rows_q, hq, rows_k, hk, d);
  if (!scratch || scratch_bytes < need) return set_error(MPIPE_ERR_WORKSPACE, "scratch too small");
  if ((uintptr_t)scratch % 16) return invalid("scratch misaligned");
  if (sides_meet_range(s, n, scratch, need, d, esz) || ranges_meet(scratch, need, lse, lse_bytes))
    return invalid("scratch shares memory with another buffer");
  p.scratch = reinterpret_cast<float*>(scratch);
  return MPIPE_OK;
}

// Tables, positions and status of a cache's rows; `rows` > 0.
mpipe_status check_rows(CacheRows& p, const mpipe_kv_cache* cache, int32_t dtype, int64_t rows,
                        const mpipe_heads* k, const mpipe_heads* v, const int32_t* table,
                        int64_t ld_table, int32_t n_seq, int32_t width, const int32_t* seq,
                        const int32_t* pos, int32_t* status, bool read) {
  std::string why;
  if (mpipe_status st = cache_ok(cache, why)) return set_error(st, why);
  if (dtype != MPIPE_F32 && dtype != MPIPE_BF16) return invalid("bad dtype");
  if (rows < 0) return invalid("negative row count");
  if (rows > (1 << 30)) return set_error(MPIPE_ERR_UNSUPPORTED, "more than 2^30 rows");
  if (n_seq < 0 || width < 0) return invalid("negative table size");
  const int esz = esz_of(dtype), d = cache->head_dim;
  const Side s[2] = {side_of(k, rows, read), side_of(v, rows, read)};
  if (s[0].v.heads != cache->heads || s[1].v.heads != cache->heads)
    return invalid("rows and cache of different head counts");
  if (mpipe_status st = sides_ok(s, 2, d, esz)) return st;
  p.cache = *cache;
  p.dtype = dtype;
  p.rows = rows;
  p.k = s[0].v;
  p.v = s[1].v;
  p.table = table;
  p.ld_table = ld_table;
  p.n_seq = n_seq;
  p.width = width;
  p.seq = seq;
  p.pos = pos;
  p.status = status;
  if (rows == 0) return MPIPE_OK;
  if (cache->n_pages == 0) return invalid("a cache of no pages");
  if (!pos || (uintptr_t)pos % 4 || (uintptr_t)seq % 4 || (uintptr_t)status % 4)
    return invalid("null positions, or positions, sequences or status misaligned");
  const bool listed = n_seq > 0 && width > 0;
  if (listed && (!table || (uintptr_t)table % 4)) return invalid("null or misaligned table");
  if (listed && (ld_table < width || ld_table > (int64_t(1) << 40)))
    return invalid("ld_table must be at least the width");
  // what is written is apart from what every wave reads
  const struct {
    const void* p;
    size_t bytes;
  } ro[3] = {{pos, rows * sizeof(int32_t)},
             {seq, seq ? rows * sizeof(int32_t) : 0},
             {table, listed ? ((n_seq - 1) * (size_t)ld_table + width) * sizeof(int32_t) : 0}};
  for (const auto& r : ro) {
    if (ranges_meet(r.p, r.bytes, status, status ? 4 : 0)) return invalid("status shares memory with another buffer");
    if (read ? sides_meet_range(s, 2, r.p, r.bytes, d, esz) : cache_meets(*cache, r.p, r.bytes))
      return invalid("an output shares memory with the table, sequences or positions");
  }
  if (cache_meets(*cache, status, status ? 4 : 0) || sides_meet_range(s, 2, status, status ? 4 : 0, d, esz))
    return invalid("status shares memory with another buffer");
  for (const Side& x : s)
    if (cache_meets(*cache, x.v, rows, esz)) return invalid("rows share memory with the cache");
  return MPIPE_OK;
}

}  // namespace

extern "C" {

mpipe_status mpipe_op_causal_attention_fwd(int32_t dtype, int32_t head_dim, int64_t rows_q,
                                           int64_t rows_k, const mpipe_heads* q,
                                           const mpipe_heads* k, const mpipe_heads* v,
                                           const int64_t* seq_row, const int64_t* seq_len,
                                           const int64_t* key_row, const int64_t* key_len,
                                           int32_t n_seq, float scale, const mpipe_heads* o,
                                           float* lse, int64_t ld_lse, void* stream) {
  return guarded([&]() -> mpipe_status {
    CausalProblem p;
    const mpipe_heads* in[5] = {q, k, v, nullptr, nullptr};
    const mpipe_heads* out[3] = {o, nullptr, nullptr};
    if (mpipe_status st = check_causal(p, dtype, head_dim, rows_q, rows_k, in, out, false, seq_row,
                                       seq_len, key_row, key_len, n_seq, scale, lse, ld_lse,
                                       nullptr, 0))
      return st;
    if (p.q.heads == 0) return MPIPE_OK;
    return hip_status(causal_attention_fwd(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

size_t mpipe_op_causal_attention_scratch_bytes(int64_t rows_q, int32_t heads_q, int64_t rows_k,
                                               int32_t heads_k, int32_t head_dim) {
  if (rows_q < 0 || rows_q > (1 << 30) || rows_k < 0 || rows_k > (1 << 30) || heads_q < 0 ||
      heads_q > 65536 || heads_k < 0 || heads_k > heads_q || (heads_q > 0 && heads_k == 0) ||
      (heads_k > 0 && heads_q % heads_k) || !dim_ok(head_dim))
    return 0;
  return causal_attention_scratch(rows_q, heads_q, rows_k, heads_k, head_dim);
}

mpipe_status mpipe_op_causal_attention_bwd(int32_t dtype, int32_t head_dim, int64_t rows_q,
                                           int64_t rows_k, const mpipe_heads* d_o,
                                           const mpipe_heads* q, const mpipe_heads* k,
                                           const mpipe_heads* v, const mpipe_heads* o,
                                           const float* lse, int64_t ld_lse,
                                           const int64_t* seq_row, const int64_t* seq_len,
                                           const int64_t* key_row, const int64_t* key_len,
                                           int32_t n_seq, float scale, const mpipe_heads* dq,
                                           const mpipe_heads* dk, const mpipe_heads* dv,
                                           void* scratch, size_t scratch_bytes, void* stream) {
  return guarded([&]() -> mpipe_status {
    CausalProblem p;
    const mpipe_heads* in[5] = {q, k, v, o, d_o};
    const mpipe_heads* out[3] = {dq, dk, dv};
    if (mpipe_status st = check_causal(p, dtype, head_dim, rows_q, rows_k, in, out, true, seq_row,
                                       seq_len, key_row, key_len, n_seq, scale,
                                       const_cast<float*>(lse), ld_lse, scratch, scratch_bytes))
      return st;
    if (p.q.heads == 0) return MPIPE_OK;
    return hip_status(causal_attention_bwd(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

mpipe_status mpipe_op_cache_write(const mpipe_kv_cache* cache, int32_t dtype, int64_t rows,
                                  const mpipe_heads* k, const mpipe_heads* v,
                                  const int32_t* table, int64_t ld_table, int32_t n_seq,
                                  int32_t width, const int32_t* seq, const int32_t* pos,
                                  int32_t* status, void* stream) {
  return guarded([&]() -> mpipe_status {
    CacheRows p;
    if (mpipe_status st = check_rows(p, cache, dtype, rows, k, v, table, ld_table, n_seq, width,
                                     seq, pos, status, false))
      return st;
    return hip_status(cache_write(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

mpipe_status mpipe_op_cache_read(const mpipe_kv_cache* cache, int32_t dtype, int64_t rows,
                                 const int32_t* table, int64_t ld_table, int32_t n_seq,
                                 int32_t width, const int32_t* seq, const int32_t* pos,
                                 const mpipe_heads* k, const mpipe_heads* v, int32_t* status,
                                 void* stream) {
  return guarded([&]() -> mpipe_status {
    CacheRows p;
    if (mpipe_status st = check_rows(p, cache, dtype, rows, k, v, table, ld_table, n_seq, width,
                                     seq, pos, status, true))
      return st;
    return hip_status(cache_read(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

size_t mpipe_op_cache_attention_scratch_bytes(int32_t n_seq, int32_t heads_q, int32_t heads_k,
                                              int32_t head_dim) {
  if (n_seq < 0 || heads_q < 1 || heads_q > 65536 || heads_k < 1 || heads_q % heads_k ||
      !dim_ok(head_dim))
    return 0;
  return cache_attention_scratch(n_seq, head_dim);
}

mpipe_status mpipe_op_cache_attention(const mpipe_kv_cache* cache, int32_t dtype, int32_t n_seq,
                                      const mpipe_heads* q, const int32_t* table,
                                      int64_t ld_table, int32_t width, const int32_t* lens,
                                      float scale, const mpipe_heads* o, float* lse,
                                      int64_t ld_lse, void* scratch, size_t scratch_bytes,
                                      void* stream) {
  return guarded([&]() -> mpipe_status {
    std::string why;
    if (mpipe_status st = cache_ok(cache, why)) return set_error(st, why);
    if (dtype != MPIPE_F32 && dtype != MPIPE_BF16) return invalid("bad dtype");
    if (cache->dtype != MPIPE_E4M3 && cache->dtype != dtype)
      return set_error(MPIPE_ERR_UNSUPPORTED, "q and the cache differ in type");
    if (n_seq < 0 || width < 0) return invalid("negative table size");
    if (!scale_ok(scale)) return invalid("scale must be positive and finite");
    const int esz = esz_of(dtype), d = cache->head_dim;
    const Side s[2] = {side_of(q, n_seq, false), side_of(o, n_seq, true)};
    const int hq = s[0].v.heads;
    if (hq != s[1].v.heads) return invalid("q and o of different head counts");
    if (mpipe_status st = heads_ok(hq, cache->heads)) return st;
    if ((int64_t)n_seq * hq > (1 << 23))
      return set_error(MPIPE_ERR_UNSUPPORTED, "more than 2^23 heads of all sequences");
    if (mpipe_status st = sides_ok(s, 2, d, esz)) return st;
    size_t lse_bytes = 0;
    if (mpipe_status st = stats_ok(lse, ld_lse, n_seq, hq, lse_bytes)) return st;
    if (n_seq == 0) return MPIPE_OK;
    if (cache->n_pages == 0) return invalid("a cache of no pages");
    if (!lens || (uintptr_t)lens % 4) return invalid("null or misaligned lengths");
    if (width > 0 && (!table || (uintptr_t)table % 4)) return invalid("null or misaligned table");
    if (width > 0 && (ld_table < width || ld_table > (int64_t(1) << 40)))
      return invalid("ld_table must be at least the width");
    if ((int64_t)width * cache->page > INT32_MAX)
      return set_error(MPIPE_ERR_UNSUPPORTED, "a table of more than 2^31 - 1 tokens");
    const size_t need = cache_attention_scratch(n_seq, d);
    if (!scratch || scratch_bytes < need) return set_error(MPIPE_ERR_WORKSPACE, "scratch too small");
    if ((uintptr_t)scratch % 16) return invalid("scratch misaligned");
    const struct {
      const void* p;
      size_t bytes;
    } ro[2] = {{lens, n_seq * sizeof(int32_t)},
               {table, width > 0 ? ((n_seq - 1) * (size_t)ld_table + width) * sizeof(int32_t) : 0}};
    for (const auto& r : ro)
      if (range_meets(r.p, r.bytes, s[1].v, n_seq, d, esz) || ranges_meet(r.p, r.bytes, lse, lse_bytes) ||
          ranges_meet(r.p, r.bytes, scratch, need))
        return invalid("an output or scratch shares memory with the table or lengths");
    if (sides_meet_range(s, 2, lse, lse_bytes, d, esz) || sides_meet_range(s, 2, scratch, need, d, esz) ||
        ranges_meet(lse, lse_bytes, scratch, need))
      return invalid("lse or scratch shares memory with another buffer");
    if (cache_meets(*cache, s[1].v, n_seq, esz) || cache_meets(*cache, lse, lse_bytes) ||
        cache_meets(*cache, scratch, need))
      return invalid("an output or scratch shares memory with the cache");
    CacheAttention p;
    p.cache = *cache;
    p.dtype = dtype;
    p.n_seq = n_seq;
    p.width = width;
    p.q = s[0].v;
    p.o = s[1].v;
    p.table = table;
    p.ld_table = ld_table;
    p.lens = lens;
    p.scale = scale;
    p.lse = lse;
    p.ld_lse = ld_lse;
    p.scratch = reinterpret_cast<float*>(scratch);
    return hip_status(cache_attention(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

}  // extern "C"
