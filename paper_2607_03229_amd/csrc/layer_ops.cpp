// Entry points of the operators around the first LLM layer and of the gradient's norm
// (include/mpipe_ops.h): every check on the host, then the launches.
#include <algorithm>
#include <cmath>
#include <exception>
#include <string>

#include "layer_kernels.h"

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

// The reciprocal root takes no subnormal, and from 2^-126 on squares that underflow (below
// 2^-150 each) stay under an fp32 step of the mean.
bool eps_ok(float eps) { return eps >= 0x1p-126f && std::isfinite(eps); }
constexpr const char* kBadEps = "eps must be finite and at least 2^-126";

HeadView view_of(const mpipe_heads* h) {
  HeadView v;
  if (h) {
    v.p = h->p;
    v.row = h->row_stride;
    v.head = h->head_stride;
    v.heads = h->heads;
  }
  return v;
}

// The checks all three rotations share; fills p.
mpipe_status check_qk(QkProblem& p, int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                      const mpipe_heads* in[2], const mpipe_heads* grad[2],
                      const mpipe_heads* out[2], const void* const gain[2], const int32_t* pos,
                      int64_t ld_pos) {
  if (dtype != MPIPE_F32 && dtype != MPIPE_BF16) return set_error(MPIPE_ERR_INVALID_ARG, "bad dtype");
  std::string why;
  if (mpipe_status st = rope_axes_table(cfg, p.table, why)) return set_error(st, why);
  if (rows < 0) return set_error(MPIPE_ERR_INVALID_ARG, "negative row count");
  if (rows > (1 << 30)) return set_error(MPIPE_ERR_UNSUPPORTED, "more than 2^30 rows");
  const int esz = dtype == MPIPE_BF16 ? 2 : 4, d = cfg->head_dim;
  p.dtype = dtype;
  p.head_dim = d;
  p.rot_dim = cfg->rot_dim;
  p.adjacent = cfg->pairing == MPIPE_ROPE_ADJACENT;
  p.rows = rows;
  p.pos = pos;
  p.ld_pos = ld_pos;
  bool any = false;
  for (int z = 0; z < 2; ++z) {
    QkSide& s = p.side[z];
    s.x = view_of(in[z]);
    s.y = view_of(out[z]);
    if (grad) s.dy = view_of(grad[z]);
    if (s.x.heads != s.y.heads || (grad && s.x.heads != s.dy.heads))
      return set_error(MPIPE_ERR_INVALID_ARG, "inputs and outputs of different head counts");
    if (s.x.heads > 65536) return set_error(MPIPE_ERR_UNSUPPORTED, "more than 65536 heads");
    if (!view_ok(s.x, rows, d, esz, false, why) || !view_ok(s.y, rows, d, esz, true, why) ||
        (grad && !view_ok(s.dy, rows, d, esz, false, why)))
      return set_error(MPIPE_ERR_INVALID_ARG, why);
    if (s.x.heads == 0 || rows == 0) continue;
    any = true;
    s.gain = gain ? gain[z] : nullptr;
    if (gain && (!s.gain || (uintptr_t)s.gain % esz))
      return set_error(MPIPE_ERR_INVALID_ARG, "a null gain, or one not aligned to its elements");
  }
  if (!any) return MPIPE_OK;
  if (!pos || (uintptr_t)pos % 4) return set_error(MPIPE_ERR_INVALID_ARG, "null or misaligned positions");
  if (cfg->axes > 1 && ld_pos != 0 && (ld_pos < rows || ld_pos > (int64_t(1) << 40)))
    return set_error(MPIPE_ERR_INVALID_ARG, "ld_pos must be at least rows, or 0");
  // an output meets an input only in place, on its own side, and never another output
  for (int z = 0; z < 2; ++z) {
    const HeadView& y = p.side[z].y;
    if (views_meet(y, p.side[1 - z].y, rows, d, esz))
      return set_error(MPIPE_ERR_INVALID_ARG, "the outputs of q and k share memory");
    for (int w = 0; w < 2; ++w)
      for (const HeadView* v : {&p.side[w].x, &p.side[w].dy})
        if (!(w == z && same_view(y, *v, rows)) && views_meet(y, *v, rows, d, esz))
          return set_error(MPIPE_ERR_INVALID_ARG, "an output shares memory with another view");
    // what every wave reads stays as it is while outputs are written
    for (int a = 0; a < cfg->axes; ++a)
      if (range_meets(pos + a * (cfg->axes > 1 ? ld_pos : 0), rows * sizeof(int32_t), y, rows, d, esz))
        return set_error(MPIPE_ERR_INVALID_ARG, "an output shares memory with the positions");
    for (const QkSide& s : p.side)
      if (s.gain && range_meets(s.gain, (size_t)d * esz, y, rows, d, esz))
        return set_error(MPIPE_ERR_INVALID_ARG, "an output shares memory with a gain");
  }
  return MPIPE_OK;
}

// The gain gradients and the scratch of a backward: gradients apart from each other and from
// the outputs; scratch, which blocks write while others still read, apart from everything.
mpipe_status check_gain_grads(const QkProblem& p, int axes, const void* scratch, size_t bytes) {
  const int esz = p.dtype == MPIPE_BF16 ? 2 : 4, d = p.head_dim;
  const size_t gb = d * sizeof(float);
  const QkSide &q = p.side[0], &k = p.side[1];
  if (q.grad && k.grad && ranges_meet(q.grad, gb, k.grad, gb))
    return set_error(MPIPE_ERR_INVALID_ARG, "the gain gradients share memory");
  for (const QkSide& s : p.side) {
    if (s.grad && (range_meets(s.grad, gb, q.y, p.rows, d, esz) ||
                   range_meets(s.grad, gb, k.y, p.rows, d, esz)))
      return set_error(MPIPE_ERR_INVALID_ARG, "a gain gradient shares memory with an output");
    bool meets = s.grad && ranges_meet(scratch, bytes, s.grad, gb);
    meets |= s.gain && ranges_meet(scratch, bytes, s.gain, (size_t)d * esz);
    for (const HeadView* v : {&s.x, &s.dy, &s.y}) meets |= range_meets(scratch, bytes, *v, p.rows, d, esz);
    if (meets) return set_error(MPIPE_ERR_INVALID_ARG, "scratch shares memory with another buffer");
  }
  for (int a = 0; a < axes && q.x.heads + k.x.heads > 0 && p.rows > 0; ++a)
    if (ranges_meet(scratch, bytes, p.pos + a * (axes > 1 ? p.ld_pos : 0), p.rows * sizeof(int32_t)))
      return set_error(MPIPE_ERR_INVALID_ARG, "scratch shares memory with another buffer");
  return MPIPE_OK;
}

}  // namespace

extern "C" {

mpipe_status mpipe_op_seam_positions(const int64_t* seq_row, const int64_t* seq_len,
                                     const int64_t* seq_pos, int32_t n_seq,
                                     const int64_t* item_row, const int32_t* grid_thw,
                                     const int32_t* time_step, int32_t n_items, int64_t n_rows,
                                     int32_t* pos, int64_t ld_pos, int64_t* next, void* stream) {
  return guarded([&]() -> mpipe_status {
    std::vector<PosSpan> spans;
    std::vector<int64_t> last(n_seq > 0 ? n_seq : 0);
    std::string why;
    int64_t end = 0;
    if (ld_pos < n_rows || ld_pos > (int64_t(1) << 40))
      return set_error(MPIPE_ERR_INVALID_ARG, "ld_pos must be at least n_rows");
    if (mpipe_status st = position_spans(seq_row, seq_len, seq_pos, n_seq, item_row, grid_thw,
                                         time_step, n_items, n_rows, last.data(), spans, end, why))
      return set_error(st, why);
    if (!spans.empty() && (!pos || (uintptr_t)pos % 4))
      return set_error(MPIPE_ERR_INVALID_ARG, "null or misaligned positions");
    const mpipe_status st = hip_status(
        seam_positions(spans, end, pos, ld_pos, reinterpret_cast<hipStream_t>(stream)));
    if (st == MPIPE_OK && next) std::copy(last.begin(), last.end(), next);
    return st;
  });
}

mpipe_status mpipe_op_rope_axes(int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                                const mpipe_heads* q, const mpipe_heads* k, const int32_t* pos,
                                int64_t ld_pos, int32_t inverse, const mpipe_heads* q_out,
                                const mpipe_heads* k_out, void* stream) {
  return guarded([&]() -> mpipe_status {
    QkProblem p;
    const mpipe_heads* in[2] = {q, k};
    const mpipe_heads* out[2] = {q_out, k_out};
    if (mpipe_status st = check_qk(p, dtype, cfg, rows, in, nullptr, out, nullptr, pos, ld_pos)) return st;
    p.inverse = inverse != 0;
    return hip_status(qk_rope_fwd(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

mpipe_status mpipe_op_qk_norm_rope_fwd(int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                                       const mpipe_heads* q, const mpipe_heads* k,
                                       const void* q_gain, const void* k_gain, float eps,
                                       const int32_t* pos, int64_t ld_pos,
                                       const mpipe_heads* q_out, const mpipe_heads* k_out,
                                       void* stream) {
  return guarded([&]() -> mpipe_status {
    QkProblem p;
    const mpipe_heads* in[2] = {q, k};
    const mpipe_heads* out[2] = {q_out, k_out};
    const void* gain[2] = {q_gain, k_gain};
    if (!eps_ok(eps)) return set_error(MPIPE_ERR_INVALID_ARG, kBadEps);
    if (mpipe_status st = check_qk(p, dtype, cfg, rows, in, nullptr, out, gain, pos, ld_pos)) return st;
    p.norm = true;
    p.eps = eps;
    return hip_status(qk_rope_fwd(p, reinterpret_cast<hipStream_t>(stream)));
  });
}

size_t mpipe_op_qk_norm_rope_scratch_bytes(int64_t rows, int32_t heads_q, int32_t heads_k,
                                           int32_t head_dim) {
  if (rows < 0 || rows > (1 << 30) || heads_q < 0 || heads_q > 65536 || heads_k < 0 ||
      heads_k > 65536 || head_dim < 8 || head_dim > kMaxHeadDim)
    return 0;
  return qk_norm_rope_bwd_scratch(rows, heads_q, heads_k, head_dim);
}

mpipe_status mpipe_op_qk_norm_rope_bwd(int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                                       const mpipe_heads* dq, const mpipe_heads* dk,
                                       const mpipe_heads* q, const mpipe_heads* k,
                                       const void* q_gain, const void* k_gain, float eps,
                                       const int32_t* pos, int64_t ld_pos,
                                       const mpipe_heads* dq_in, const mpipe_heads* dk_in,
                                       float* grad_q_gain, float* grad_k_gain, int32_t accumulate,
                                       void* scratch, size_t scratch_bytes, void* stream) {
  return guarded([&]() -> mpipe_status {
    QkProblem p;
    const mpipe_heads* in[2] = {q, k};
    const mpipe_heads* grad[2] = {dq, dk};
    const mpipe_heads* out[2] = {dq_in, dk_in};
    const void* gain[2] = {q_gain, k_gain};
    if (!eps_ok(eps)) return set_error(MPIPE_ERR_INVALID_ARG, kBadEps);
    if (mpipe_status st = check_qk(p, dtype, cfg, rows, in, grad, out, gain, pos, ld_pos)) return st;
    if ((uintptr_t)grad_q_gain % 4 || (uintptr_t)grad_k_gain % 4)
      return set_error(MPIPE_ERR_INVALID_ARG, "gain gradients misaligned");
    p.norm = p.inverse = true;
    p.eps = eps;
    p.side[0].grad = grad_q_gain;
    p.side[1].grad = grad_k_gain;
    const size_t need = qk_norm_rope_bwd_scratch(rows, p.side[0].x.heads, p.side[1].x.heads, p.head_dim);
    const bool sums = (grad_q_gain || grad_k_gain) && rows > 0;
    if (sums && (!scratch || scratch_bytes < need))
      return set_error(MPIPE_ERR_WORKSPACE, "scratch too small");
    if ((uintptr_t)scratch % 4) return set_error(MPIPE_ERR_INVALID_ARG, "scratch misaligned");
    if (mpipe_status st = check_gain_grads(p, cfg->axes, scratch, sums ? need : 0)) return st;
    return hip_status(qk_norm_rope_bwd(p, accumulate != 0, reinterpret_cast<float*>(scratch),
                                       reinterpret_cast<hipStream_t>(stream)));
  });
}

size_t mpipe_op_grad_scratch_bytes(const mpipe_grad_tensor* grads, int32_t n) {
  size_t bytes = 0;
  guarded([&]() -> mpipe_status {
    GradPlan p;
    std::string why;
    if (mpipe_status st = grad_plan(grads, n, p, why)) return set_error(st, why);
    bytes = grad_norm_scratch(n, p);
    return MPIPE_OK;
  });
  return bytes;
}

mpipe_status mpipe_op_grad_norm(const mpipe_grad_tensor* grads, int32_t n, double* sumsq,
                                float* norms, void* scratch, size_t scratch_bytes, void* stream) {
  return guarded([&]() -> mpipe_status {
    GradPlan p;
    std::string why;
    if (mpipe_status st = grad_plan(grads, n, p, why)) return set_error(st, why);
    if (!sumsq || (uintptr_t)sumsq % 8 || (uintptr_t)norms % 4)
      return set_error(MPIPE_ERR_INVALID_ARG, "null or misaligned result");
    const size_t need = grad_norm_scratch(n, p), norms_bytes = norms ? n * sizeof(float) : 0;
    if (!scratch || scratch_bytes < need) return set_error(MPIPE_ERR_WORKSPACE, "scratch too small");
    if ((uintptr_t)scratch % 8) return set_error(MPIPE_ERR_INVALID_ARG, "scratch misaligned");
    if (ranges_meet(sumsq, sizeof(double), norms, norms_bytes) ||
        ranges_meet(scratch, need, sumsq, sizeof(double)) ||
        ranges_meet(scratch, need, norms, norms_bytes))
      return set_error(MPIPE_ERR_INVALID_ARG, "results or scratch share memory");
    if (list_meets(grads, n, sumsq, sizeof(double)) || list_meets(grads, n, norms, norms_bytes) ||
        list_meets(grads, n, scratch, need))
      return set_error(MPIPE_ERR_INVALID_ARG, "a result or scratch shares memory with a gradient");
    return hip_status(grad_norm(grads, n, p, sumsq, norms, reinterpret_cast<char*>(scratch),
                                reinterpret_cast<hipStream_t>(stream)));
  });
}

mpipe_status mpipe_op_grad_clip(const mpipe_grad_tensor* grads, const mpipe_grad_tensor* out,
                                int32_t n, const double* sumsq, double max_norm, float* norm,
                                void* stream) {
  return guarded([&]() -> mpipe_status {
    GradPlan p;
    std::string why;
    if (mpipe_status st = grad_plan(grads, n, p, why)) return set_error(st, why);
    if (!out) out = grads;
    if (out != grads)
      if (mpipe_status st = grad_outputs_ok(grads, out, n, why)) return set_error(st, why);
    if (!sumsq || (uintptr_t)sumsq % 8 || (uintptr_t)norm % 4)
      return set_error(MPIPE_ERR_INVALID_ARG, "null sumsq, or a misaligned result");
    // read by every block, or written by one, while others read gradients and write outputs
    const size_t norm_bytes = norm ? sizeof(float) : 0;
    if (ranges_meet(sumsq, sizeof(double), norm, norm_bytes))
      return set_error(MPIPE_ERR_INVALID_ARG, "norm shares memory with sumsq");
    if (list_meets(out, n, sumsq, sizeof(double)) || list_meets(out, n, norm, norm_bytes) ||
        (out != grads && list_meets(grads, n, norm, norm_bytes)))
      return set_error(MPIPE_ERR_INVALID_ARG, "norm or sumsq shares memory with a tensor");
    if (!(max_norm >= 0.0)) return set_error(MPIPE_ERR_INVALID_ARG, "max_norm must be 0 or more");
    return hip_status(grad_clip(grads, out, n, p, sumsq, max_norm, norm,
                                reinterpret_cast<hipStream_t>(stream)));
  });
}

}  // extern "C"
