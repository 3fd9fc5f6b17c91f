/*
 * libmpipe kernel-level entry points.
 *
 * The encoder step of mpipe.h is a sequence of these operations; they are
 * exported individually so that each gfx950 kernel can be checked against the
 * CPU oracle's building block of the same name.  Same conventions as mpipe.h:
 * device pointers unless marked host, row-major, work enqueued on hip_stream,
 * status return, nothing enqueued on a non-OK status.  Calls that upload host
 * metadata (segment tables, positions) synchronize hip_stream before returning.
 */
#ifndef MPIPE_OPS_H
#define MPIPE_OPS_H
#include "mpipe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Layouts: 0 NT  C[m][n] = sum_k A[m][k] B[n][k]     (Linear forward, Y = X W^T)
 *          1 NN  C[m][n] = sum_k A[m][k] B[k][n]     (input gradient, dX = dY W)
 *          2 TN  C[m][n] = sum_k A[k][m] B[k][n]     (weight gradient, dW = dY^T X)
 * Epilogues (acc = the sum, bias per column, cfg dtype unless noted):
 *          0 C = acc + bias
 *          1 u = acc + bias rounded to dtype: C = GELU(u), C2 = GELU'(u) (C2 optional).
 *            GELU is the erf form: fp32 evaluates erf exactly; bf16 uses the
 *            Abramowitz & Stegun 7.1.26 erf (|error| <= 1.5e-7), in every kernel.
 *          2 C(fp32) = aux(fp32, nullable, may alias C) + acc + bias
 *          3 C = acc * aux   (aux = the GELU'(u) that epilogue 1 stored: the MLP backward)
 *          4 C(fp32) = acc, or C + acc when beta != 0; with k_per_split > 0 the
 *            K range is split and split s writes C + s * split_stride.
 * Requirements: K-contiguous operands need K and their row stride to be
 * multiples of 8 (bf16) / 4 (fp32); K-major operands need their column count
 * and row stride to be multiples of 8 / 4; 16-byte aligned pointers. */
mpipe_status mpipe_op_gemm(int32_t dtype, int32_t layout, int32_t epilogue, int32_t M, int32_t N,
                           int32_t K, const void* A, int64_t lda, const void* B, int64_t ldb,
                           void* C, int64_t ldc, const void* bias, const void* aux, int64_t ld_aux,
                           void* C2, int64_t ldc2, int32_t beta, int32_t k_per_split,
                           int64_t split_stride, void* hip_stream);

/* The kernel mpipe_op_gemm runs a product on (host query, no device work), for dense
 * operands on 16 bytes: 0 general 128x128, 1 fp32 32x32 tiles, 2 / 3 / 4 bf16 tiles of
 * 64x64 / 64x128 / 128x128, 5 the large bf16 tiles (128x256 for NN, 256x256 for NT and
 * TN).  -1 for arguments out of range. */
int32_t mpipe_op_gemm_kernel(int32_t dtype, int32_t layout, int32_t epilogue, int32_t M,
                             int32_t N, int32_t K, int32_t k_per_split);

/* Deterministic split-K reduction of the weight gradient (the Accumulate edge of
 * Sec. 4.1: gradients are added into what the buffer holds):
 *   out[m][n] += sum over s = 0 .. splits-1, in that order, of part[s][m][n]
 * part: fp32 [splits][M][N] dense (the partials epilogue 4 writes with split_stride
 * M*N); out: fp32 [M][ldo], ldo >= N.  Four columns per thread when N and ldo are
 * multiples of 4 and both pointers 16-byte aligned, one column per thread otherwise;
 * both paths add in the same order. */
mpipe_status mpipe_op_splitk_reduce(const float* part, int32_t splits, int64_t M, int64_t N,
                                    float* out, int64_t ldo, void* hip_stream);

/* The number of K splits the encoder backward gives the weight-gradient product
 * dW[M][N] = sum over K tokens (host query, no device work): 1 means one unsplit
 * launch accumulating into d_weights; s > 1 means s fp32 partials then
 * mpipe_op_splitk_reduce.  -1 for negative sizes. */
int32_t mpipe_op_weight_grad_splits(int64_t M, int64_t N, int64_t K);

/* LayerNorm over rows of width n (n % 4 == 0, n <= 2048): X fp32 [rows][n];
 * g, b, Y in dtype; mean, rstd fp32 [rows] (nullable). */
mpipe_status mpipe_op_layernorm_fwd(int32_t dtype, const float* X, int64_t rows, int32_t n,
                                    const void* g, const void* b, float eps, void* Y, float* mean,
                                    float* rstd, void* hip_stream);

/* LayerNorm backward: dX = dres + LN'(dY) (fp32), dXt = the same in dtype
 * (nullable), grad_g / grad_b += column sums of dY*xhat and dY, colsum_dx +=
 * column sums of dX (the bias gradient of the product whose output gradient dX
 * is), all fp32 [n] and nullable.  scratch: at least
 * mpipe_op_scratch_bytes(rows, 1, n, 0) bytes. */
mpipe_status mpipe_op_layernorm_bwd(int32_t dtype, const float* dY, const float* X,
                                    const float* mean, const float* rstd, const void* g,
                                    int64_t rows, int32_t n, const float* dres, float* dX,
                                    void* dXt, float* grad_g, float* grad_b, float* colsum_dx,
                                    void* scratch, size_t scratch_bytes, void* hip_stream);

/* 2D rotary position, in place on the q and k blocks of qkv [rows][3*heads*d]
 * (inverse != 0 rotates back: the backward).  Positions come from grid_thw
 * (host) in the packed row order of mpipe.h. */
mpipe_status mpipe_op_rope(int32_t dtype, void* qkv, int64_t rows, int32_t heads, int32_t head_dim,
                           const int32_t* grid_thw, int32_t n_items, float theta, int32_t inverse,
                           void* scratch, size_t scratch_bytes, void* hip_stream);

/* Block-diagonal attention over segments cu_seqlens (host) of qkv [N][3*heads*d]
 * (columns q | k | v, head j at j*d).  o: [N][heads*d]; lse: fp32 [heads][N]
 * natural-log sum-exp of the scaled scores. */
mpipe_status mpipe_op_attention_fwd(int32_t dtype, const void* qkv, int64_t N, int32_t heads,
                                    int32_t head_dim, const int32_t* cu_seqlens, int32_t n_seg,
                                    void* o, float* lse, void* scratch, size_t scratch_bytes,
                                    void* hip_stream);

/* Attention backward: dqkv [N][3*heads*d] overwritten with dQ | dK | dV. */
mpipe_status mpipe_op_attention_bwd(int32_t dtype, const void* qkv, const void* o, const void* d_o,
                                    const float* lse, int64_t N, int32_t heads, int32_t head_dim,
                                    const int32_t* cu_seqlens, int32_t n_seg, void* dqkv,
                                    void* scratch, size_t scratch_bytes, void* hip_stream);

/* Scratch bytes the ops above need for rows N, heads, width n and n_seg segments. */
size_t mpipe_op_scratch_bytes(int64_t N, int32_t heads, int32_t n, int32_t n_seg);

/* ---- The first LLM layer behind the seam, and the end of a trained step ----------------
 * What a step does next with the rows mpipe_merge_scatter placed and with the gradient
 * mpipe_encoder_bwd accumulated.  None of these calls synchronizes, allocates device memory
 * or keeps anything: metadata and tables travel in the kernels' arguments, so every call can
 * be captured into a graph, and a replay reads the buffers anew (host arguments stay as
 * captured).  The current device has to be that of the stream and the buffers.  Calls that
 * overlap need scratch and results of their own. */

/* Positions of the LLM's input rows on three axes (time, height, width): pos[axis * ld_pos
 * + row], device int32, for every row of the sequences; other rows are not written.
 *   seq_row, seq_len  host [n_seq]: sequence s is the rows seq_row[s] .. + seq_len[s] of the
 *                     n_rows rows (padded batches leave gaps; an empty one is allowed).
 *                     Sequences must not overlap; any order.
 *   seq_pos           host [n_seq], nullable (all 0): the first position of each sequence, for
 *                     sequences that go on (the next token of a running one).
 *   item_row          host [n_items]: first row of each item's merged rows, which are adjacent
 *                     and in the order of mpipe.h (tau, hb, wb); any order, each inside one
 *                     sequence, none overlapping.
 *   grid_thw          host [n_items][3], in patches as for the encoder (gh, gw even).
 *   time_step         host [n_items], nullable (all 1): positions from slice to slice, >= 0.
 * With p = the sequence's first position, rows in order: a text row gets (p, p, p) and p += 1;
 * an item of t slices of h x w merged rows gets (p + time_step * tau, p + y, p + x), then
 * p += max(time_step * (t - 1) + 1, h, w).  next: host int64 [n_seq], nullable: p after each
 * sequence's last row.  Positions reach 2^31 - 1 at most; an item 2^28 rows. */
mpipe_status mpipe_op_seam_positions(const int64_t* seq_row, const int64_t* seq_len,
                                     const int64_t* seq_pos, int32_t n_seq,
                                     const int64_t* item_row, const int32_t* grid_thw,
                                     const int32_t* time_step, int32_t n_items, int64_t n_rows,
                                     int32_t* pos, int64_t ld_pos, int64_t* next,
                                     void* hip_stream);

/* Rotary positions with several axes.  The first rot_dim columns of a head are rot_dim / 2
 * pairs; pair i turns by pos[axis(i)][row] * freq(i), the columns behind them pass through.
 *   order     MPIPE_ROPE_BLOCKS: the first section[0] pairs belong to axis 0, the next
 *             section[1] to axis 1, ...; MPIPE_ROPE_INTERLEAVED: pair i belongs to axis
 *             a = i mod axes while i / axes < section[a], else to axis 0 (the sections must
 *             come out as the number of pairs of each axis).
 *   spectrum  MPIPE_ROPE_ONE_SPECTRUM: freq(i) = theta^(-2i / rot_dim) over all pairs;
 *             MPIPE_ROPE_AXIS_SPECTRA: theta^(-c / section[a]) for the c-th pair of axis a
 *             (axes 2, sections d/4 and d/4 in blocks: the encoder's (y, x)).
 *   pairing   MPIPE_ROPE_HALVES: columns (i, i + rot_dim / 2); MPIPE_ROPE_ADJACENT:
 *             columns (2i, 2i + 1).
 * head_dim and rot_dim: multiples of 8, 8 <= rot_dim <= head_dim <= 256; theta > 1; the
 * sections sum to rot_dim / 2 (zeros allowed). */
#define MPIPE_ROPE_MAX_AXES 4
typedef enum { MPIPE_ROPE_BLOCKS = 0, MPIPE_ROPE_INTERLEAVED = 1 } mpipe_rope_order;
typedef enum { MPIPE_ROPE_ONE_SPECTRUM = 0, MPIPE_ROPE_AXIS_SPECTRA = 1 } mpipe_rope_spectrum;
typedef enum { MPIPE_ROPE_HALVES = 0, MPIPE_ROPE_ADJACENT = 1 } mpipe_rope_pairing;
typedef struct {
  int32_t head_dim, rot_dim, axes;
  int32_t section[MPIPE_ROPE_MAX_AXES];
  int32_t order, spectrum, pairing;
  double theta;
} mpipe_rope_cfg;

/* Heads of q or k: element (row, head, column) at p[row * row_stride + head * head_stride +
 * column], strides in elements, aligned to one element; heads == 0: none (p may be null).
 * Inputs take any strides >= 0.  An output's elements must be distinct, and it may share
 * memory with an input only as the very same view of the same side (in place), or as other
 * columns of rows of one stride (q, k and v of one product, side by side or head by head); never
 * with positions or gains. */
typedef struct {
  void* p;
  int64_t row_stride, head_stride;
  int32_t heads;
} mpipe_heads;

/* q_out, k_out = q, k turned by the positions pos[axis * ld_pos + row] (device int32, any
 * values; ld_pos at least rows, or 0: one row of positions for all axes, as text has them);
 * inverse != 0 turns back, which is the gradient.  Angles keep their phase at any position
 * (whole-number products modulo one turn); arithmetic in fp32, one rounding. */
mpipe_status mpipe_op_rope_axes(int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                                const mpipe_heads* q, const mpipe_heads* k, const int32_t* pos,
                                int64_t ld_pos, int32_t inverse, const mpipe_heads* q_out,
                                const mpipe_heads* k_out, void* hip_stream);

/* The same behind a root-mean-square norm of every head, in one pass: n = g * x * r,
 * r = 1 / sqrt(mean of x^2 over head_dim + eps), then the rotation.  q_gain, k_gain:
 * [head_dim] in dtype; eps finite, at least 2^-126.  Statistics and arithmetic in fp32 (|x| below
 * 1e18, as squares are summed), one rounding.  The backward needs q and k as they went in: in
 * place only without it. */
mpipe_status mpipe_op_qk_norm_rope_fwd(int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                                       const mpipe_heads* q, const mpipe_heads* k,
                                       const void* q_gain, const void* k_gain, float eps,
                                       const int32_t* pos, int64_t ld_pos,
                                       const mpipe_heads* q_out, const mpipe_heads* k_out,
                                       void* hip_stream);

/* Its backward from dq, dk (gradients of q_out, k_out) and the forward's q, k, gains, eps and
 * positions; the norms' statistics are recomputed.  dq_in, dk_in: overwritten with the
 * gradients of q and k (may be the same views as dq, dk or as q, k).  grad_q_gain,
 * grad_k_gain: fp32 [head_dim], nullable, apart from each other and from dq_in and dk_in;
 * accumulate != 0 adds into them (the Accumulate edge), else they are overwritten, also where
 * there are no rows.  Every row counts in them: leave rows of padding out of the call (a call
 * per sequence, accumulating), or give them finite q, k and zero dq, dk.  Summed in a fixed
 * order: the same call gives the same bits.  scratch: mpipe_op_qk_norm_rope_scratch_bytes, not
 * kept, aligned to 4 bytes, apart from every other buffer. */
mpipe_status mpipe_op_qk_norm_rope_bwd(int32_t dtype, const mpipe_rope_cfg* cfg, int64_t rows,
                                       const mpipe_heads* dq, const mpipe_heads* dk,
                                       const mpipe_heads* q, const mpipe_heads* k,
                                       const void* q_gain, const void* k_gain, float eps,
                                       const int32_t* pos, int64_t ld_pos,
                                       const mpipe_heads* dq_in, const mpipe_heads* dk_in,
                                       float* grad_q_gain, float* grad_k_gain, int32_t accumulate,
                                       void* scratch, size_t scratch_bytes, void* hip_stream);
/* 0 for arguments out of range. */
size_t mpipe_op_qk_norm_rope_scratch_bytes(int64_t rows, int32_t heads_q, int32_t heads_k,
                                           int32_t head_dim);

/* A gradient of several tensors (dtype MPIPE_F32 or MPIPE_BF16, aligned to one element; n may
 * be 0).  The list is read during the call only. */
typedef struct {
  void* data;
  int64_t n;
  int32_t dtype;
  int32_t reserved;   /* 0 */
} mpipe_grad_tensor;

/* sumsq (device fp64 [1]) = the sum of squares of every element; norms (device fp32 [n],
 * nullable) = the L2 norm of each tensor.  Squares and sums in fp64 and in a fixed order: no
 * overflow for any fp32 gradient, and the same call gives the same bits.  sumsq is apart from
 * the norm so that a program can add the ranks' values first.  Two tensors of a list must not
 * share memory, nor sumsq, norms and scratch with each other or with a tensor.  scratch:
 * mpipe_op_grad_scratch_bytes, 8-byte aligned, not kept. */
mpipe_status mpipe_op_grad_norm(const mpipe_grad_tensor* grads, int32_t n, double* sumsq,
                                float* norms, void* scratch, size_t scratch_bytes,
                                void* hip_stream);
/* 0 for a list that is refused. */
size_t mpipe_op_grad_scratch_bytes(const mpipe_grad_tensor* grads, int32_t n);

/* norm (device fp32 [1], nullable) = sqrt(sumsq); with f = max_norm / sqrt(sumsq) where the root
 * is above max_norm and f = 1 elsewhere (a root that is infinite or not a number included: the
 * caller sees it in norm), out[i] = grads[i] * f in out[i]'s dtype.  The root and f are fp64:
 * where the root is finite but beyond fp32, so that norm is infinite, f still scales.
 * out == NULL or out[i].data == grads[i].data: in place, where f == 1 writes nothing.  Other
 * outputs are apart from every input and always written.  sumsq: device fp64 [1], as of this
 * call's turn on the stream, apart from every output; norm apart from sumsq and from every
 * tensor.  max_norm >= 0 (infinity: never scales). */
mpipe_status mpipe_op_grad_clip(const mpipe_grad_tensor* grads, const mpipe_grad_tensor* out,
                                int32_t n, const double* sumsq, double max_norm, float* norm,
                                void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
