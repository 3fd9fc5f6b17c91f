// Host-only planning of the operators around the first LLM layer (mpipe_ops.h): position
// spans, rotary tables, head-view checks and gradient work lists.  No HIP: the sanitizer
// tests build it with g++.
#pragma once
#include <cstddef>
#include <cstdint>
#include <string>
#include <vector>

#include "../../include/mpipe_ops.h"

namespace mpipe {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxPairs = kMaxHeadDim / 2;

// ---- positions ------------------------------------------------------------------------
// A run of rows: text (w == 0: every axis counts on from pos), an item (w > 0: slices of hw
// rows in lines of w, step between slices) or rows of no sequence (w < 0: not written).
struct PosSpan {
  int64_t row;
  int32_t pos, step, hw, w;
};
// Sorted spans covering [spans[0].row, end), each at most 2^28 rows of text or none, or one
// item.  Rows between two sequences are a span of their own.
mpipe_status position_spans(const int64_t* seq_row, const int64_t* seq_len,
                            const int64_t* seq_pos, int32_t n_seq, const int64_t* item_row,
                            const int32_t* grid_thw, const int32_t* time_step, int32_t n_items,
                            int64_t n_rows, int64_t* next, std::vector<PosSpan>& spans,
                            int64_t& end, std::string& why);

// ---- rotary tables ----------------------------------------------------------------------
// Pair i of a head turns by pos[axis[i]] * turn[i] / 2^64 of a full turn.  Whole-number
// products of the position with a 64-bit fraction keep the phase of a far position, which
// an fp32 (or for very far ones an fp64) product would lose.
struct RopeTable {
  uint64_t turn[kMaxPairs];
  uint8_t axis[kMaxPairs];
};
mpipe_status rope_axes_table(const mpipe_rope_cfg* cfg, RopeTable& t, std::string& why);

// ---- views of heads ---------------------------------------------------------------------
// [rows][heads][d], the columns of a head adjacent; strides in elements.
struct HeadView {
  const void* p = nullptr;
  int64_t row = 0, head = 0;
  int32_t heads = 0;
};
// A view that can be read: non-null, strides >= 0, no overflow.  `written`: also no element
// of it twice.
bool view_ok(const HeadView& v, int64_t rows, int32_t d, int esz, bool written, std::string& why);
// the same elements (a stride over one row or head does not count)
bool same_view(const HeadView& a, const HeadView& b, int64_t rows);
// Whether two (valid) views may share an element: exactly where their rows and their heads have
// one stride each, or their rows and a row holds either; else not if their ranges are apart.
bool views_meet(const HeadView& a, const HeadView& b, int64_t rows, int32_t d, int esz);
// Whether two ranges of bytes share one, and whether a range shares one with an element of a
// (valid) view.
bool ranges_meet(const void* a, size_t a_bytes, const void* b, size_t b_bytes);
bool range_meets(const void* p, size_t bytes, const HeadView& v, int64_t rows, int32_t d, int esz);

// ---- gradient lists -----------------------------------------------------------------------
// Elements of a work chunk: enough chunks for every compute unit from 8 M elements on.
int64_t grad_chunk(int64_t total);
struct GradPlan {
  int64_t chunk = 0, chunks = 0, total = 0;
};
mpipe_status grad_plan(const mpipe_grad_tensor* t, int32_t n, GradPlan& p, std::string& why);
// Outputs for the inputs `in`: alike in number and lengths, apart from each other, and each
// either its own input (same type) or apart from every input.
mpipe_status grad_outputs_ok(const mpipe_grad_tensor* in, const mpipe_grad_tensor* out, int32_t n,
                             std::string& why);
// Whether a range of bytes shares one with a tensor of a (valid) list.
bool list_meets(const mpipe_grad_tensor* t, int32_t n, const void* p, size_t bytes);

}  // namespace mpipe
