// Positions of the LLM's input rows on three axes (mpipe_op_seam_positions).
//
// The host cuts the rows into spans of text and items (layer_plan.cpp) and passes them in the
// kernel's arguments, kSpans at a time: no upload, no wait, and the launch can be captured.  A
// thread finds its row's span by halving a copy of the spans' first rows in LDS and writes
// three words; 12 bytes a row, so the launch itself is what a call costs (2.4 us for 32 rows,
// 7.9 us in two launches for 262144 rows and their items).
#include <algorithm>

#include "layer_kernels.h"

namespace mpipe {
namespace {

constexpr int kSpans = 200;   // 20 bytes each; a launch's arguments stay below 4 KB

struct SpanArgs {
  int32_t row[kSpans];   // first row, from base; sorted
  int32_t pos[kSpans], step[kSpans], hw[kSpans], w[kSpans];
};

__global__ __launch_bounds__(256) void positions_kernel(SpanArgs a, int n, int64_t base, int count,
                                                        int32_t* pos, int64_t ld) {
  __shared__ int32_t first[kSpans];
  for (int i = threadIdx.x; i < n; i += 256) first[i] = a.row[i];
  __syncthreads();
  const int r = (int)(blockIdx.x * 256u + threadIdx.x);
  if (r >= count) return;
  int lo = 0, hi = n;   // first[lo] <= r < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= r) lo = mid; else hi = mid;
  }
  const int w = a.w[lo];
  if (w < 0) return;
  const int p = a.pos[lo];
  const uint32_t k = (uint32_t)(r - first[lo]);
  int t = (int)k, y = (int)k, x = (int)k;
  if (w > 0) {
    const uint32_t hw = (uint32_t)a.hw[lo], tau = k / hw, in = k - tau * hw;
    t = (int)tau * a.step[lo];
    y = (int)(in / (uint32_t)w);
    x = (int)(in - (uint32_t)y * (uint32_t)w);
  }
  int32_t* o = pos + base + r;
  o[0] = p + t;
  o[ld] = p + y;
  o[2 * ld] = p + x;
}

}  // namespace

hipError_t seam_positions(const std::vector<PosSpan>& spans, int64_t end, int32_t* pos,
                          int64_t ld_pos, hipStream_t s) {
  for (size_t i = 0; i < spans.size();) {
    SpanArgs a;
    const int64_t base = spans[i].row;
    int n = 0;
    // a span has at most 2^28 rows: rows from the base stay below 2^31
    for (; i < spans.size() && n < kSpans && spans[i].row - base < (int64_t(1) << 30); ++i, ++n) {
      a.row[n] = (int32_t)(spans[i].row - base);
      a.pos[n] = spans[i].pos;
      a.step[n] = spans[i].step;
      a.hw[n] = spans[i].hw;
      a.w[n] = spans[i].w;
    }
    const int count = (int)((i < spans.size() ? spans[i].row : end) - base);
    hipLaunchKernelGGL(positions_kernel, dim3((count + 255) / 256), dim3(256), 0, s, a, n, base,
                       count, pos, ld_pos);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mpipe
