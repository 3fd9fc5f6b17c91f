// Launch interface of the operators around the first LLM layer (qk_rope.hip,
// positions.hip, grad_clip.hip); arguments are checked by layer_ops.cpp.
#pragma once
#include <hip/hip_runtime.h>

#include "internal.h"
#include "layer_plan.h"

namespace mpipe {

hipError_t seam_positions(const std::vector<PosSpan>& spans, int64_t end, int32_t* pos,
                          int64_t ld_pos, hipStream_t s);

// One side (0: q, 1: k) of a rotation: x -> y, and in a backward dy, x -> y.
struct QkSide {
  HeadView x, dy, y;
  const void* gain = nullptr;
  float* grad = nullptr;   // backward: gain gradient, nullable
};
struct QkProblem {
  int dtype = 0, head_dim = 0, rot_dim = 0;
  bool adjacent = false, inverse = false, norm = false;
  int64_t rows = 0;
  const int32_t* pos = nullptr;
  int64_t ld_pos = 0;
  float eps = 0.f;
  RopeTable table;
  QkSide side[2];
};
hipError_t qk_rope_fwd(const QkProblem& p, hipStream_t s);
hipError_t qk_norm_rope_bwd(const QkProblem& p, bool accumulate, float* scratch, hipStream_t s);
size_t qk_norm_rope_bwd_scratch(int64_t rows, int heads_q, int heads_k, int head_dim);

hipError_t grad_norm(const mpipe_grad_tensor* t, int n, const GradPlan& p, double* sumsq,
                     float* norms, char* scratch, hipStream_t s);
size_t grad_norm_scratch(int n, const GradPlan& p);
hipError_t grad_clip(const mpipe_grad_tensor* in, const mpipe_grad_tensor* out, int n,
                     const GradPlan& p, const double* sumsq, double max_norm, float* norm,
                     hipStream_t s);

}  // namespace mpipe
