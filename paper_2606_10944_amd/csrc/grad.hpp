// The gradient of coreset attention: arguments and launch shapes.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "grad_plan.hpp"

namespace thin {

struct GradArgs {
  const void *Q, *K, *V, *dO;
  const int32_t* idx;
  const float* logw;  // nullable
  void *dQ, *dK, *dV;
  float* dlogw;  // nullable
  int64_t S, n, n_q, n_out;
  GradShape shape;
  bool zeros;     // the zeros of dK and dV come from a launch of their own
  float* part;    // [S, chunks, parts, keys, 2, d]: sums of dK and dV
  float* part_w;  // [S, chunks, parts, keys]: of dlogw (null without)
  float* stats;   // [3, S, n_q] where a row's statistics need a pass of their own
};
// dtype of Q, K, V and the gradients; out_dtype of dO.
hipError_t launch_grad_zeros(int64_t row_bytes, const GradArgs& a, hipStream_t st);
hipError_t launch_grad_rows(int dtype, int out_dtype, int64_t d, const GradArgs& a, hipStream_t st);
hipError_t launch_grad_keys(int dtype, int out_dtype, int64_t d, const GradArgs& a, hipStream_t st);
hipError_t launch_grad_join(int dtype, int64_t d, const GradArgs& a, hipStream_t st);

}  // namespace thin
