// Layer norm over the last axis of a matrix of rows (layer_norm.cu): launch plans and launches, for the entry points.
#pragma once

#include <cuda_runtime.h>

#include "../../include/xconv.h"

namespace xconv {

struct NormPlan {
  bool vec;              // 16-byte accesses
  bool full;             // every thread of a row has all its vectors
  bool wide;             // a row does not fit the registers of a block
  int V, group, threads; // vectors (or elements) a thread, threads a row, threads a block
  bool words;            // runs two values at a time
  int run;               // rows of a run (dense rows that are not aligned), or 0
  int smem;
  long blocks;
  long parts;            // partial sums of dweight and dbias (backward)
};
NormPlan plan_norm_forward(const xconv_norm_desc* d, const void* X, const void* weight, const void* bias, const void* Y);
// (the number of partial sums depends on the descriptor alone)
NormPlan plan_norm_backward(const xconv_norm_desc* d, const void* dY, const void* X, const void* weight, const void* dX);
long norm_backward_parts(const xconv_norm_desc* d);

cudaError_t launch_norm_forward(const xconv_norm_desc* d, const NormPlan& p, const void* X, const void* weight, const void* bias, void* Y, float* mean, float* rstd,
                                cudaStream_t st);
// part: norm_backward_parts * 2 * C floats, or null with dweight and dbias
cudaError_t launch_norm_backward(const xconv_norm_desc* d, const NormPlan& p, const void* dY, const void* X, const float* mean, const float* rstd, const void* weight,
                                 void* dX, float* part, cudaStream_t st);
cudaError_t launch_norm_sums(const xconv_norm_desc* d, const float* part, long parts, float* dweight, float* dbias, cudaStream_t st);

}  // namespace xconv
