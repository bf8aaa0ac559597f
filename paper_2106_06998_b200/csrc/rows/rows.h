// Operators on rows of C values at the borders of a block: dropout, the residual's addition, RMS norm, 8 bits (rows/*.cu): launches, for the entry points.
#pragma once

#include <cuda_runtime.h>

#include "../../../include/xconv.h"

namespace xconv {

// (bytes of partial sums that the backward call leaves in the scratch memory: by the descriptor alone)
size_t rms_backward_part_bytes(const xconv_rows_desc* d);

cudaError_t launch_rms_forward(const xconv_rows_desc* d, const void* X, const void* residual, const void* weight, void* H, void* Y, float* scales, float* rstd,
                               cudaStream_t st);
// part: rms_backward_part_bytes, or null with dweight; launches: how many kernels were launched
cudaError_t launch_rms_backward(const xconv_rows_desc* d, const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX, void* dR,
                                float* dweight, float* part, cudaStream_t st, int* launches);
cudaError_t launch_dropout(const xconv_rows_desc* d, const void* X, const void* residual, void* Y, cudaStream_t st);
cudaError_t launch_dequantize(const xconv_rows_desc* d, const void* Q, const float* scales, void* X, cudaStream_t st);

}  // namespace xconv
