// Rows that do not begin on 16-byte boundaries, by runs through shared memory (rms_staged.cu): false where they do not go that way (strided rows, tensors that do not begin on a
// boundary, rows of more than 8192 values, scales for parts of a row), and nothing was launched.
#pragma once

#include "rows.h"

namespace xconv {

bool rms_staged_forward(const xconv_rows_desc* d, const void* X, const void* residual, const void* weight, void* H, void* Y, float* scales, float* rstd, cudaStream_t st,
                        cudaError_t* e);
// parts: partial sums of dweight that it leaves (at most rms_staged_backward_parts)
long rms_staged_backward_parts(const xconv_rows_desc* d);
bool rms_staged_backward(const xconv_rows_desc* d, const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX, void* dR, float* part, long* parts,
                         cudaStream_t st, cudaError_t* e);

}  // namespace xconv
