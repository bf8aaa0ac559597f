// C ABI of the layer norm: argument checks and dispatch (kernels: layer_norm.cu).
#include "../../include/xconv.h"

#include <algorithm>

#include "api_state.h"
#include "layer_norm.h"

namespace xconv {

// dx_stride is the gradients' alone.
static xconv_status validate_norm(const xconv_norm_desc* d, bool gradients) {
  if (!d || d->rows <= 0 || d->C <= 0 || !(d->eps >= 0.f)) return XCONV_ERR_INVALID_ARG;
  if (d->dtype != XCONV_F32 && d->dtype != XCONV_BF16 && d->dtype != XCONV_F16) return XCONV_ERR_INVALID_ARG;
  if (d->param_dtype != XCONV_F32 && d->param_dtype != d->dtype) return XCONV_ERR_INVALID_ARG;
  if (d->x_stride < 0 || d->y_stride < 0 || (gradients && d->dx_stride < 0)) return XCONV_ERR_INVALID_ARG;
  // 32-bit grids, and 64-bit element offsets with room to spare
  if (d->rows > 2000000000L || d->C > (1 << 30)) return XCONV_ERR_UNSUPPORTED;
  const long most = 1L << 60;
  if (d->x_stride > most / d->rows || d->y_stride > most / d->rows || (gradients && d->dx_stride > most / d->rows)) return XCONV_ERR_UNSUPPORTED;
  return XCONV_OK;
}
// The words at the front of the scratch memory that xconv_workspace_status reads: no kernel of the norm waits on anything, and they stay as they are.
static const size_t NORM_HEADER = 256;

static inline bool off(const void* p, size_t a) { return p && reinterpret_cast<uintptr_t>(p) % a != 0; }
static inline size_t size_of(int dtype) { return dtype == XCONV_F32 ? 4 : 2; }
static xconv_status cuda_status(cudaError_t e) {
  if (e == cudaSuccess) return XCONV_OK;
  g_last_cuda_error = (int)e;
  return XCONV_ERR_CUDA;
}

}  // namespace xconv

using namespace xconv;

extern "C" {

size_t xconv_layernorm_workspace_bytes(const xconv_norm_desc* desc) {
  if (validate_norm(desc, true) != XCONV_OK) return 0;
  return NORM_HEADER + (size_t)norm_backward_parts(desc) * 2 * (size_t)desc->C * sizeof(float);
}

xconv_status xconv_layernorm_forward(const xconv_norm_desc* desc, const void* X, const void* weight, const void* bias, void* Y, float* mean, float* rstd,
                                     void* cuda_stream) {
  const xconv_status s = validate_norm(desc, false);
  if (s != XCONV_OK) return s;
  if (!X || !Y || !mean != !rstd || desc->y_stride < desc->C) return XCONV_ERR_INVALID_ARG;
  const size_t es = size_of(desc->dtype), ps = size_of(desc->param_dtype);
  if (off(X, es) || off(Y, es) || off(weight, ps) || off(bias, ps) || off(mean, 4) || off(rstd, 4)) return XCONV_ERR_ALIGNMENT;
  const NormPlan p = plan_norm_forward(desc, X, weight, bias, Y);
  new_call();
  ++g_launches;
  return cuda_status(launch_norm_forward(desc, p, X, weight, bias, Y, mean, rstd, static_cast<cudaStream_t>(cuda_stream)));
}

xconv_status xconv_layernorm_backward(const xconv_norm_desc* desc, const void* dY, const void* X, const float* mean, const float* rstd, const void* weight, void* dX,
                                      float* dweight, float* dbias, void* ws, size_t ws_bytes, void* cuda_stream) {
  const xconv_status s = validate_norm(desc, true);
  if (s != XCONV_OK) return s;
  if (!dY || !X || !mean || !rstd || !dX || desc->dx_stride < desc->C) return XCONV_ERR_INVALID_ARG;
  const size_t es = size_of(desc->dtype), ps = size_of(desc->param_dtype);
  if (off(dY, es) || off(X, es) || off(dX, es) || off(weight, ps) || off(mean, 4) || off(rstd, 4) || off(dweight, 4) || off(dbias, 4)) return XCONV_ERR_ALIGNMENT;
  const bool sums = dweight || dbias;
  if (sums && (!ws || ws_bytes < xconv_layernorm_workspace_bytes(desc))) return XCONV_ERR_WORKSPACE;
  if (sums && off(ws, 16)) return XCONV_ERR_ALIGNMENT;
  const NormPlan p = plan_norm_backward(desc, dY, X, weight, dX);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  float* part = sums ? reinterpret_cast<float*>(static_cast<char*>(ws) + NORM_HEADER) : nullptr;
  new_call();
  ++g_launches;
  xconv_status r = cuda_status(launch_norm_backward(desc, p, dY, X, mean, rstd, weight, dX, part, st));
  if (r != XCONV_OK || !sums) return r;
  g_launches += p.wide ? 2 : 1;
  return cuda_status(launch_norm_sums(desc, part, p.parts, dweight, dbias, st));
}

}  // extern "C"
