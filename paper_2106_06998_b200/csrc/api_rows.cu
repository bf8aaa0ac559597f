// C ABI of the operators on rows (dropout, RMS norm, 8 bits): argument checks and dispatch (kernels: rows/).
#include "../../include/xconv.h"

#include "api_state.h"
#include "rows/rows.h"

namespace xconv {

static bool is_dtype(int t) { return t == XCONV_F32 || t == XCONV_BF16 || t == XCONV_F16; }
static size_t size_of(int dtype) { return dtype == XCONV_F32 ? 4 : 2; }
static bool off(const void* p, size_t a) { return p && reinterpret_cast<uintptr_t>(p) % a != 0; }

// What all calls mention: sizes, the storage type.
static xconv_status validate_rows(const xconv_rows_desc* d) {
  if (!d || d->rows < 0 || d->C <= 0 || !is_dtype(d->dtype)) return XCONV_ERR_INVALID_ARG;
  // 32-bit grids, and 64-bit element offsets with room to spare
  if (d->rows > 2000000000L || d->C > (1 << 30)) return XCONV_ERR_UNSUPPORTED;
  return XCONV_OK;
}
static xconv_status validate_norm(const xconv_rows_desc* d) {
  const xconv_status s = validate_rows(d);
  if (s != XCONV_OK) return s;
  return !(d->eps >= 0.f) || (d->param_dtype != XCONV_F32 && d->param_dtype != d->dtype) ? XCONV_ERR_INVALID_ARG : XCONV_OK;
}
static xconv_status validate_drop(const xconv_rows_desc* d) {
  if (!(d->p >= 0.0 && d->p <= 1.0) || (d->p > 0.0 && d->rows_per_mask < 1)) return XCONV_ERR_INVALID_ARG;
  return d->p > 0.0 && off(d->seed_add, 8) ? XCONV_ERR_ALIGNMENT : XCONV_OK;
}
static xconv_status validate_q(const xconv_rows_desc* d) {
  if (d->q_type != XCONV_Q_E4M3 && d->q_type != XCONV_Q_INT8) return XCONV_ERR_INVALID_ARG;
  if (d->q_group < 0) return XCONV_ERR_INVALID_ARG;
  return d->q_group < d->C && d->q_group != 0 && d->q_group != 32 && d->q_group != 64 && d->q_group != 128 ? XCONV_ERR_UNSUPPORTED : XCONV_OK;
}
namespace {
// A tensor that is there, or may be missing.
struct RowTensor {
  const void* p;
  int64_t stride;
  size_t size;
  bool out, must;
};
}  // namespace
template <int N>
static xconv_status validate_tensors(const xconv_rows_desc* d, const RowTensor (&tensors)[N]) {
  const int64_t most = 1L << 60;
  for (const RowTensor& t : tensors)
    if ((t.must && !t.p) || (t.p && (t.stride < 0 || (t.out && t.stride < d->C)))) return XCONV_ERR_INVALID_ARG;
  for (const RowTensor& t : tensors)
    if (t.p && d->rows > 0 && t.stride > most / d->rows) return XCONV_ERR_UNSUPPORTED;
  for (const RowTensor& t : tensors)
    if (off(t.p, t.size)) return XCONV_ERR_ALIGNMENT;
  return XCONV_OK;
}
static xconv_status cuda_status(cudaError_t e) {
  if (e == cudaSuccess) return XCONV_OK;
  g_last_cuda_error = (int)e;
  return XCONV_ERR_CUDA;
}
// The words at the front of the scratch memory that xconv_workspace_status reads stay as they are: nothing here waits.
static const size_t ROWS_HEADER = 256;

}  // namespace xconv

using namespace xconv;

extern "C" {

xconv_status xconv_rmsnorm_forward(const xconv_rows_desc* desc, const void* X, const void* residual, const void* weight, void* H, void* Y, float* scales, float* rstd,
                                   void* cuda_stream) {
  xconv_status s = validate_norm(desc);
  if (s == XCONV_OK) s = validate_drop(desc);
  if (s != XCONV_OK) return s;
  if (desc->q_type != XCONV_Q_NONE && (s = validate_q(desc)) != XCONV_OK) return s;
  if (!scales != (desc->q_type == XCONV_Q_NONE)) return XCONV_ERR_INVALID_ARG;
  const size_t es = size_of(desc->dtype);
  s = validate_tensors(desc, {{X, desc->x_stride, es, false, true}, {residual, desc->r_stride, es, false, false}, {H, desc->h_stride, es, true, false},
                              {Y, desc->y_stride, desc->q_type == XCONV_Q_NONE ? es : 1, true, true}});
  if (s != XCONV_OK) return s;
  if (off(weight, size_of(desc->param_dtype)) || off(scales, 4) || off(rstd, 4)) return XCONV_ERR_ALIGNMENT;
  new_call();
  if (desc->rows == 0) return XCONV_OK;
  ++g_launches;
  return cuda_status(launch_rms_forward(desc, X, residual, weight, H, Y, scales, rstd, static_cast<cudaStream_t>(cuda_stream)));
}

size_t xconv_rmsnorm_workspace_bytes(const xconv_rows_desc* desc) { return validate_norm(desc) == XCONV_OK ? ROWS_HEADER + rms_backward_part_bytes(desc) : 0; }

xconv_status xconv_rmsnorm_backward(const xconv_rows_desc* desc, const void* dY, const void* H, const float* rstd, const void* weight, const void* dH, void* dX, void* dresidual,
                                    float* dweight, void* ws, size_t ws_bytes, void* cuda_stream) {
  xconv_status s = validate_norm(desc);
  if (s == XCONV_OK) s = validate_drop(desc);
  if (s != XCONV_OK) return s;
  if (!rstd || (!dX && !dresidual && !dweight)) return XCONV_ERR_INVALID_ARG;
  const size_t es = size_of(desc->dtype);
  s = validate_tensors(desc, {{dY, desc->y_stride, es, false, true}, {H, desc->h_stride, es, false, true}, {dH, desc->dh_stride, es, false, false},
                              {dX, desc->x_stride, es, true, false}, {dresidual, desc->r_stride, es, true, false}});
  if (s != XCONV_OK) return s;
  if (off(weight, size_of(desc->param_dtype)) || off(rstd, 4) || off(dweight, 4)) return XCONV_ERR_ALIGNMENT;
  if (dweight && (!ws || ws_bytes < xconv_rmsnorm_workspace_bytes(desc))) return XCONV_ERR_WORKSPACE;
  if (dweight && off(ws, 16)) return XCONV_ERR_ALIGNMENT;
  new_call();
  int launches = 0;
  s = cuda_status(launch_rms_backward(desc, dY, H, rstd, weight, dH, dX, dresidual, dweight, dweight ? reinterpret_cast<float*>(static_cast<char*>(ws) + ROWS_HEADER) : nullptr,
                                      static_cast<cudaStream_t>(cuda_stream), &launches));
  g_launches += launches;
  return s;
}

xconv_status xconv_dropout(const xconv_rows_desc* desc, const void* X, const void* residual, void* Y, void* cuda_stream) {
  xconv_status s = validate_rows(desc);
  if (s == XCONV_OK) s = validate_drop(desc);
  if (s != XCONV_OK) return s;
  const size_t es = size_of(desc->dtype);
  s = validate_tensors(desc, {{X, desc->x_stride, es, false, true}, {residual, desc->r_stride, es, false, false}, {Y, desc->y_stride, es, true, true}});
  if (s != XCONV_OK) return s;
  new_call();
  if (desc->rows == 0) return XCONV_OK;
  ++g_launches;
  return cuda_status(launch_dropout(desc, X, residual, Y, static_cast<cudaStream_t>(cuda_stream)));
}

xconv_status xconv_dequantize(const xconv_rows_desc* desc, const void* Q, const float* scales, void* X, void* cuda_stream) {
  xconv_status s = validate_rows(desc);
  if (s == XCONV_OK) s = validate_q(desc);
  if (s != XCONV_OK) return s;
  s = validate_tensors(desc, {{Q, desc->y_stride, 1, false, true}, {X, desc->x_stride, size_of(desc->dtype), true, true}});
  if (s != XCONV_OK) return s;
  if (!scales) return XCONV_ERR_INVALID_ARG;
  if (off(scales, 4)) return XCONV_ERR_ALIGNMENT;
  new_call();
  if (desc->rows == 0) return XCONV_OK;
  ++g_launches;
  return cuda_status(launch_dequantize(desc, Q, scales, X, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
