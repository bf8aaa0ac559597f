// The binding's calls on ordinary tensors, in native code: what binding.py does for the same call -- checks of layout and shape, the descriptor, the outputs,
// the scratch buffer, the C ABI's call on the current stream -- without the interpreter.  A training step is three calls of 14 to 25 us through the
// interpreter, of 5 to 12 here (57 -> 26 us of host time a step of 16 volumes of 5 x 19 x 19, whose kernels take 54; the launches are two thirds of the rest).
//
// A function returns None for whatever is not the ordinary case (tensors that are not dense CUDA tensors, subclasses, modes that want to see every call, a
// layout or shape that does not fit, an option that is rarely given): binding.py then goes its own way, which is where every error is raised.
#include <torch/csrc/Device.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>
#include <vector>

#include "../../include/xconv.h"

namespace {

// Entry points of the library that binding.py has loaded, and its functions that raise for a status and hand out scratch buffers.
struct Library {
  decltype(&xconv_workspace_bytes) workspace_bytes;
  decltype(&xconv_forward) forward;
  decltype(&xconv_sketch) sketch;
  decltype(&xconv_wgrad) wgrad;
  decltype(&xconv_dgrad) dgrad;
  decltype(&xconv_sketch_seeded) sketch_seeded;
  decltype(&xconv_wgrad_seeded) wgrad_seeded;
  decltype(&xconv_backprobe) backprobe;
  decltype(&xconv_contract) contract;
  decltype(&xconv_layernorm_workspace_bytes) norm_workspace_bytes;
  decltype(&xconv_layernorm_forward) norm_forward;
  decltype(&xconv_layernorm_backward) norm_backward;
  decltype(&xconv_update_workspace_bytes) update_workspace_bytes;
  decltype(&xconv_orthogonalize) orthogonalize;
  decltype(&xconv_muon_step) muon_step;
} lib{};
PyObject *raise_for_status = nullptr, *workspace = nullptr;

bool watched() {      // modes that are to see the tensor functions of the Python path
  return at::impl::PythonTorchFunctionTLS::stack_len() > 0 || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// The tensor in `o` if it is an ordinary dense CUDA tensor.
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided) return nullptr;
  using K = c10::DispatchKey;
  const c10::DispatchKeySet keys = t.key_set();
  for (K k : {K::Python, K::PythonTLSSnapshot, K::FuncTorchBatched, K::FuncTorchGradWrapper, K::Functionalize, K::Batched, K::ZeroTensor, K::Conjugate, K::Negative,
              K::Named, K::Fake})
    if (keys.has(k)) return nullptr;
  return &t;
}

int dtype_code(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return XCONV_F32;
    case at::kBFloat16: return XCONV_BF16;
    case at::kHalf: return XCONV_F16;
    default: return -1;
  }
}

// A 4-d tensor in channels_last or a 5-d one in channels_last_3d.
struct Image {
  const at::Tensor* t = nullptr;
  int dim = 0, dtype = -1;
  int32_t n = 0, c = 0, D = 1, H = 0, W = 0;
  explicit Image(PyObject* o) {
    const at::Tensor* x = plain(o);
    if (!x) return;
    dim = (int)x->dim();
    if (dim != 4 && dim != 5) return;
    if (!x->is_contiguous(dim == 4 ? at::MemoryFormat::ChannelsLast : at::MemoryFormat::ChannelsLast3d)) return;
    dtype = dtype_code(*x);
    if (dtype < 0) return;
    for (int i = 0; i < dim; ++i)
      if (x->size(i) <= 0 || x->size(i) > INT32_MAX) return;
    n = (int32_t)x->size(0); c = (int32_t)x->size(1);
    D = dim == 5 ? (int32_t)x->size(2) : 1;
    H = (int32_t)x->size(dim - 2); W = (int32_t)x->size(dim - 1);
    t = x;
  }
  explicit operator bool() const { return t != nullptr; }
  bool same_plane(const Image& o) const { return dim == o.dim && D == o.D && H == o.H && W == o.W && dtype == o.dtype; }
};

// The [r, B] sketch: a contiguous float matrix.
const at::Tensor* sketch_of(PyObject* o, int32_t B) {
  const at::Tensor* s = plain(o);
  return s && s->dim() == 2 && s->size(1) == B && s->size(0) > 0 && s->size(0) <= INT32_MAX && s->scalar_type() == at::kFloat && s->is_contiguous() ? s : nullptr;
}

bool small_int(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long x = PyLong_AsLongAndOverflow(o, &over);
  if (over || x < 1 || x > 64) return false;
  *v = (int32_t)x;
  return true;
}

// A square kernel, as the descriptor has it (which is made from the last extent alone).
bool square(const Image& W) { return W.H == W.W && W.W <= 64 && W.D <= 64; }
// A kernel over planes, for tensors that have planes: the weights of a planar layer are allocated without them.
bool planes_fit(const Image& g, int32_t KD) { return g.dim == 5 || KD == 1; }

xconv_desc descriptor(int32_t B, int32_t Cin, int32_t Cout, const Image& g, int32_t r, int32_t K, int32_t KD, bool circular) {
  xconv_desc d;
  std::memset(&d, 0, sizeof d);
  d.B = B; d.Cin = Cin; d.Cout = Cout; d.H = g.H; d.W = g.W; d.KH = d.KW = K; d.pad_h = d.pad_w = (K - 1) / 2; d.r = r; d.dtype = g.dtype;
  d.circular = circular ? 1 : 0; d.D = g.D; d.KD = KD; d.pad_d = (KD - 1) / 2;
  return d;
}

// Scratch bytes of a layer, remembered by its sizes (the pointers of a descriptor made here are null).
size_t scratch_bytes(const xconv_desc& d, int op) {
  struct Entry { xconv_desc d; int op = -1; size_t bytes; };
  static thread_local Entry table[64];
  uint32_t h = (uint32_t)op * 2654435761u;
  for (int32_t v : {d.B, d.Cin, d.Cout, d.H, d.W, d.KH, d.r, d.dtype, d.D, d.KD, d.circular}) h = (h ^ (uint32_t)v) * 16777619u;
  Entry& e = table[(h >> 20) & 63];
  if (e.op != op || std::memcmp(&e.d, &d, sizeof d) != 0) {
    e.d = d; e.op = op;
    e.bytes = lib.workspace_bytes(&d, op);
  }
  return e.bytes;
}

// binding.workspace's buffer for this thread and stream.  That pool owns it; what is kept here only finds it again without the interpreter, and holds nothing alive.
struct Found { c10::DeviceIndex device; cudaStream_t stream; c10::weak_intrusive_ptr<c10::TensorImpl> buffer; };
thread_local std::vector<Found> found;

at::Tensor scratch(size_t bytes, const at::Tensor& like, cudaStream_t stream) {
  if (stream && c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None)      // (the graph's own, as binding.workspace does)
    return at::empty({(int64_t)std::max<size_t>(bytes, 256)}, like.options().dtype(at::kByte).requires_grad(false));
  const c10::DeviceIndex device = like.device().index();
  for (size_t i = 0; i < found.size(); ++i)
    if (found[i].device == device && found[i].stream == stream) {
      auto impl = found[i].buffer.lock();
      if (impl && (size_t)impl->numel() >= bytes) return at::Tensor(std::move(impl));
      found.erase(found.begin() + (long)i);
      break;
    }
  THPObjectPtr where(THPDevice_New(like.device()));
  THPObjectPtr buffer(where ? PyObject_CallFunction(workspace, "nO", (Py_ssize_t)bytes, where.get()) : nullptr);
  if (!buffer) throw python_error();
  TORCH_CHECK(THPVariable_Check(buffer.get()), "workspace() returns a tensor");
  at::Tensor t = THPVariable_Unpack(buffer.get());
  if (found.size() >= 8) found.erase(found.begin());
  found.push_back({device, stream, c10::weak_intrusive_ptr<c10::TensorImpl>(t.getIntrusivePtr())});
  return t;
}

at::Tensor image_like(const Image& g, int64_t n, int64_t c) {
  const auto opt = g.t->options().requires_grad(false);
  return g.dim == 4 ? at::empty({n, c, g.H, g.W}, opt, at::MemoryFormat::ChannelsLast) : at::empty({n, c, g.D, g.H, g.W}, opt, at::MemoryFormat::ChannelsLast3d);
}
at::Tensor weights_like(const Image& g, int64_t Cout, int64_t Cin, int64_t K, int64_t KD) {
  const auto opt = g.t->options().dtype(at::kFloat).requires_grad(false);
  return g.dim == 4 ? at::empty({Cout, Cin, K, K}, opt, at::MemoryFormat::ChannelsLast) : at::empty({Cout, Cin, KD, K, K}, opt, at::MemoryFormat::ChannelsLast3d);
}
at::Tensor matrix_like(const Image& g, int64_t rows, int64_t cols) { return at::empty({rows, cols}, g.t->options().dtype(at::kFloat).requires_grad(false)); }

// The call itself, with scratch memory, without the interpreter's lock; false with a Python error set.
template <class Call>
bool run(const Image& g, const xconv_desc& d, int op, const char* name, Call&& call) {
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
  const at::Tensor ws = scratch(scratch_bytes(d, op), *g.t, stream);
  void* p = ws.data_ptr();
  const size_t bytes = (size_t)ws.numel();
  xconv_status s;
  Py_BEGIN_ALLOW_THREADS
  s = call(&d, p, bytes, (void*)stream);
  Py_END_ALLOW_THREADS
  if (s == XCONV_OK) return true;
  PyObject* r = PyObject_CallFunction(raise_for_status, "is", (int)s, name);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
  return false;
}

#define XM_BEGIN(N) HANDLE_TH_ERRORS if (nargs != (N) || !lib.forward || watched()) Py_RETURN_NONE;
#define XM_END END_HANDLE_TH_ERRORS

// forward(X, W, Z, circular) -> (Y, S)
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(4)
  const Image X(a[0]), W(a[1]), Z(a[2]);
  if (!X || !W || !Z || !PyBool_Check(a[3])) Py_RETURN_NONE;
  if (!Z.same_plane(X) || Z.c != X.c || W.c != X.c || W.dim != X.dim || W.dtype != X.dtype || !square(W)) Py_RETURN_NONE;
  const xconv_desc d = descriptor(X.n, X.c, W.n, X, Z.n, W.W, W.D, a[3] == Py_True);
  const at::Tensor Y = image_like(X, X.n, W.n), S = matrix_like(X, Z.n, X.n);
  if (!run(X, d, XCONV_OP_FORWARD, "xconv_forward", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.forward(q, X.t->data_ptr(), W.t->data_ptr(), Z.t->data_ptr(), Y.data_ptr(), (float*)S.data_ptr(), ws, n, st); }))
    return nullptr;
  return Py_BuildValue("(NN)", THPVariable_Wrap(Y), THPVariable_Wrap(S));
  XM_END
}

// sketch(X, Z) -> S
PyObject* sketch(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(2)
  const Image X(a[0]), Z(a[1]);
  if (!X || !Z || !Z.same_plane(X) || Z.c != X.c) Py_RETURN_NONE;
  const xconv_desc d = descriptor(X.n, X.c, 1, X, Z.n, 3, 1, false);
  const at::Tensor S = matrix_like(X, Z.n, X.n);
  if (!run(X, d, XCONV_OP_SKETCH, "xconv_sketch", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.sketch(q, X.t->data_ptr(), Z.t->data_ptr(), (float*)S.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(S);
  XM_END
}

// sketch_seeded(X, seed, r) -> S
PyObject* sketch_seeded(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(3)
  const Image X(a[0]);
  if (!X || !PyLong_CheckExact(a[1]) || !PyLong_CheckExact(a[2])) Py_RETURN_NONE;
  int over = 0;
  const long r = PyLong_AsLongAndOverflow(a[2], &over);
  if (over || r <= 0 || r > INT32_MAX) Py_RETURN_NONE;
  const unsigned long long seed = PyLong_AsUnsignedLongLongMask(a[1]);
  const xconv_desc d = descriptor(X.n, X.c, 1, X, (int32_t)r, 3, 1, false);
  const at::Tensor S = matrix_like(X, r, X.n);
  if (!run(X, d, XCONV_OP_SKETCH_SEEDED, "xconv_sketch_seeded", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.sketch_seeded(q, X.t->data_ptr(), seed, (float*)S.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(S);
  XM_END
}

// wgrad(sketch, dY, Z, kernel_size, kernel_depth, circular) -> dW
PyObject* wgrad(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(6)
  const Image Y(a[1]), Z(a[2]);
  int32_t K, KD;
  if (!Y || !Z || !Z.same_plane(Y) || !small_int(a[3], &K) || !small_int(a[4], &KD) || !planes_fit(Y, KD) || !PyBool_Check(a[5])) Py_RETURN_NONE;
  const at::Tensor* S = sketch_of(a[0], Y.n);
  if (!S || S->size(0) != Z.n) Py_RETURN_NONE;
  const xconv_desc d = descriptor(Y.n, Z.c, Y.c, Y, Z.n, K, KD, a[5] == Py_True);
  const at::Tensor dW = weights_like(Y, Y.c, Z.c, K, KD);
  if (!run(Y, d, XCONV_OP_WGRAD, "xconv_wgrad", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.wgrad(q, (const float*)S->data_ptr(), Y.t->data_ptr(), Z.t->data_ptr(), (float*)dW.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(dW);
  XM_END
}

// wgrad_seeded(sketch, dY, seed, Cin, kernel_size, kernel_depth, circular) -> dW
PyObject* wgrad_seeded(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(7)
  const Image Y(a[1]);
  int32_t K, KD;
  if (!Y || !PyLong_CheckExact(a[2]) || !PyLong_CheckExact(a[3]) || !small_int(a[4], &K) || !small_int(a[5], &KD) || !planes_fit(Y, KD) || !PyBool_Check(a[6]))
    Py_RETURN_NONE;
  int over = 0;
  const long Cin = PyLong_AsLongAndOverflow(a[3], &over);
  if (over || Cin <= 0 || Cin > INT32_MAX) Py_RETURN_NONE;
  const at::Tensor* S = sketch_of(a[0], Y.n);
  if (!S) Py_RETURN_NONE;
  const unsigned long long seed = PyLong_AsUnsignedLongLongMask(a[2]);
  const xconv_desc d = descriptor(Y.n, (int32_t)Cin, Y.c, Y, (int32_t)S->size(0), K, KD, a[6] == Py_True);
  const at::Tensor dW = weights_like(Y, Y.c, Cin, K, KD);
  if (!run(Y, d, XCONV_OP_WGRAD_SEEDED, "xconv_wgrad_seeded", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.wgrad_seeded(q, (const float*)S->data_ptr(), Y.t->data_ptr(), seed, (float*)dW.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(dW);
  XM_END
}

// dgrad(dY, W, circular) -> dX
PyObject* dgrad(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(3)
  const Image Y(a[0]), W(a[1]);
  if (!Y || !W || !PyBool_Check(a[2]) || W.n != Y.c || W.dtype != Y.dtype || W.dim != Y.dim || !square(W)) Py_RETURN_NONE;
  const xconv_desc d = descriptor(Y.n, W.c, Y.c, Y, 1, W.W, W.D, a[2] == Py_True);
  const at::Tensor dX = image_like(Y, Y.n, W.c);
  if (!run(Y, d, XCONV_OP_DGRAD, "xconv_dgrad", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.dgrad(q, Y.t->data_ptr(), W.t->data_ptr(), dX.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(dX);
  XM_END
}

// backprobe(sketch, dY) -> L
PyObject* backprobe(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(2)
  const Image Y(a[1]);
  if (!Y) Py_RETURN_NONE;
  const at::Tensor* S = sketch_of(a[0], Y.n);
  if (!S) Py_RETURN_NONE;
  const xconv_desc d = descriptor(Y.n, 1, Y.c, Y, (int32_t)S->size(0), 3, 1, false);
  const at::Tensor L = image_like(Y, S->size(0), Y.c);
  if (!run(Y, d, XCONV_OP_WGRAD, "xconv_backprobe", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.backprobe(q, (const float*)S->data_ptr(), Y.t->data_ptr(), L.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(L);
  XM_END
}

// contract(L, Z, kernel_size, kernel_depth, circular) -> dW
PyObject* contract(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(5)
  const Image L(a[0]), Z(a[1]);
  int32_t K, KD;
  if (!L || !Z || !Z.same_plane(L) || Z.n != L.n || !small_int(a[2], &K) || !small_int(a[3], &KD) || !planes_fit(L, KD) || !PyBool_Check(a[4])) Py_RETURN_NONE;
  const xconv_desc d = descriptor(1, Z.c, L.c, L, L.n, K, KD, a[4] == Py_True);
  const at::Tensor dW = weights_like(L, L.c, Z.c, K, KD);
  if (!run(L, d, XCONV_OP_WGRAD, "xconv_contract", [&](const xconv_desc* q, void* ws, size_t n, void* st) {
        return lib.contract(q, L.t->data_ptr(), Z.t->data_ptr(), (float*)dW.data_ptr(), ws, n, st); }))
    return nullptr;
  return THPVariable_Wrap(dW);
  XM_END
}

// ---- around the layers

bool raise(xconv_status s, const char* name) {
  if (s == XCONV_OK) return true;
  PyObject* r = PyObject_CallFunction(raise_for_status, "is", (int)s, name);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
  return false;
}
bool on_current_device(const at::Tensor& t) { return t.device().index() == c10::cuda::current_device(); }

// A dense tensor of the library's layout: matrices and tokens (1-d to 3-d) row-major, images and volumes channels-last.
const at::Tensor* dense(PyObject* o) {
  const at::Tensor* t = plain(o);
  if (!t || t->dim() < 1 || t->dim() > 5 || t->numel() == 0 || dtype_code(*t) < 0 || !on_current_device(*t)) return nullptr;
  const auto fmt = t->dim() == 4 ? at::MemoryFormat::ChannelsLast : t->dim() == 5 ? at::MemoryFormat::ChannelsLast3d : at::MemoryFormat::Contiguous;
  return t->is_contiguous(fmt) ? t : nullptr;
}
at::Tensor dense_like(const at::Tensor& t) {
  const auto fmt = t.dim() == 4 ? at::MemoryFormat::ChannelsLast : t.dim() == 5 ? at::MemoryFormat::ChannelsLast3d : at::MemoryFormat::Contiguous;
  return at::empty(t.sizes(), t.options().requires_grad(false), fmt);
}
// The rows of a dense tensor: their shape, and the number of values in each.
int64_t rows_of(const at::Tensor& t, std::vector<int64_t>* shape) {
  const int c = t.dim() >= 4 ? 1 : (int)t.dim() - 1;
  for (int i = 0; i < t.dim(); ++i)
    if (i != c) shape->push_back(t.size(i));
  return t.size(c);
}
// A vector of C parameters in X's type or float (code: of both), or None.
bool param_of(PyObject* o, const at::Tensor& X, int64_t C, const at::Tensor** p, int* code) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  if (!t || t->dim() != 1 || t->size(0) != C || !t->is_contiguous() || t->device() != X.device()) return false;
  const int c = dtype_code(*t);
  if (c < 0 || (c != XCONV_F32 && c != dtype_code(X)) || (*code >= 0 && *code != c)) return false;
  *code = c;
  *p = t;
  return true;
}
xconv_norm_desc norm_desc(const at::Tensor& X, int64_t C, int code, float eps) {
  xconv_norm_desc d;
  std::memset(&d, 0, sizeof d);
  d.rows = X.numel() / C; d.C = (int32_t)C; d.dtype = dtype_code(X); d.param_dtype = code < 0 ? XCONV_F32 : code; d.eps = eps;
  d.x_stride = d.y_stride = d.dx_stride = C;
  return d;
}
void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
// A call into the library without the interpreter's lock.
template <class Call>
xconv_status unlocked(Call&& call) {
  xconv_status s;
  Py_BEGIN_ALLOW_THREADS
  s = call();
  Py_END_ALLOW_THREADS
  return s;
}

// layernorm(X, weight, bias, eps) -> (Y, mean, rstd)
PyObject* layernorm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(4)
  const at::Tensor* X = dense(a[0]);
  if (!X || !PyFloat_CheckExact(a[3])) Py_RETURN_NONE;
  std::vector<int64_t> shape;
  const int64_t C = rows_of(*X, &shape);
  const at::Tensor *w, *b;
  int code = -1;
  if (C > INT32_MAX || !param_of(a[1], *X, C, &w, &code) || !param_of(a[2], *X, C, &b, &code)) Py_RETURN_NONE;
  const xconv_norm_desc d = norm_desc(*X, C, code, (float)PyFloat_AS_DOUBLE(a[3]));
  const auto opt = X->options().dtype(at::kFloat).requires_grad(false);
  const at::Tensor Y = dense_like(*X), mean = at::empty(shape, opt), rstd = at::empty(shape, opt);
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
  const void *x = X->data_ptr(), *wp = address(w), *bp = address(b);
  const xconv_status s = unlocked([&] { return lib.norm_forward(&d, x, wp, bp, Y.data_ptr(), (float*)mean.data_ptr(), (float*)rstd.data_ptr(), stream); });
  if (!raise(s, "xconv_layernorm_forward")) return nullptr;
  return Py_BuildValue("(NNN)", THPVariable_Wrap(Y), THPVariable_Wrap(mean), THPVariable_Wrap(rstd));
  XM_END
}

// layernorm_backward(dY, X, mean, rstd, weight) -> (dX, dweight, dbias)
PyObject* layernorm_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(5)
  const at::Tensor *dY = dense(a[0]), *X = dense(a[1]), *mean = plain(a[2]), *rstd = plain(a[3]);
  if (!dY || !X || !mean || !rstd || dY->sizes() != X->sizes() || dY->scalar_type() != X->scalar_type() || dY->device() != X->device()) Py_RETURN_NONE;
  std::vector<int64_t> shape;
  const int64_t C = rows_of(*X, &shape);
  for (const at::Tensor* t : {mean, rstd})
    if (t->scalar_type() != at::kFloat || t->sizes() != at::IntArrayRef(shape) || !t->is_contiguous() || t->device() != X->device()) Py_RETURN_NONE;
  const at::Tensor* w;
  int code = -1;
  if (C > INT32_MAX || !param_of(a[4], *X, C, &w, &code)) Py_RETURN_NONE;
  const xconv_norm_desc d = norm_desc(*X, C, code, 0.f);
  const auto opt = X->options().dtype(at::kFloat).requires_grad(false);
  const at::Tensor dX = dense_like(*X), dw = at::empty({C}, opt), db = at::empty({C}, opt);
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
  const at::Tensor ws = scratch(lib.norm_workspace_bytes(&d), *X, stream);
  const void *dy = dY->data_ptr(), *x = X->data_ptr(), *wp = address(w);
  const float *m = (const float*)mean->data_ptr(), *r = (const float*)rstd->data_ptr();
  const xconv_status s = unlocked([&] {
    return lib.norm_backward(&d, dy, x, m, r, wp, dX.data_ptr(), (float*)dw.data_ptr(), (float*)db.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), stream); });
  if (!raise(s, "xconv_layernorm_backward")) return nullptr;
  return Py_BuildValue("(NNN)", THPVariable_Wrap(dX), THPVariable_Wrap(dw), THPVariable_Wrap(db));
  XM_END
}

// The matrices that a dense tensor of weights holds: two or three dimensions, or a convolution's.
bool matrices_of(const at::Tensor& t, xconv_matrices* m) {
  const int64_t dim = t.dim(), rows = dim == 3 ? t.size(1) : t.size(0), batch = dim == 3 ? t.size(0) : 1;
  if (dim < 2) return false;
  const int64_t cols = t.numel() / (rows * batch);
  if (rows > INT32_MAX || cols > INT32_MAX || batch > INT32_MAX) return false;
  std::memset(m, 0, sizeof *m);
  m->rows = (int32_t)rows; m->cols = (int32_t)cols; m->batch = (int32_t)batch;
  return true;
}
bool number(PyObject* o, float* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = (float)PyFloat_AS_DOUBLE(o);
  return true;
}
// steps, coefficients (three floats in a tuple), eps
bool steps_of(PyObject* steps, PyObject* coefficients, PyObject* eps, xconv_update_desc* d) {
  std::memset(d, 0, sizeof *d);
  return small_int(steps, &d->steps) && PyTuple_CheckExact(coefficients) && PyTuple_GET_SIZE(coefficients) == 3 && number(PyTuple_GET_ITEM(coefficients, 0), &d->a) &&
         number(PyTuple_GET_ITEM(coefficients, 1), &d->b) && number(PyTuple_GET_ITEM(coefficients, 2), &d->c) && number(eps, &d->eps);
}
// The items of a list, or the one tensor that is given in its place.
struct Several {
  PyObject* list;
  PyObject* one;
  explicit Several(PyObject* o) : list(PyList_CheckExact(o) ? o : nullptr), one(o) {}
  Py_ssize_t size() const { return list ? PyList_GET_SIZE(list) : 1; }
  PyObject* operator[](Py_ssize_t i) const { return list ? PyList_GET_ITEM(list, i) : one; }
};
xconv_status update(decltype(&xconv_orthogonalize) call, const xconv_update_desc& d, const std::vector<xconv_matrices>& items, const at::Tensor& like) {
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream().stream();
  const at::Tensor ws = scratch(lib.update_workspace_bytes(items.data(), (int)items.size()), like, stream);
  return unlocked([&] { return call(&d, items.data(), (int)items.size(), ws.data_ptr(), (size_t)ws.numel(), stream); });
}

// orthogonalize(G or list, steps, coefficients, eps) -> O or list
PyObject* orthogonalize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(4)
  xconv_update_desc d;
  const Several G(a[0]);
  if (G.size() == 0 || !steps_of(a[1], a[2], a[3], &d)) Py_RETURN_NONE;
  std::vector<xconv_matrices> items((size_t)G.size());
  std::vector<at::Tensor> in;                        // (held: other threads run during the call, and the list is theirs too)
  for (Py_ssize_t i = 0; i < G.size(); ++i) {
    const at::Tensor* g = dense(G[i]);
    if (!g || !matrices_of(*g, &items[i])) Py_RETURN_NONE;
    in.push_back(*g);
  }
  std::vector<at::Tensor> out;
  for (size_t i = 0; i < in.size(); ++i) {
    out.push_back(dense_like(in[i]));
    items[i].G = in[i].data_ptr(); items[i].O = out[i].data_ptr();
    items[i].g_dtype = items[i].o_dtype = dtype_code(in[i]);
  }
  if (!raise(update(lib.orthogonalize, d, items, out[0]), "xconv_orthogonalize")) return nullptr;
  if (!G.list) return THPVariable_Wrap(out[0]);
  THPObjectPtr list(PyList_New((Py_ssize_t)out.size()));
  if (!list) return nullptr;
  for (size_t i = 0; i < out.size(); ++i) PyList_SET_ITEM(list.get(), (Py_ssize_t)i, THPVariable_Wrap(out[i]));
  return list.release();
  XM_END
}

// muon_step(W, dW, M (or lists), lr, momentum, nesterov, weight_decay, steps, coefficients, eps, adjust) -> True
PyObject* muon_step(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  XM_BEGIN(11)
  xconv_update_desc d;
  int32_t adjust;
  const Several W(a[0]), G(a[1]), M(a[2]);
  if (W.size() == 0 || W.size() != G.size() || W.size() != M.size() || !steps_of(a[7], a[8], a[9], &d) || !number(a[3], &d.lr) || !number(a[4], &d.momentum) ||
      !PyBool_Check(a[5]) || !number(a[6], &d.weight_decay) || !PyLong_CheckExact(a[10]))
    Py_RETURN_NONE;
  adjust = (int32_t)PyLong_AsLong(a[10]);
  d.nesterov = a[5] == Py_True; d.adjust = adjust;
  std::vector<xconv_matrices> items((size_t)W.size());
  std::vector<at::Tensor> written, read;             // (held)
  for (Py_ssize_t i = 0; i < W.size(); ++i) {
    const at::Tensor *w = dense(W[i]), *g = dense(G[i]), *m = dense(M[i]);
    if (!w || !g || !m || g->sizes() != w->sizes() || m->sizes() != w->sizes() || m->scalar_type() != at::kFloat || !matrices_of(*w, &items[i])) Py_RETURN_NONE;
    items[i].G = g->data_ptr(); items[i].M = (float*)m->data_ptr(); items[i].O = w->data_ptr();
    items[i].g_dtype = dtype_code(*g); items[i].o_dtype = dtype_code(*w);
    written.push_back(*w); written.push_back(*m); read.push_back(*g);
  }
  if (!raise(update(lib.muon_step, d, items, written[0]), "xconv_muon_step")) return nullptr;
  // As every in-place operation: a graph that kept one of them for its backward pass says so.
  for (const at::Tensor& t : written)
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  Py_RETURN_TRUE;
  XM_END
}

// use_library(address of each entry point in the order of Library, raise(status, name), workspace(bytes, device))
PyObject* use_library(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  constexpr Py_ssize_t N = sizeof(Library) / sizeof(void*);
  if (nargs != N + 2) { PyErr_SetString(PyExc_TypeError, "use_library takes the entry points and two functions"); return nullptr; }
  void* at[N];
  for (Py_ssize_t i = 0; i < N; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  std::memcpy(&lib, at, sizeof lib);
  Py_INCREF(a[N]);
  Py_XSETREF(raise_for_status, a[N]);
  Py_INCREF(a[N + 1]);
  Py_XSETREF(workspace, a[N + 1]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
#define XM_FAST(F) {#F, (PyCFunction)(void (*)(void))F, METH_FASTCALL, nullptr}
    XM_FAST(forward), XM_FAST(sketch), XM_FAST(sketch_seeded), XM_FAST(wgrad), XM_FAST(wgrad_seeded), XM_FAST(dgrad), XM_FAST(backprobe), XM_FAST(contract),
    XM_FAST(layernorm), XM_FAST(layernorm_backward), XM_FAST(orthogonalize), XM_FAST(muon_step),
    XM_FAST(use_library), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (`key`: what the module was compiled against; binding.py and build.py compare it with what is installed)
PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&module_def);
  if (m && PyModule_AddStringConstant(m, "key", XM_KEY) != 0) { Py_DECREF(m); return nullptr; }
  return m;
}
