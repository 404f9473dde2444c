// Compiled binding of the operators that a training loop calls with torch tensors: the head losses and
// the gated norm pair.  Checks of arguments, output and workspace tensors from torch's allocator on the
// operands' device and its current stream, then the C call.  These operators take a few microseconds on small
// inputs; the same binding written in Python took 18 to 36 us of host time a call where this takes 7 to 20.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <climits>
#include <string>
#include "../../include/ppu.h"

namespace {

PyObject* g_error = nullptr;                 // PpuError(code, message)

struct Refused { int code; std::string what; };
[[noreturn]] void refuse(const std::string& what, int code = PPU_EINVAL) { throw Refused{code, what}; }

std::string shape_text(at::IntArrayRef s) {
  std::string t = "(";
  for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + (s.size() == 1 ? ",)" : ")");
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a CUDA tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse(std::string(name) + " must be a CUDA tensor");
  return t;
}
const at::Tensor& matrix(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 2) refuse(std::string(name) + " must have two dimensions");
  return t;
}
void check_form(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, int device) {
  if (t.scalar_type() != type)
    refuse(std::string(name) + " must be " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  if (t.sizes() != shape) refuse(std::string(name) + " must have shape " + shape_text(shape) + ", got " + shape_text(t.sizes()));
  if (t.get_device() != device)
    refuse(std::string(name) + " is on cuda:" + std::to_string(t.get_device()) + ", other operands on cuda:" + std::to_string(device));
}
// address of a contiguous tensor of this type and shape
void* dense(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape, int device) {
  const at::Tensor& t = tensor(o, name);
  check_form(t, name, type, shape, device);
  if (!t.is_contiguous()) refuse(std::string(name) + " must be contiguous");
  return t.data_ptr();
}
void* optional(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape, int device) {
  return o == Py_None ? nullptr : dense(o, name, type, shape, device);
}
// address and row stride of a matrix whose rows may be strided
struct Rows { void* p; int64_t ld; };
Rows rows(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, int device) {
  check_form(t, name, type, shape, device);
  const int64_t n = shape[0], m = shape[1];
  if (!t.is_contiguous() && ((m > 1 && t.stride(1) != 1) || (n > 1 && t.stride(0) < m)))
    refuse(std::string(name) + ": the values of a row must be adjacent and rows must not overlap");
  return {t.data_ptr(), n > 1 ? t.stride(0) : m};
}
int as_int(int64_t v, const char* name) {
  if (v > INT_MAX || v < INT_MIN) refuse(std::string(name) + " is too large", PPU_ESHAPE);
  return (int)v;
}
int int_arg(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return as_int(v, name);
}
bool truth_arg(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}
float float_arg(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, int device) {
  return at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}
// the caller's workspace, or one of this call (its memory goes back to the allocator when the call
// returns, for later work on the same stream)
at::Tensor workspace(PyObject* given, size_t bytes, int device) {
  if (given == Py_None) return make({(int64_t)(bytes < 256 ? 256 : bytes)}, at::kByte, device);
  const at::Tensor& t = tensor(given, "workspace");
  if (t.scalar_type() != at::kByte || !t.is_contiguous() || t.get_device() != device)
    refuse("workspace must be a contiguous uint8 tensor on the operands' device");
  return t;
}
void check(int rc) { if (rc != PPU_OK) refuse(ppu_last_error(), rc); }

PyObject* wrap(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
template <size_t N>
PyObject* tuple_of(const at::Tensor (&ts)[N]) {
  PyObject* out = PyTuple_New(N);
  if (!out) throw python_error();
  for (size_t i = 0; i < N; ++i) {
    PyObject* o = wrap(ts[i]);
    if (!o) { Py_DECREF(out); throw python_error(); }
    PyTuple_SET_ITEM(out, i, o);
  }
  return out;
}
struct NoGil {
  PyThreadState* s = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(s); }
};

// runs a binding, turning refusals into PpuError and torch's exceptions into torch's
template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F body) {
  HANDLE_TH_ERRORS
  try {
    if (given != wanted) refuse("wrong number of arguments");
    return body();
  } catch (const Refused& r) {
    PyObject* args = Py_BuildValue("(is)", r.code, r.what.c_str());
    PyErr_SetObject(g_error ? g_error : PyExc_RuntimeError, args);
    Py_XDECREF(args);
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

struct Head { Rows X, E; int T, d, V, dev; };
Head head_operands(PyObject* x, PyObject* e) {
  const at::Tensor &X = matrix(x, "X"), &E = matrix(e, "E");
  Head h;
  h.T = as_int(X.size(0), "X"); h.d = as_int(X.size(1), "X"); h.V = as_int(E.size(0), "E");
  h.dev = X.get_device();
  h.X = rows(X, "X", at::kBFloat16, {h.T, h.d}, h.dev);
  h.E = rows(E, "E", at::kBFloat16, {h.V, h.d}, h.dev);
  return h;
}
// outputs and workspace of a head loss; call(loss, row_loss, lse, dX, dE, workspace, bytes, stream)
template <typename F>
PyObject* head_call(const Head& h, int k, int grads, int chunk_rows, PyObject* ws_given, F call) {
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)h.dev);
  size_t bytes = 0;
  check(ppu_head_query_bytes(h.T, h.d, h.V, grads, chunk_rows, k, &bytes));
  const at::Tensor ws = workspace(ws_given, bytes, h.dev);
  at::Tensor out[5] = {make({}, at::kFloat, h.dev), make({h.T}, at::kFloat, h.dev), make({h.T}, at::kFloat, h.dev), at::Tensor(), at::Tensor()};
  if (grads & 1) out[3] = make({h.T, h.d}, at::kBFloat16, h.dev);
  if (grads & 2) out[4] = make({h.V, h.d}, at::kBFloat16, h.dev);
  void* dX = (grads & 1) ? out[3].data_ptr() : nullptr;      // (null without rows)
  void* dE = (grads & 2) ? out[4].data_ptr() : nullptr;
  const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h.dev);
  int rc;
  {
    NoGil nogil;
    rc = call((float*)out[0].data_ptr(), (float*)out[1].data_ptr(), (float*)out[2].data_ptr(), dX, dE, ws.data_ptr(), (size_t)ws.numel(),
              (void*)st.stream());
  }
  check(rc);
  return tuple_of(out);
}

PyObject* head_xent(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const Head h = head_operands(a[0], a[1]);
    const int32_t* target = (const int32_t*)dense(a[2], "target", at::kInt, {h.T}, h.dev);
    const float* w = (const float*)optional(a[3], "row_weight", at::kFloat, {h.T}, h.dev);
    const int grads = int_arg(a[4], "grad"), chunk = int_arg(a[5], "chunk_rows");
    int32_t* flags = (int32_t*)optional(a[7], "flags", at::kInt, {8}, h.dev);
    return head_call(h, 1, grads, chunk, a[6], [&](float* loss, float* row, float* lse, void* dX, void* dE, void* ws, size_t nb, void* st) {
      return ppu_head_xent(h.X.p, h.X.ld, h.E.p, h.E.ld, target, w, h.T, h.d, h.V, loss, row, lse, dX, h.d, dE, h.d, chunk, ws, nb, flags, st);
    });
  });
}

PyObject* head_distill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    const Head h = head_operands(a[0], a[1]);
    const at::Tensor &I = matrix(a[2], "teacher_ids"), &Z = matrix(a[3], "teacher_logits");
    const int k = as_int(I.size(1), "teacher_ids");
    const Rows ids = rows(I, "teacher_ids", at::kInt, {h.T, k}, h.dev), z = rows(Z, "teacher_logits", at::kFloat, {h.T, k}, h.dev);
    const float temp = float_arg(a[4]);
    const float* tl = (const float*)optional(a[5], "teacher_lse", at::kFloat, {h.T}, h.dev);
    const float* w = (const float*)optional(a[6], "row_weight", at::kFloat, {h.T}, h.dev);
    const int grads = int_arg(a[7], "grad"), chunk = int_arg(a[8], "chunk_rows");
    int32_t* flags = (int32_t*)optional(a[10], "flags", at::kInt, {8}, h.dev);
    return head_call(h, k, grads, chunk, a[9], [&](float* loss, float* row, float* lse, void* dX, void* dE, void* ws, size_t nb, void* st) {
      return ppu_head_distill(h.X.p, h.X.ld, h.E.p, h.E.ld, (const int32_t*)ids.p, ids.ld, (const float*)z.p, z.ld, k, tl, temp, w, h.T, h.d, h.V,
                              loss, row, lse, dX, h.d, dE, h.d, chunk, ws, nb, flags, st);
    });
  });
}

struct Norm { const void* y; const float *r, *gate, *g1, *b1, *g2, *b2; int T, d, dev, gate_rows; };
Norm norm_operands(PyObject* y, PyObject* r, PyObject* g1, PyObject* g2, PyObject* b1, PyObject* b2, PyObject* gate, PyObject* gate_rows) {
  Norm o;
  const at::Tensor& Y = matrix(y, "y");
  o.T = as_int(Y.size(0), "y"); o.d = as_int(Y.size(1), "y");
  o.dev = Y.get_device();
  o.y = dense(y, "y", at::kBFloat16, {o.T, o.d}, o.dev);
  o.r = (const float*)dense(r, "r", at::kFloat, {o.T, o.d}, o.dev);
  o.g1 = (const float*)dense(g1, "post_gain", at::kFloat, {o.d}, o.dev);
  o.g2 = (const float*)dense(g2, "pre_gain", at::kFloat, {o.d}, o.dev);
  o.b1 = (const float*)optional(b1, "post_shift", at::kFloat, {o.d}, o.dev);
  o.b2 = (const float*)optional(b2, "pre_shift", at::kFloat, {o.d}, o.dev);
  o.gate = nullptr;
  o.gate_rows = 0;
  if (gate != Py_None) {
    o.gate_rows = int_arg(gate_rows, "gate_rows");
    if (o.gate_rows < 0) refuse("gate_rows must not be negative");
    const bool one = o.gate_rows == 0;       // one row for all rows; without any it may also be left out
    if (one) o.gate_rows = o.T > 0 ? o.T : 1;
    int64_t n = ((int64_t)o.T + o.gate_rows - 1) / o.gate_rows;
    if (one && o.T == 0 && matrix(gate, "gate").size(0) == 1) n = 1;
    o.gate = (const float*)dense(gate, "gate", at::kFloat, {n, o.d}, o.dev);
  }
  return o;
}

PyObject* norm_gate_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    const Norm o = norm_operands(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
    const int kind = int_arg(a[8], "kind");
    const bool in_place = truth_arg(a[11]);
    const float scale = float_arg(a[9]), eps = float_arg(a[10]);
    if (in_place) {                          // as torch's own in-place calls: a graph that saved r is told, and one that leads to r is not cut
      const at::Tensor& r = THPVariable_Unpack(a[1]);
      if (r.requires_grad() && c10::GradMode::is_enabled()) refuse("in_place: r requires a gradient (call under torch.no_grad, or pass r.detach())");
      if (!r.is_inference()) r.unsafeGetTensorImpl()->bump_version();
    }
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)o.dev);
    const at::Tensor out[3] = {in_place ? THPVariable_Unpack(a[1]) : make({o.T, o.d}, at::kFloat, o.dev), make({o.T, o.d}, at::kBFloat16, o.dev),
                               make({o.T, 4}, at::kFloat, o.dev)};
    const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)o.dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_norm_gate_fwd(o.y, o.r, o.gate, o.gate_rows, o.g1, o.b1, o.g2, o.b2, kind, scale, eps, (float*)out[0].data_ptr(), out[1].data_ptr(),
                             (float*)out[2].data_ptr(), o.T, o.d, (void*)st.stream());
    }
    check(rc);
    return tuple_of(out);
  });
}

PyObject* norm_gate_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&] {
    const Norm o = norm_operands(a[2], a[3], a[5], a[6], a[7], a[8], a[9], a[10]);
    const void* dh = dense(a[0], "dh", at::kBFloat16, {o.T, o.d}, o.dev);
    const float* dr = (const float*)optional(a[1], "dr_out", at::kFloat, {o.T, o.d}, o.dev);
    const float* stats = (const float*)dense(a[4], "stats", at::kFloat, {o.T, 4}, o.dev);
    const int kind = int_arg(a[11], "kind");
    const float scale = float_arg(a[12]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)o.dev);
    size_t bytes = 0;
    check(ppu_norm_gate_query_bytes(o.T, o.d, o.gate_rows, &bytes));
    const at::Tensor ws = workspace(a[13], bytes, o.dev);
    at::Tensor out[7] = {make({o.T, o.d}, at::kBFloat16, o.dev), make({o.T, o.d}, at::kFloat, o.dev), make({o.d}, at::kFloat, o.dev), at::Tensor(),
                         make({o.d}, at::kFloat, o.dev), at::Tensor(), at::Tensor()};
    if (o.b1) out[3] = make({o.d}, at::kFloat, o.dev);
    if (o.b2) out[5] = make({o.d}, at::kFloat, o.dev);
    if (o.gate || a[9] != Py_None) out[6] = o.T ? at::empty_like(THPVariable_Unpack(a[9])) : at::zeros_like(THPVariable_Unpack(a[9]));
    auto f = [&](int i) { return out[i].defined() ? (float*)out[i].data_ptr() : nullptr; };
    const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)o.dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_norm_gate_bwd(dh, dr, o.y, o.r, stats, o.gate, o.gate_rows, o.g1, o.b1, o.g2, kind, scale, out[0].data_ptr(), f(1), f(2), f(3), f(4),
                             f(5), o.gate ? f(6) : nullptr, o.T, o.d, ws.data_ptr(), (size_t)ws.numel(), (void*)st.stream());
    }
    check(rc);
    return tuple_of(out);
  });
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(head_xent), FAST(head_distill), FAST(norm_gate_fwd), FAST(norm_gate_bwd), {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__ops(void) { return PyModule_Create(&module); }
