// Compiled binding of the operators that a training loop calls with torch tensors: the head losses, the gated norm
// pair, the embedding pair, the norms of queries and keys and the orthogonalised update.  Checks of arguments, output and workspace tensors from torch's allocator on the
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

int type_of(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == at::kBFloat16) return PPU_BF16;
  if (t.scalar_type() == at::kFloat) return PPU_F32;
  refuse(std::string(name) + " must be BFloat16 or Float, got " + c10::toString(t.scalar_type()));
}
at::ScalarType torch_type(int t) { return t == PPU_BF16 ? at::kBFloat16 : at::kFloat; }
// a tensor that is written over: as torch's own in-place calls, a graph that saved it is told, and one that leads to it is not cut
void overwritten(const at::Tensor& t, const char* name) {
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse(std::string("in_place: ") + name + " requires a gradient (call under torch.no_grad, or pass " + name + ".detach())");
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void* stream_of(int dev) { return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(); }

// ids, E, scale, dtype, flags
PyObject* embed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const at::Tensor &I = tensor(a[0], "ids"), &E = matrix(a[1], "E");
    const int dev = E.get_device(), V = as_int(E.size(0), "E"), d = as_int(E.size(1), "E"), et = type_of(E, "E");
    if (I.dim() != 1) refuse("ids must have one dimension");
    const int T = as_int(I.size(0), "ids");
    const int32_t* ids = (const int32_t*)dense(a[0], "ids", at::kInt, {T}, dev);
    const Rows e = rows(E, "E", E.scalar_type(), {V, d}, dev);
    const float scale = float_arg(a[2]);
    const int ot = int_arg(a[3], "dtype");
    int32_t* flags = (int32_t*)optional(a[4], "flags", at::kInt, {8}, dev);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
    const at::Tensor out = make({T, d}, torch_type(ot), dev);
    void* st = stream_of(dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_embed_fwd(ids, e.p, e.ld, et, scale, out.data_ptr(), d, ot, T, d, V, flags, st);
    }
    check(rc);
    return wrap(out);
  });
}

// ids, dout, V, scale, dtype, add, in_place, workspace, flags
PyObject* embed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const at::Tensor& D = matrix(a[1], "dout");
    const int dev = D.get_device(), T = as_int(D.size(0), "dout"), d = as_int(D.size(1), "dout"), V = int_arg(a[2], "V"), dt = type_of(D, "dout");
    const int32_t* ids = (const int32_t*)dense(a[0], "ids", at::kInt, {T}, dev);
    const Rows g = rows(D, "dout", D.scalar_type(), {T, d}, dev);
    const float scale = float_arg(a[3]);
    int gt = int_arg(a[4], "dtype");
    const bool in_place = truth_arg(a[6]);
    Rows add = {nullptr, d};
    if (a[5] != Py_None) {
      const at::Tensor& A = matrix(a[5], "add");
      const int at_ = type_of(A, "add");
      if (gt >= 0 && gt != at_) refuse("add must be of the gradient's type");
      gt = at_;
      add = rows(A, "add", A.scalar_type(), {V, d}, dev);
    }
    if (gt < 0) gt = PPU_BF16;
    int32_t* flags = (int32_t*)optional(a[8], "flags", at::kInt, {8}, dev);
    if (in_place && a[5] == Py_None) refuse("in_place needs add");
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
    size_t bytes = 0;
    check(ppu_embed_query_bytes(T, d, V, &bytes));
    const at::Tensor ws = workspace(a[7], bytes, dev);
    if (in_place) overwritten(THPVariable_Unpack(a[5]), "add");
    const at::Tensor out = in_place ? THPVariable_Unpack(a[5]) : make({V, d}, torch_type(gt), dev);
    void* st = stream_of(dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_embed_bwd(ids, g.p, g.ld, dt, scale, add.p, add.ld, out.data_ptr(), in_place ? add.ld : d, gt, T, d, V, ws.data_ptr(), (size_t)ws.numel(), flags, st);
    }
    check(rc);
    return wrap(out);
  });
}

struct Qk { Rows x; int T, n_q, n_k, n_v, dh, dev, per_head, seq, kind, rot, pairs; const float *q_gain, *k_gain, *freq; const int32_t* pos; float eps, base; };
const float* gain_of(PyObject* o, const char* name, int heads, int dh, int dev, int& per_head) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  const int each = t.dim() == 2;
  if (per_head >= 0 && per_head != each) refuse("gains of queries and keys must both be shared by the heads or both not");
  per_head = each;
  return (const float*)(each ? dense(o, name, at::kFloat, {heads, dh}, dev) : dense(o, name, at::kFloat, {dh}, dev));
}
// qkv, n_q, n_k, n_v, q_gain, k_gain, positions, seq, kind, eps, rope_base, inv_freq, rot_dim, pairs
Qk qk_operands(PyObject* const* a) {
  Qk q;
  const at::Tensor& X = matrix(a[0], "qkv");
  q.dev = X.get_device(); q.T = as_int(X.size(0), "qkv");
  q.n_q = int_arg(a[1], "n_q"); q.n_k = int_arg(a[2], "n_k"); q.n_v = int_arg(a[3], "n_v");
  const int64_t heads = (int64_t)q.n_q + q.n_k + q.n_v, cols = as_int(X.size(1), "qkv");
  if (q.n_q < 0 || q.n_k < 0 || q.n_v < 0 || heads < 1 || cols % heads) refuse("qkv must have a whole number of columns for each of its heads");
  q.dh = (int)(cols / heads);
  q.x = rows(X, "qkv", at::kBFloat16, {q.T, cols}, q.dev);
  q.per_head = -1;
  q.q_gain = gain_of(a[4], "q_gain", q.n_q, q.dh, q.dev, q.per_head);
  q.k_gain = gain_of(a[5], "k_gain", q.n_k, q.dh, q.dev, q.per_head);
  if (q.per_head < 0) q.per_head = 0;
  q.pos = (const int32_t*)optional(a[6], "positions", at::kInt, {q.T}, q.dev);
  q.seq = int_arg(a[7], "seq"); q.kind = int_arg(a[8], "kind");
  q.eps = float_arg(a[9]); q.base = float_arg(a[10]);
  q.rot = a[12] == Py_None ? q.dh : int_arg(a[12], "rot_dim");
  q.freq = a[11] == Py_None ? nullptr : (const float*)dense(a[11], "inv_freq", at::kFloat, {q.rot / 2}, q.dev);
  q.pairs = int_arg(a[13], "pairs");
  return q;
}

// the operands, in_place
PyObject* qk_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&] {
    const Qk q = qk_operands(a);
    const bool in_place = truth_arg(a[14]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)q.dev);
    const at::Tensor& X = THPVariable_Unpack(a[0]);
    if (in_place) overwritten(X, "qkv");
    const at::Tensor out = in_place ? X : make(X.sizes(), at::kBFloat16, q.dev);
    void* st = stream_of(q.dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_qk_norm_fwd(q.x.p, q.x.ld, q.q_gain, q.k_gain, q.per_head, q.pos, q.seq, q.kind, q.eps, q.base, q.freq, q.rot, q.pairs, out.data_ptr(),
                           in_place ? q.x.ld : X.size(1), q.T, q.n_q, q.n_k, q.n_v, q.dh, st);
    }
    check(rc);
    return wrap(out);
  });
}

// the operands, dout, in_place, workspace
PyObject* qk_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 17, [&] {
    const Qk q = qk_operands(a);
    const at::Tensor &X = THPVariable_Unpack(a[0]), &D = matrix(a[14], "dout");
    const Rows dy = rows(D, "dout", at::kBFloat16, X.sizes(), q.dev);
    const bool in_place = truth_arg(a[15]);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)q.dev);
    size_t bytes = 0;
    check(ppu_qk_norm_query_bytes(q.T, q.n_q, q.n_k, q.n_v, q.dh, q.per_head, &bytes));
    const at::Tensor ws = workspace(a[16], bytes, q.dev);
    if (in_place) overwritten(D, "dout");
    at::Tensor out[3] = {in_place ? D : make(X.sizes(), at::kBFloat16, q.dev), at::Tensor(), at::Tensor()};
    if (q.q_gain || a[4] != Py_None) out[1] = make(THPVariable_Unpack(a[4]).sizes(), at::kFloat, q.dev);
    if (q.k_gain || a[5] != Py_None) out[2] = make(THPVariable_Unpack(a[5]).sizes(), at::kFloat, q.dev);
    auto f = [&](int i) { return out[i].defined() ? (float*)out[i].data_ptr() : nullptr; };
    void* st = stream_of(q.dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_qk_norm_bwd(dy.p, dy.ld, q.x.p, q.x.ld, q.q_gain, q.k_gain, q.per_head, q.pos, q.seq, q.kind, q.eps, q.base, q.freq, q.rot, q.pairs, out[0].data_ptr(),
                           in_place ? dy.ld : X.size(1), f(1), f(2), q.T, q.n_q, q.n_k, q.n_v, q.dh, ws.data_ptr(), (size_t)ws.numel(), st);
    }
    check(rc);
    return tuple_of(out);
  });
}

// matrices [batch, m, n] (or one, [m, n]) whose rows may be strided: address, strides of rows and matrices
struct Matrices { void* p; int64_t ld, stride; };
Matrices matrices(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, int dev) {
  check_form(t, name, type, shape, dev);
  const int k = (int)t.dim();
  const int64_t m = t.size(k - 2), n = t.size(k - 1), batch = k == 3 ? t.size(0) : 1;
  Matrices r = {t.data_ptr(), m > 1 ? t.stride(k - 2) : n, 0};
  r.stride = batch > 1 ? t.stride(0) : m * r.ld;
  // (one matrix behind another, or the rows of all matrices beside one another: the heads of one projection)
  const bool behind = r.stride >= (m - 1) * r.ld + n, beside = r.stride >= n && r.ld >= (batch - 1) * r.stride + n;
  if ((n > 1 && t.stride(k - 1) != 1) || r.ld < n || (batch > 1 && !behind && !beside))
    refuse(std::string(name) + ": the values of a row must be adjacent, rows and matrices must not overlap");
  return r;
}

// G, momentum, beta, weight, nesterov, coefficients (a tuple of 3 or 3 steps), steps, eps, scale, in_place, workspace, flags
PyObject* orthogonalize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 12, [&] {
    const at::Tensor& G = tensor(a[0], "G");
    if (G.dim() != 2 && G.dim() != 3) refuse("G must have two or three dimensions");
    const int dev = G.get_device(), k = (int)G.dim(), gt = type_of(G, "G");
    const int m = as_int(G.size(k - 2), "G"), n = as_int(G.size(k - 1), "G"), batch = k == 3 ? as_int(G.size(0), "G") : 1;
    const Matrices g = matrices(G, "G", G.scalar_type(), G.sizes(), dev);
    Matrices mom = {}, mom_out = {};
    const bool has = a[1] != Py_None;
    if (has) mom = matrices(tensor(a[1], "momentum"), "momentum", at::kFloat, G.sizes(), dev);
    const float beta = float_arg(a[2]), weight = float_arg(a[3]);
    const bool nesterov = truth_arg(a[4]);
    float coef[96];
    if (!PyTuple_Check(a[5]) || PyTuple_GET_SIZE(a[5]) % 3 || PyTuple_GET_SIZE(a[5]) > 96) refuse("coef must be a triple, or one for each step");
    const int n_coef = (int)PyTuple_GET_SIZE(a[5]) / 3;
    for (int i = 0; i < 3 * n_coef; ++i) coef[i] = float_arg(PyTuple_GET_ITEM(a[5], i));
    const int steps = int_arg(a[6], "steps");
    const float eps = float_arg(a[7]), scale = float_arg(a[8]);
    const bool in_place = truth_arg(a[9]);
    if (in_place && !has) refuse("in_place needs a momentum");
    int32_t* flags = (int32_t*)optional(a[11], "flags", at::kInt, {8}, dev);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
    size_t bytes = 0;
    check(ppu_orthogonalize_query_bytes(batch, m, n, steps, &bytes));
    const at::Tensor ws = workspace(a[10], bytes, dev);
    at::Tensor out[2] = {make(G.sizes(), at::kBFloat16, dev), at::Tensor()};
    if (in_place) { overwritten(THPVariable_Unpack(a[1]), "momentum"); out[1] = THPVariable_Unpack(a[1]); mom_out = mom; }
    else if (has) { out[1] = make(G.sizes(), at::kFloat, dev); mom_out = {out[1].data_ptr(), n, (int64_t)m * n}; }
    void* st = stream_of(dev);
    int rc;
    {
      NoGil nogil;
      rc = ppu_orthogonalize(g.p, g.ld, g.stride, gt, (const float*)mom.p, mom.ld, mom.stride, (float*)mom_out.p, mom_out.ld, mom_out.stride, beta, weight, nesterov, coef,
                             n_coef, steps, eps, scale, out[0].data_ptr(), batch, m, n, ws.data_ptr(), (size_t)ws.numel(), flags, st);
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
PyMethodDef methods[] = {FAST(head_xent), FAST(head_distill), FAST(norm_gate_fwd), FAST(norm_gate_bwd), FAST(embed_fwd), FAST(embed_bwd), FAST(qk_norm_fwd), FAST(qk_norm_bwd), FAST(orthogonalize),
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__ops(void) { return PyModule_Create(&module); }
