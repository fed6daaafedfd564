// Native part of the Python binding: the calls of the training step that are small enough for Python's own time to
// count (norms, rotary positions, gradient norm and clipping).  Each checks its tensors, makes its outputs on the current stream
// of their device and calls the C entry point (include/dflare.h), whose address dflare.py hands over once.
// In Python the same work made a norm of 16 rows 11 us long instead of 7.0 (its kernel takes 3.7), rotary positions of 32 rows
// 16 instead of 6.3 (3.8), and a list of 301 gradients 0.8 ms instead of 38 us.
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <string>
#include <vector>

#include "dflare.h"

namespace {

decltype(&dflare_norm_fwd) p_norm_fwd;
decltype(&dflare_norm_bwd_workspace) p_norm_bwd_workspace;
decltype(&dflare_norm_bwd) p_norm_bwd;
decltype(&dflare_rope) p_rope;
decltype(&dflare_grad_norm_workspace) p_grad_norm_workspace;
decltype(&dflare_grad_norm) p_grad_norm;
decltype(&dflare_clip_grads) p_clip_grads;
PyObject* p_raw_stream;     // device index -> address of its current stream
PyObject* p_out_of_memory;  // torch's exception

// a refusal: the Python exception and what it says
struct Refused {
  PyObject* type;
  std::string why;
};
[[noreturn]] void type_error(const std::string& why) { throw Refused{PyExc_TypeError, why}; }
[[noreturn]] void value_error(const std::string& why) { throw Refused{PyExc_ValueError, why}; }

int type_code(const at::Tensor& t) {
  const auto s = t.scalar_type();
  if (s == at::kFloat) return DFLARE_F32;
  if (s == at::kBFloat16 || s == at::kShort || s == at::kUInt16) return DFLARE_BF16;  // 16-bit integers: bf16 bits
  type_error("expected a bf16 or fp32 tensor");
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) type_error("expected a device tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) type_error("expected a device tensor");
  return t;
}
const at::Tensor& dense(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (!t.is_contiguous()) value_error("tensor must be contiguous");
  return t;
}
// address of a contiguous tensor of these sizes on ref's device, of type `exact` or of ref's; null for None
void* like(PyObject* o, const char* name, at::IntArrayRef sizes, const at::Tensor& ref, at::ScalarType exact = at::ScalarType::Undefined) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = dense(o);
  if (t.sizes() != sizes) value_error(std::string(name) + " has another shape than expected");
  if (t.device() != ref.device()) value_error(std::string(name) + " is on another device");
  if (exact == at::ScalarType::Undefined ? type_code(t) != type_code(ref) : t.scalar_type() != exact)
    type_error(std::string(name) + " has another type than expected");
  return t.data_ptr();
}
int32_t to32(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) value_error(std::string(name) + " is beyond 32 bits");
  return (int32_t)v;
}
// the current stream of the device, which is current while the guard lives
struct Here {
  c10::DeviceGuard guard;
  void* stream;
  explicit Here(const at::Device& d) : guard(d) {
    PyObject* r = PyObject_CallFunction(p_raw_stream, "i", (int)d.index());
    stream = r ? PyLong_AsVoidPtr(r) : nullptr;
    Py_XDECREF(r);
    if (PyErr_Occurred()) throw Refused{PyExc_RuntimeError, "no current stream on the tensors' device"};
  }
};
template <typename F>
int unlocked(F&& f) {
  PyThreadState* state = PyEval_SaveThread();
  const int rc = f();
  PyEval_RestoreThread(state);
  return rc;
}
at::Tensor fresh(at::IntArrayRef sizes, const at::Tensor& ref, at::ScalarType type) {
  return at::empty(sizes, ref.options().dtype(type));
}
PyObject* wrapped(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// Every function gives its outputs, or the status of a call that was refused.

// norm_fwd(x, gain, bias, residual, kind, eps) -> (y, h, mean, rstd)
PyObject* norm_fwd(PyObject* const* a) {
  const at::Tensor& x = dense(a[0]);
  const int dtype = type_code(x);
  if (x.dim() != 2) value_error("expected a [rows, H] tensor");
  const int32_t rows = to32(x.size(0), "rows"), H = to32(x.size(1), "H");
  void *gain = like(a[1], "gain", {H}, x), *bias = like(a[2], "bias", {H}, x), *res = like(a[3], "residual", x.sizes(), x);
  const int32_t kind = to32(PyLong_AsLongLong(a[4]), "kind");
  const double eps = PyFloat_AsDouble(a[5]);
  if (PyErr_Occurred()) return nullptr;
  const Here here(x.device());
  const at::Tensor h = res ? fresh(x.sizes(), x, x.scalar_type()) : x, y = fresh(x.sizes(), x, x.scalar_type());
  const at::Tensor mean = kind == DFLARE_NORM_LAYER ? fresh({rows}, x, at::kFloat) : at::Tensor(), rstd = fresh({rows}, x, at::kFloat);
  const int rc = unlocked([&] {
    return p_norm_fwd(x.data_ptr(), res, gain, bias, rows, H, dtype, kind, (float)eps, res ? h.data_ptr() : nullptr, y.data_ptr(),
                      (float*)address(mean), (float*)rstd.data_ptr(), here.stream);
  });
  if (rc != DFLARE_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("NNNN", wrapped(y), res ? wrapped(h) : Py_NewRef(a[0]), wrapped(mean), wrapped(rstd));
}

// norm_bwd(dy, h, gain, mean, rstd, dsum, kind) -> (dx, dgain, dbias)
PyObject* norm_bwd(PyObject* const* a) {
  const at::Tensor& h = dense(a[1]);
  const int dtype = type_code(h);
  if (h.dim() != 2) value_error("expected a [rows, H] tensor");
  const int32_t rows = to32(h.size(0), "rows"), H = to32(h.size(1), "H");
  void *dy = like(a[0], "dy", h.sizes(), h), *gain = like(a[2], "gain", {H}, h), *dsum = like(a[5], "dsum", h.sizes(), h);
  void *mean = like(a[3], "mean", {rows}, h, at::kFloat), *rstd = like(a[4], "rstd", {rows}, h, at::kFloat);
  const int32_t kind = to32(PyLong_AsLongLong(a[6]), "kind");
  if (PyErr_Occurred()) return nullptr;
  const Here here(h.device());
  const at::Tensor dx = fresh(h.sizes(), h, h.scalar_type()), dgain = fresh({H}, h, at::kFloat);
  const at::Tensor dbias = kind == DFLARE_NORM_LAYER ? fresh({H}, h, at::kFloat) : at::Tensor();
  const size_t bytes = p_norm_bwd_workspace(rows, H, kind);
  const at::Tensor ws = fresh({(int64_t)std::max<size_t>(bytes, 16)}, h, at::kByte);
  const int rc = unlocked([&] {
    return p_norm_bwd(dy, h.data_ptr(), gain, (const float*)mean, (const float*)rstd, dsum, rows, H, dtype, kind, dx.data_ptr(),
                      (float*)dgain.data_ptr(), (float*)address(dbias), ws.data_ptr(), bytes, here.stream);
  });
  if (rc != DFLARE_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("NNN", wrapped(dx), wrapped(dgain), wrapped(dbias));
}

// rope(tuple of one or two x, inv_freq, positions, B, layout, scale, inverse, None or tuple of outputs) -> tuple of outputs
PyObject* rope(PyObject* const* a) {
  if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) < 1 || PyTuple_GET_SIZE(a[0]) > 2) value_error("expected one tensor or a pair");
  const int n = (int)PyTuple_GET_SIZE(a[0]);
  const bool given = a[7] != Py_None;
  if (given && (!PyTuple_Check(a[7]) || PyTuple_GET_SIZE(a[7]) != n)) value_error("out and x differ in number");
  const at::Tensor& first = tensor(PyTuple_GET_ITEM(a[0], 0));
  const int dtype = type_code(first);
  if (first.dim() != 3) value_error("expected [rows, n_heads, head_dim] tensors");
  const int32_t rows = to32(first.size(0), "rows"), hd = to32(first.size(2), "head_dim"), B = to32(PyLong_AsLongLong(a[3]), "B");
  const int32_t layout = to32(PyLong_AsLongLong(a[4]), "layout");
  const double scale = PyFloat_AsDouble(a[5]);
  const int inverse = PyObject_IsTrue(a[6]);
  if (PyErr_Occurred()) return nullptr;
  if (B < 1) value_error("B must be positive");
  const at::Tensor& freq = dense(a[1]);
  like(a[1], "inv_freq", {freq.numel()}, first, at::kDouble);
  void* pos = like(a[2], "positions", {((int64_t)rows + B - 1) / B}, first, at::kInt);
  const Here here(first.device());
  dflare_rope_tensor tab[2] = {};
  at::Tensor outs[2];
  for (int k = 0; k < n; ++k) {
    const at::Tensor& x = tensor(PyTuple_GET_ITEM(a[0], k));
    if (x.dim() != 3 || x.size(0) != rows || x.size(2) != hd) value_error("expected [rows, n_heads, head_dim] tensors with the same rows and head_dim");
    if (type_code(x) != dtype || x.device() != first.device()) value_error("the tensors differ in type or device");
    outs[k] = given ? tensor(PyTuple_GET_ITEM(a[7], k)) : fresh(x.sizes(), x, x.scalar_type());
    const at::Tensor& y = outs[k];
    if (y.sizes() != x.sizes() || y.scalar_type() != x.scalar_type() || y.device() != x.device()) value_error("x and out differ in shape, type or device");
    if (hd > 1 && x.numel() && (x.stride(2) != 1 || y.stride(2) != 1)) value_error("the last dimension must be contiguous");
    tab[k] = {x.data_ptr(), y.data_ptr(), x.stride(0), x.stride(1), y.stride(0), y.stride(1), to32(x.size(1), "n_heads")};
  }
  const int32_t rot = to32(2 * freq.numel(), "rotary_dim");
  const int rc = unlocked([&] {
    return p_rope(tab, n, (const int32_t*)pos, (const double*)freq.data_ptr(), rows, B, hd, rot, dtype, layout, (float)scale, inverse,
                  here.stream);
  });
  if (rc != DFLARE_OK) return PyLong_FromLong(rc);
  if (given) return Py_NewRef(a[7]);
  return n == 1 ? Py_BuildValue("(N)", wrapped(outs[0])) : Py_BuildValue("NN", wrapped(outs[0]), wrapped(outs[1]));
}

// the entries of a list of gradients, with the outputs of another list or None; gives the first tensor
const at::Tensor& grad_table(PyObject* grads, PyObject* outs, std::vector<dflare_grad_tensor>& table) {
  if (!PyList_Check(grads) || (outs != Py_None && !PyList_Check(outs))) type_error("expected a list");
  const Py_ssize_t n = PyList_GET_SIZE(grads);
  if (n < 1) value_error("expected at least one gradient");
  to32(n, "the number of gradients");
  if (outs != Py_None && PyList_GET_SIZE(outs) != n) value_error("out and grads differ in number");
  const at::Tensor& first = dense(PyList_GET_ITEM(grads, 0));
  table.resize(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor& t = dense(PyList_GET_ITEM(grads, i));
    if (t.device() != first.device()) value_error("the gradients are on different devices");
    table[i] = {t.data_ptr(), nullptr, t.numel(), type_code(t)};
    if (outs == Py_None) continue;
    const at::Tensor& o = dense(PyList_GET_ITEM(outs, i));
    if (type_code(o) != table[i].dtype || o.device() != first.device() || o.sizes() != t.sizes())
      value_error("out and grads differ in shape, type or device");
    table[i].out = o.data_ptr();
  }
  return first;
}

// grad_norm(grads) -> (norm, sumsq)
PyObject* grad_norm(PyObject* const* a) {
  std::vector<dflare_grad_tensor> table;
  const at::Tensor& first = grad_table(a[0], Py_None, table);
  const int32_t n = (int32_t)table.size();
  const Here here(first.device());
  const at::Tensor sumsq = fresh({1}, first, at::kDouble), norm = fresh({1}, first, at::kFloat);
  const size_t bytes = p_grad_norm_workspace(n);
  const at::Tensor ws = fresh({(int64_t)bytes}, first, at::kByte);
  const int rc = unlocked([&] {
    return p_grad_norm(table.data(), n, (double*)sumsq.data_ptr(), (float*)norm.data_ptr(), ws.data_ptr(), bytes, here.stream);
  });
  return rc != DFLARE_OK ? PyLong_FromLong(rc) : Py_BuildValue("NN", wrapped(norm), wrapped(sumsq));
}

// clip_grads(grads, sumsq, max_norm, outs or None) -> status
PyObject* clip_grads(PyObject* const* a) {
  std::vector<dflare_grad_tensor> table;
  const at::Tensor& first = grad_table(a[0], a[3], table);
  const double max_norm = PyFloat_AsDouble(a[2]);
  if (PyErr_Occurred()) return nullptr;
  dense(a[1]);
  const void* sumsq = like(a[1], "sumsq", {1}, first, at::kDouble);
  const Here here(first.device());
  return PyLong_FromLong(unlocked([&] {
    return p_clip_grads(table.data(), (int32_t)table.size(), (const double*)sumsq, (float)max_norm, here.stream);
  }));
}

// F with exactly N arguments, its refusals and C++ exceptions as Python's
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Refused& r) {
    PyErr_Clear();
    PyErr_SetString(r.type, r.why.c_str());
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(p_out_of_memory, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// bind(addresses of the entry points in the order below, function from a device index to its current stream's address,
// torch's out-of-memory exception)
PyObject* bind(PyObject* const* a) {
  void** to[] = {(void**)&p_norm_fwd, (void**)&p_norm_bwd_workspace, (void**)&p_norm_bwd, (void**)&p_rope,
                 (void**)&p_grad_norm_workspace, (void**)&p_grad_norm, (void**)&p_clip_grads};
  for (int k = 0; k < 7; ++k) *to[k] = PyLong_AsVoidPtr(a[k]);
  if (PyErr_Occurred()) return nullptr;
  p_raw_stream = Py_NewRef(a[7]);
  p_out_of_memory = Py_NewRef(a[8]);
  return Py_NewRef(Py_None);
}

#define FUNCTION(f, n) {#f, (PyCFunction)(void*)guarded<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FUNCTION(bind, 9), FUNCTION(norm_fwd, 6), FUNCTION(norm_bwd, 7), FUNCTION(rope, 8), FUNCTION(grad_norm, 1),
                         FUNCTION(clip_grads, 4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
