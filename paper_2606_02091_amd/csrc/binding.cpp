// Native part of the Python binding: the calls of the training step that are small enough for Python's own time to
// count (norms, rotary positions, projections of few rows, gradient norm and clipping, AdamW).  Each checks its tensors, makes its outputs on the current stream
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
decltype(&dflare_qk_norm_rope_fwd) p_qk_norm_rope_fwd;
decltype(&dflare_qk_norm_rope_bwd_workspace) p_qk_norm_rope_bwd_workspace;
decltype(&dflare_qk_norm_rope_bwd) p_qk_norm_rope_bwd;
decltype(&dflare_linear_plan) p_linear_plan;
decltype(&dflare_linear_fwd) p_linear_fwd;
decltype(&dflare_linear_bwd) p_linear_bwd;
decltype(&dflare_gated_plan) p_gated_plan;
decltype(&dflare_gated_fwd) p_gated_fwd;
decltype(&dflare_gated_bwd) p_gated_bwd;
decltype(&dflare_adamw) p_adamw;
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
  if (!THPVariable_CheckExact(o) && !THPVariable_Check(o)) type_error("expected a device tensor");
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

// one or two [rows, n_heads, head_dim] tensors with the positions, gains and numbers of a call on them
struct Heads {
  int n = 0;
  const at::Tensor* x[2];
  PyObject* x_items[2];
  void* gain[2];
  int32_t rows, hd, rot, B, layout;
  int dtype;
  double scale, eps;
  void *positions, *freq;
  // (x tuple, gain tuple, inv_freq, positions, B, layout, scale, eps)
  explicit Heads(PyObject* const* a) {
    if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) < 1 || PyTuple_GET_SIZE(a[0]) > 2) value_error("expected one tensor or a pair");
    n = (int)PyTuple_GET_SIZE(a[0]);
    if (!PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != n) value_error("gain and x differ in number");
    B = to32(PyLong_AsLongLong(a[4]), "B");
    layout = to32(PyLong_AsLongLong(a[5]), "layout");
    scale = PyFloat_AsDouble(a[6]);
    eps = PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) throw Refused{nullptr, ""};
    if (B < 1) value_error("B must be positive");
    const at::Tensor& first = tensor(PyTuple_GET_ITEM(a[0], 0));
    dtype = type_code(first);
    if (first.dim() != 3) value_error("expected [rows, n_heads, head_dim] tensors");
    rows = to32(first.size(0), "rows");
    hd = to32(first.size(2), "head_dim");
    const at::Tensor& f = dense(a[2]);
    freq = like(a[2], "inv_freq", {f.numel()}, first, at::kDouble);
    rot = to32(2 * f.numel(), "rotary_dim");
    positions = like(a[3], "positions", {((int64_t)rows + B - 1) / B}, first, at::kInt);
    for (int k = 0; k < n; ++k) {
      x_items[k] = PyTuple_GET_ITEM(a[0], k);
      x[k] = &tensor(x_items[k]);
      if (x[k]->dim() != 3 || x[k]->size(0) != rows || x[k]->size(2) != hd)
        value_error("expected [rows, n_heads, head_dim] tensors with the same rows and head_dim");
      if (type_code(*x[k]) != dtype || x[k]->device() != first.device()) value_error("the tensors differ in type or device");
      contiguous_heads(*x[k]);
      gain[k] = like(PyTuple_GET_ITEM(a[1], k), "gain", {hd}, first);
      to32(x[k]->size(1), "n_heads");
    }
  }
  void contiguous_heads(const at::Tensor& t) const {
    if (hd > 1 && t.numel() && t.stride(2) != 1) value_error("the last dimension must be contiguous");
  }
  // a tensor beside x[k]
  const at::Tensor& beside(PyObject* o, int k, const char* name) const {
    const at::Tensor& t = tensor(o);
    if (t.sizes() != x[k]->sizes() || t.device() != x[k]->device()) value_error(std::string(name) + " and x differ in shape or device");
    if (type_code(t) != dtype) type_error(std::string(name) + " and x differ in type");
    contiguous_heads(t);
    return t;
  }
};
PyObject* pair_of(const at::Tensor (&t)[2], int n) { return n == 1 ? Py_BuildValue("(N)", wrapped(t[0])) : Py_BuildValue("NN", wrapped(t[0]), wrapped(t[1])); }

// qk_norm_rope_fwd(x, gain, inv_freq, positions, B, layout, scale, eps, None or tuple of outputs) -> tuple of outputs
PyObject* qk_norm_rope_fwd(PyObject* const* a) {
  const Heads h(a);
  const bool given = a[8] != Py_None;
  if (given && (!PyTuple_Check(a[8]) || PyTuple_GET_SIZE(a[8]) != h.n)) value_error("out and x differ in number");
  const Here here(h.x[0]->device());
  dflare_qk_tensor tab[2] = {};
  at::Tensor outs[2];
  for (int k = 0; k < h.n; ++k) {
    const at::Tensor& x = *h.x[k];
    outs[k] = given ? h.beside(PyTuple_GET_ITEM(a[8], k), k, "out") : fresh(x.sizes(), x, x.scalar_type());
    const at::Tensor& y = outs[k];
    tab[k] = {x.data_ptr(), y.data_ptr(), h.gain[k], x.stride(0), x.stride(1), y.stride(0), y.stride(1), (int32_t)x.size(1)};
  }
  const int rc = unlocked([&] {
    return p_qk_norm_rope_fwd(tab, h.n, (const int32_t*)h.positions, (const double*)h.freq, h.rows, h.B, h.hd, h.rot, h.dtype, h.layout,
                              (float)h.scale, (float)h.eps, here.stream);
  });
  if (rc != DFLARE_OK) return PyLong_FromLong(rc);
  return given ? Py_NewRef(a[8]) : pair_of(outs, h.n);
}

// qk_norm_rope_bwd(x, gain, inv_freq, positions, B, layout, scale, eps, dy) -> (tuple of dx, tuple of dgain)
PyObject* qk_norm_rope_bwd(PyObject* const* a) {
  const Heads h(a);
  if (!PyTuple_Check(a[8]) || PyTuple_GET_SIZE(a[8]) != h.n) value_error("dy and x differ in number");
  const Here here(h.x[0]->device());
  dflare_qk_grad tab[2] = {};
  at::Tensor dx[2], dgain[2];
  for (int k = 0; k < h.n; ++k) {
    const at::Tensor &x = *h.x[k], &dy = h.beside(PyTuple_GET_ITEM(a[8], k), k, "dy");
    dx[k] = fresh(x.sizes(), x, x.scalar_type());
    if (h.gain[k]) dgain[k] = fresh({h.hd}, x, at::kFloat);
    tab[k] = {x.data_ptr(), dy.data_ptr(), dx[k].data_ptr(), h.gain[k], (float*)address(dgain[k]), x.stride(0), x.stride(1),
              dy.stride(0), dy.stride(1), dx[k].stride(0), dx[k].stride(1), (int32_t)x.size(1)};
  }
  const size_t bytes = p_qk_norm_rope_bwd_workspace(h.rows, h.hd, h.n);
  const at::Tensor ws = fresh({(int64_t)std::max<size_t>(bytes, 16)}, *h.x[0], at::kByte);
  const int rc = unlocked([&] {
    return p_qk_norm_rope_bwd(tab, h.n, (const int32_t*)h.positions, (const double*)h.freq, h.rows, h.B, h.hd, h.rot, h.dtype, h.layout,
                              (float)h.scale, (float)h.eps, ws.data_ptr(), bytes, here.stream);
  });
  if (rc != DFLARE_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("NN", pair_of(dx, h.n), pair_of(dgain, h.n));
}

// rows and weights of a projection: x [rows, K] and w [N, K], both bf16
struct Projection {
  const at::Tensor &x, &w;
  int32_t rows, N, K;
  Projection(PyObject* px, PyObject* pw, const char* name) : x(dense(px)), w(dense(pw)) {
    if (x.dim() != 2 || w.dim() != 2) value_error("expected bf16 tensors x [rows, K] and weights [N, K]");
    if (type_code(x) != DFLARE_BF16) type_error("expected bf16 tensors");
    rows = to32(x.size(0), "rows");
    K = to32(x.size(1), "K");
    N = to32(w.size(0), "N");
    like(pw, name, {N, K}, x);
  }
};
at::Tensor scratch(size_t bytes, const at::Tensor& ref) { return fresh({(int64_t)std::max<size_t>(bytes, 16)}, ref, at::kByte); }
int truth(PyObject* o) {
  const int r = PyObject_IsTrue(o);
  if (r < 0) throw Refused{nullptr, ""};
  return r;
}

// linear_fwd(x, w, bias, residual, act, save) -> (y, z)
PyObject* linear_fwd(PyObject* const* a) {
  const Projection p(a[0], a[1], "w");
  void *bias = like(a[2], "bias", {p.N}, p.x), *res = like(a[3], "residual", {p.rows, p.N}, p.x);
  const int32_t act = to32(PyLong_AsLongLong(a[4]), "act");
  if (PyErr_Occurred()) return nullptr;
  const bool save = truth(a[5]);
  const Here here(p.x.device());
  dflare_product_plan plan{};  // (of sizes that are refused below: 0 bytes)
  p_linear_plan(p.rows, p.N, p.K, act, 0, 0, 0, &plan, nullptr);
  const size_t bytes = plan.workspace;
  const at::Tensor ws = scratch(bytes, p.x), y = fresh({p.rows, p.N}, p.x, p.x.scalar_type());
  const at::Tensor z = save ? fresh({p.rows, p.N}, p.x, p.x.scalar_type()) : at::Tensor();
  const int rc = unlocked([&] {
    return p_linear_fwd(p.x.data_ptr(), p.w.data_ptr(), bias, res, p.rows, p.N, p.K, act, y.data_ptr(), address(z), ws.data_ptr(), bytes,
                        here.stream);
  });
  return rc != DFLARE_OK ? PyLong_FromLong(rc) : Py_BuildValue("NN", wrapped(y), wrapped(z));
}

// linear_bwd(dy, x, w, z, act, need_dx, need_dw, need_dbias) -> (dx, dw, dbias)
PyObject* linear_bwd(PyObject* const* a) {
  const Projection p(a[1], a[2], "w");
  void *dy = like(a[0], "dy", {p.rows, p.N}, p.x), *z = like(a[3], "z", {p.rows, p.N}, p.x);
  const int32_t act = to32(PyLong_AsLongLong(a[4]), "act");
  if (PyErr_Occurred()) return nullptr;
  tensor(a[0]);
  const int need_dx = truth(a[5]), need_dw = truth(a[6]), need_dbias = truth(a[7]);
  const Here here(p.x.device());
  dflare_product_plan plan{};
  p_linear_plan(p.rows, p.N, p.K, act, need_dx, need_dw, need_dbias, nullptr, &plan);
  const size_t bytes = plan.workspace;
  const auto type = p.x.scalar_type();
  const at::Tensor ws = scratch(bytes, p.x), dx = need_dx ? fresh(p.x.sizes(), p.x, type) : at::Tensor();
  const at::Tensor dw = need_dw ? fresh(p.w.sizes(), p.x, type) : at::Tensor(), dbias = need_dbias ? fresh({p.N}, p.x, type) : at::Tensor();
  const int rc = unlocked([&] {
    return p_linear_bwd(dy, p.x.data_ptr(), p.w.data_ptr(), z, p.rows, p.N, p.K, act, address(dx), address(dw), address(dbias), ws.data_ptr(),
                        bytes, here.stream);
  });
  return rc != DFLARE_OK ? PyLong_FromLong(rc) : Py_BuildValue("NNN", wrapped(dx), wrapped(dw), wrapped(dbias));
}

// gated_fwd(x, w_gate, w_up, act, save) -> (h, gate, up)
PyObject* gated_fwd(PyObject* const* a) {
  const Projection p(a[0], a[1], "w_gate");
  void* up_w = dense(a[2]).data_ptr();
  like(a[2], "w_up", p.w.sizes(), p.x);
  const int32_t act = to32(PyLong_AsLongLong(a[3]), "act");
  if (PyErr_Occurred()) return nullptr;
  const bool save = truth(a[4]);
  const Here here(p.x.device());
  dflare_product_plan plan{};
  p_gated_plan(p.rows, p.K, p.N, 0, 0, &plan, nullptr);
  const size_t bytes = plan.workspace;
  auto rows_of = [&] { return fresh({p.rows, p.N}, p.x, p.x.scalar_type()); };
  const at::Tensor ws = scratch(bytes, p.x), h = rows_of(), gate = save ? rows_of() : at::Tensor(), up = save ? rows_of() : at::Tensor();
  const int rc = unlocked([&] {
    return p_gated_fwd(p.x.data_ptr(), p.w.data_ptr(), up_w, p.rows, p.K, p.N, act, h.data_ptr(), address(gate), address(up), ws.data_ptr(), bytes,
                       here.stream);
  });
  return rc != DFLARE_OK ? PyLong_FromLong(rc) : Py_BuildValue("NNN", wrapped(h), wrapped(gate), wrapped(up));
}

// gated_bwd(dh, x, gate, up, w_gate, w_up, act, need_dx, need_dw) -> (dx, dw_gate, dw_up)
PyObject* gated_bwd(PyObject* const* a) {
  const Projection p(a[1], a[4], "w_gate");
  void *dh = like(a[0], "dh", {p.rows, p.N}, p.x), *gate = like(a[2], "gate", {p.rows, p.N}, p.x), *up = like(a[3], "up", {p.rows, p.N}, p.x);
  void* up_w = like(a[5], "w_up", p.w.sizes(), p.x);
  const int32_t act = to32(PyLong_AsLongLong(a[6]), "act");
  if (PyErr_Occurred()) return nullptr;
  for (int k : {0, 2, 3, 5}) tensor(a[k]);
  const int need_dx = truth(a[7]), need_dw = truth(a[8]);
  const Here here(p.x.device());
  dflare_product_plan plan{};
  p_gated_plan(p.rows, p.K, p.N, need_dx, need_dw, nullptr, &plan);
  const size_t bytes = plan.workspace;
  const auto type = p.x.scalar_type();
  auto weights = [&] { return need_dw ? fresh(p.w.sizes(), p.x, type) : at::Tensor(); };
  const at::Tensor ws = scratch(bytes, p.x), dx = need_dx ? fresh(p.x.sizes(), p.x, type) : at::Tensor(), dg = weights(), du = weights();
  const int rc = unlocked([&] {
    return p_gated_bwd(dh, p.x.data_ptr(), gate, up, p.w.data_ptr(), up_w, p.rows, p.K, p.N, act, address(dx), address(dg), address(du),
                       ws.data_ptr(), bytes, here.stream);
  });
  return rc != DFLARE_OK ? PyLong_FromLong(rc) : Py_BuildValue("NNN", wrapped(dx), wrapped(dg), wrapped(du));
}

// adamw(params, grads, m, v, masters, m_scales, v_scales, step, lr, beta1, beta2, eps, weight_decay, sumsq, max_norm) -> status;
// lists of tensors; masters and scales: lists, in which tensors may be None, or None; step and lr: numbers, or tensors of one
PyObject* adamw(PyObject* const* a) {
  for (int k = 0; k < 7; ++k)
    if (!PyList_Check(a[k]) && (k < 4 || a[k] != Py_None)) type_error("expected a list");
  const Py_ssize_t n = PyList_GET_SIZE(a[0]);
  if (n < 1) value_error("expected at least one parameter");
  to32(n, "the number of parameters");
  for (int k = 1; k < 7; ++k)
    if (a[k] != Py_None && PyList_GET_SIZE(a[k]) != n) value_error("the lists differ in length");
  const at::Tensor& first = dense(PyList_GET_ITEM(a[0], 0));
  std::vector<dflare_adamw_tensor> table(n);
  const at::ScalarType state = tensor(PyList_GET_ITEM(a[2], 0)).scalar_type();
  if (state != at::kFloat && state != at::kFloat8_e4m3fn) type_error("the moments are fp32 or float8_e4m3fn tensors");
  const bool byte = state == at::kFloat8_e4m3fn;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor &p = dense(PyList_GET_ITEM(a[0], i)), &g = dense(PyList_GET_ITEM(a[1], i));
    if (p.device() != first.device() || g.device() != first.device()) value_error("the tensors are on different devices");
    if (g.sizes() != p.sizes()) value_error("a gradient has another shape than its parameter");
    auto item = [&](int k) { return a[k] == Py_None ? Py_None : PyList_GET_ITEM(a[k], i); };
    auto moment = [&](int k, const char* name) {
      const at::Tensor& t = dense(item(k));
      if (t.sizes() != p.sizes()) value_error(std::string(name) + " has another shape than its parameter");
      if (t.device() != p.device() || t.scalar_type() != state) type_error("the moments differ in type or device");
      return t.data_ptr();
    };
    dflare_adamw_tensor& t = table[i];
    t = {p.data_ptr(), g.data_ptr(), nullptr, moment(2, "m"), moment(3, "v"), nullptr, nullptr, p.numel(), type_code(p), type_code(g)};
    t.master = (float*)like(item(4), "master", p.sizes(), p, at::kFloat);
    const int64_t scales = (p.numel() + 255) / 256;
    if (byte) {
      t.m_scale = (float*)like(item(5), "m_scale", {scales}, p, at::kFloat);
      t.v_scale = (float*)like(item(6), "v_scale", {scales}, p, at::kFloat);
    } else if (item(5) != Py_None || item(6) != Py_None) {
      value_error("scales beside fp32 moments");
    }
  }
  dflare_adamw_options o{};
  const bool step_there = THPVariable_Check(a[7]), lr_there = THPVariable_Check(a[8]);
  if (step_there) o.step_device = (const int64_t*)like(a[7], "step", {1}, first, at::kLong);
  if (lr_there) o.lr_device = (const double*)like(a[8], "lr", {1}, first, at::kDouble);
  if (!step_there) o.step = PyLong_AsLongLong(a[7]);
  if (!PyErr_Occurred() && !lr_there) o.lr = PyFloat_AsDouble(a[8]);
  if (PyErr_Occurred()) return nullptr;
  o.beta1 = PyFloat_AsDouble(a[9]);
  o.beta2 = PyFloat_AsDouble(a[10]);
  o.eps = PyFloat_AsDouble(a[11]);
  o.weight_decay = PyFloat_AsDouble(a[12]);
  const double max_norm = PyFloat_AsDouble(a[14]);
  if (PyErr_Occurred()) return nullptr;
  o.sumsq = (const double*)like(a[13], "sumsq", {1}, first, at::kDouble);
  o.max_norm = (float)max_norm;
  o.state_bits = byte ? 8 : 32;
  const Here here(first.device());
  return PyLong_FromLong(unlocked([&] { return p_adamw(table.data(), (int32_t)n, &o, here.stream); }));
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
    if (!r.type) return nullptr;  // (Python's own error stands)
    PyErr_Clear();
    PyErr_SetString(r.type, r.why.c_str());
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(p_out_of_memory, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

constexpr int kBound = 19;
// bind(addresses of the entry points in the order below, function from a device index to its current stream's address,
// torch's out-of-memory exception)
PyObject* bind(PyObject* const* a) {
  void** to[] = {(void**)&p_norm_fwd, (void**)&p_norm_bwd_workspace, (void**)&p_norm_bwd, (void**)&p_rope,
                 (void**)&p_grad_norm_workspace, (void**)&p_grad_norm, (void**)&p_clip_grads,
                 (void**)&p_qk_norm_rope_fwd, (void**)&p_qk_norm_rope_bwd_workspace, (void**)&p_qk_norm_rope_bwd,
                 (void**)&p_linear_plan, (void**)&p_linear_fwd, (void**)&p_linear_bwd, (void**)&p_gated_plan, (void**)&p_gated_fwd,
                 (void**)&p_gated_bwd, (void**)&p_adamw};
  constexpr int n = sizeof(to) / sizeof(to[0]);
  static_assert(n + 2 == kBound);
  for (int k = 0; k < n; ++k) *to[k] = PyLong_AsVoidPtr(a[k]);
  if (PyErr_Occurred()) return nullptr;
  p_raw_stream = Py_NewRef(a[n]);
  p_out_of_memory = Py_NewRef(a[n + 1]);
  return Py_NewRef(Py_None);
}

#define FUNCTION(f, n) {#f, (PyCFunction)(void*)guarded<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FUNCTION(bind, kBound), FUNCTION(norm_fwd, 6), FUNCTION(norm_bwd, 7), FUNCTION(rope, 8), FUNCTION(grad_norm, 1),
                         FUNCTION(clip_grads, 4), FUNCTION(qk_norm_rope_fwd, 9), FUNCTION(qk_norm_rope_bwd, 9), FUNCTION(linear_fwd, 6),
                         FUNCTION(linear_bwd, 8), FUNCTION(gated_fwd, 5), FUNCTION(gated_bwd, 9), FUNCTION(adamw, 15), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
