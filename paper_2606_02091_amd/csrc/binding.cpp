// Native part of the Python binding: the table of a list of gradient tensors (dflare_grad_tensor of
// include/dflare.h).  A list of hundreds of tensors costs 0.1 ms and more when Python asks each tensor for
// its address, size, type, device and layout, more than the kernels that read the table take; here a few microseconds.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "dflare.h"

namespace {

// what is wrong with o as an entry, or null; otherwise its tensor and type
const char* entry(PyObject* o, const at::Tensor** tensor, int* dtype, PyObject** type) {
  *type = PyExc_TypeError;
  if (!THPVariable_Check(o)) return "expected a device tensor";
  const at::Tensor& t = THPVariable_Unpack(o);
  const auto s = t.scalar_type();
  if (s == at::kFloat) *dtype = DFLARE_F32;
  else if (s == at::kBFloat16 || s == at::kShort || s == at::kUInt16) *dtype = DFLARE_BF16;  // 16-bit integers: bf16 bits
  else return "expected bf16 or fp32 tensors";
  if (!t.is_cuda()) return "expected a device tensor";
  *type = PyExc_ValueError;
  *tensor = &t;
  return t.is_contiguous() ? nullptr : "tensor must be contiguous";
}

PyObject* refuse(PyObject* type, const char* why) {
  PyErr_SetString(type, why);
  return nullptr;
}

// grad_table(grads, outs or None) -> (bytes: the table, index of the tensors' device)
PyObject* grad_table(PyObject*, PyObject* args) {
  PyObject *grads, *outs;
  if (!PyArg_ParseTuple(args, "O!O", &PyList_Type, &grads, &outs)) return nullptr;
  const Py_ssize_t n = PyList_GET_SIZE(grads);
  if (outs != Py_None && !PyList_Check(outs)) return refuse(PyExc_TypeError, "expected a list");
  if (outs != Py_None && PyList_GET_SIZE(outs) != n) return refuse(PyExc_ValueError, "out and grads differ in number");
  PyObject* table = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(dflare_grad_tensor));
  if (!table) return nullptr;
  auto* e = reinterpret_cast<dflare_grad_tensor*>(PyBytes_AS_STRING(table));
  int device = -1;
  const char* why = nullptr;
  PyObject* type = PyExc_ValueError;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor *t, *o;
    int dtype = 0, odtype = 0;
    if ((why = entry(PyList_GET_ITEM(grads, i), &t, &dtype, &type))) break;
    if (device < 0) device = t->get_device();
    if (t->get_device() != device) {
      why = "the gradients are on different devices";
      break;
    }
    e[i] = {t->data_ptr(), nullptr, t->numel(), dtype};
    if (outs == Py_None) continue;
    if ((why = entry(PyList_GET_ITEM(outs, i), &o, &odtype, &type))) break;
    if (odtype != dtype || o->get_device() != device || o->sizes() != t->sizes()) {
      why = "out and grads differ in shape, type or device";
      break;
    }
    e[i].out = o->data_ptr();
  }
  if (why) {
    Py_DECREF(table);
    return refuse(type, why);
  }
  return Py_BuildValue("Ni", table, device);
}

PyObject* guarded(PyObject* self, PyObject* args) {
  try {
    return grad_table(self, args);
  } catch (const std::exception& x) {
    return refuse(PyExc_RuntimeError, x.what());
  }
}

PyMethodDef methods[] = {{"grad_table", guarded, METH_VARARGS, "table of gradient tensors"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
