// Checks of tensor arguments for binding.py, in the process of a Python call: a tensor's type, device, size and layout in one call each
// instead of five (a call of ams_attend with eight tensors spends half of the host's time on them otherwise).  No device code, no launches.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool number(PyObject* o, long long& x) {
  x = PyLong_AsLongLong(o);
  return !(x == -1 && PyErr_Occurred());
}

// f() of what is no plain tensor (a batch of nested ones, a tensor inside a transform, ...) may throw: false then, as where it says so itself.
template <typename F>
bool held(F f) {
  try {
    return f();
  } catch (...) {
    PyErr_Clear();
    return false;
  }
}

bool fits(PyObject* t, PyObject* dtype, long long gpu) {
  return THPVariable_Check(t) && THPDtype_Check(dtype) && THPVariable_Unpack(t).scalar_type() == reinterpret_cast<THPDtype*>(dtype)->scalar_type &&
         THPVariable_Unpack(t).layout() == at::kStrided && THPVariable_Unpack(t).get_device() == gpu;
}

// arg(t, dtype, numel, gpu, what): pointer of a contiguous tensor of at least numel elements on that GPU; None stays None.
PyObject* arg(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long numel, gpu;
  if (n != 5) return PyErr_Format(PyExc_TypeError, "arg: five arguments expected");
  if (a[0] == Py_None) Py_RETURN_NONE;
  if (!number(a[2], numel) || !number(a[3], gpu)) return nullptr;
  void* at = nullptr;
  const bool good = held([&] {
    if (!fits(a[0], a[1], gpu)) return false;
    const at::Tensor& t = THPVariable_Unpack(a[0]);
    if (t.is_nested() || t.numel() < numel || !t.is_contiguous()) return false;
    at = t.data_ptr();
    return at != nullptr || t.numel() == 0;
  });
  if (!good) return PyErr_Format(PyExc_ValueError, "%S: contiguous %S tensor of at least %lld elements on GPU %lld expected", a[4], a[1], numel, gpu);
  return PyLong_FromVoidPtr(at);
}

// token_rows(t, shape, dtype, gpu, what): (pointer, elements from token to token) of [layers, batch, new, heads, channels], shape a tuple of
// these: any slice of a projection's output along the heads.
PyObject* token_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long gpu, s[5];
  if (n != 5 || !PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 5) return PyErr_Format(PyExc_TypeError, "token_rows: five arguments, a shape of five expected");
  if (!number(a[3], gpu)) return nullptr;
  for (int i = 0; i < 5; ++i)
    if (!number(PyTuple_GET_ITEM(a[1], i), s[i])) return nullptr;
  void* at = nullptr;
  long long stride[5] = {0, 0, 0, 0, 0};
  const bool good = held([&] {
    if (!fits(a[0], a[2], gpu)) return false;
    const at::Tensor& t = THPVariable_Unpack(a[0]);
    if (t.is_nested() || t.dim() != 5) return false;
    for (int i = 0; i < 5; ++i) {
      if (t.size(i) != s[i]) return false;
      stride[i] = t.stride(i);
    }
    at = t.data_ptr();
    return stride[4] == 1 && (s[3] <= 1 || stride[3] == s[4]) && (at != nullptr || t.numel() == 0);
  });
  if (!good)
    return PyErr_Format(PyExc_ValueError, "%S: %S [%lld, %lld, %lld, %lld, %lld] (layers, batch, new, heads, channels) on GPU %lld with contiguous heads expected",
                        a[4], a[2], s[0], s[1], s[2], s[3], s[4], gpu);
  // one stride from token to token, over those of a sequence, the batch and the layers (extents of one have none)
  const long long step = s[2] > 1 ? stride[2] : s[1] > 1 ? stride[1] : s[0] > 1 ? stride[0] : s[3] * s[4];
  if ((s[1] > 1 && stride[1] != step * s[2]) || (s[0] > 1 && stride[0] != step * s[2] * s[1]))
    return PyErr_Format(PyExc_ValueError, "%S: one stride from token to token expected", a[4]);
  return Py_BuildValue("NL", PyLong_FromVoidPtr(at), step);
}

PyMethodDef methods[] = {{"arg", (PyCFunction)(void*)arg, METH_FASTCALL, nullptr},
                         {"token_rows", (PyCFunction)(void*)token_rows, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__args() { return PyModule_Create(&module); }
