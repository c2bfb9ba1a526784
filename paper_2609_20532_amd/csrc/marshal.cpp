// Checks and addresses of lists of tensors for the Python binding, read from the
// tensors themselves: a step over many small tensors is bound by these, and one check
// of one tensor from Python takes as long as the whole list here.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

// addresses(tensors, sizes, element, device, to): whether every tensor of the list is
// a contiguous CUDA tensor on `device` with sizes[k] entries and the type code
// `element`; their addresses are written to the buffer `to` (8 bytes each).
PyObject* addresses(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 5) {
    PyErr_SetString(PyExc_TypeError, "addresses(tensors, sizes, element, device, to)");
    return nullptr;
  }
  PyObject* tensors = PySequence_Fast(args[0], "tensors must be a list");
  if (!tensors) return nullptr;
  PyObject* sizes = PySequence_Fast(args[1], "sizes must be a list");
  if (!sizes) {
    Py_DECREF(tensors);
    return nullptr;
  }
  PyObject* answer = nullptr;
  Py_buffer to{};
  const long element = PyLong_AsLong(args[2]), device = PyLong_AsLong(args[3]);
  if (!PyErr_Occurred() && PyObject_GetBuffer(args[4], &to, PyBUF_WRITABLE) == 0) {
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(tensors);
    bool good = n == PySequence_Fast_GET_SIZE(sizes) && n * 8 <= to.len;
    for (Py_ssize_t k = 0; good && k < n; ++k) {
      PyObject* t = PySequence_Fast_GET_ITEM(tensors, k);
      const long long size = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(sizes, k));
      good = THPVariable_Check(t) && !PyErr_Occurred();
      if (!good) break;
      const at::Tensor& v = THPVariable_Unpack(t);
      good = v.is_cuda() && v.get_device() == device && static_cast<long>(v.scalar_type()) == element &&
             v.layout() == at::kStrided && v.is_contiguous() && v.numel() == size;
      if (good) static_cast<uint64_t*>(to.buf)[k] = reinterpret_cast<uint64_t>(v.data_ptr());
    }
    PyBuffer_Release(&to);
    if (!PyErr_Occurred()) answer = PyBool_FromLong(good);
  }
  Py_DECREF(tensors);
  Py_DECREF(sizes);
  return answer;
}

PyMethodDef methods[] = {
    {"addresses", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(addresses)), METH_FASTCALL,
     "Checks a list of tensors and writes their addresses."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
