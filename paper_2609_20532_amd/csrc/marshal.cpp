// Checks and addresses of tensors for the Python binding, read from the tensors
// themselves: a call on small tensors is bound by these (0.7 us for a tensor that is
// checked from Python, a tenth of it here). Where a check fails, the binding finds out
// which one, and says so. What a tensor throws (one without storage, inside a function
// transform, has no address) becomes the Python exception that its own method raises.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>

#include "dpsgd.h"

namespace {

bool plain(const at::Tensor& v, long device) {
  return v.is_cuda() && v.get_device() == device && v.layout() == at::kStrided;
}

// The address of v, null for a tensor of no entries.
void* address_of(const at::Tensor& v) {
  void* p = v.data_ptr();
  TORCH_CHECK(p || v.numel() == 0, "the tensor has no memory");
  return p;
}

// f(); a C++ exception, which may not pass through the interpreter's frames, is set as
// the Python error that it stands for. Whether there was none.
template <class F>
bool guarded(F f) {
  try {
    f();
    return true;
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return false;
  }
}

// addresses(tensors, layers, per_block, element, device, to): whether every tensor of
// the list is a contiguous CUDA tensor on `device` with the type code `element` and, for
// layer k of the buffer `layers` (dpsgd_layer), d_out d_in entries, or with per_block 2
// for every 256 of them; their addresses are written to the buffer `to` (8 bytes each).
PyObject* addresses(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 6) {
    PyErr_SetString(PyExc_TypeError, "addresses(tensors, layers, per_block, element, device, to)");
    return nullptr;
  }
  PyObject* tensors = PySequence_Fast(args[0], "tensors must be a list");
  if (!tensors) return nullptr;
  PyObject* answer = nullptr;
  Py_buffer layers{}, to{};
  const long per_block = PyLong_AsLong(args[2]), element = PyLong_AsLong(args[3]),
             device = PyLong_AsLong(args[4]);
  if (!PyErr_Occurred() && PyObject_GetBuffer(args[1], &layers, PyBUF_SIMPLE) == 0) {
    if (PyObject_GetBuffer(args[5], &to, PyBUF_WRITABLE) == 0) {
      const Py_ssize_t n = PySequence_Fast_GET_SIZE(tensors);
      bool good = n * (Py_ssize_t)sizeof(dpsgd_layer) == layers.len && n * 8 <= to.len;
      const auto each = [&] {
        for (Py_ssize_t k = 0; good && k < n; ++k) {
          PyObject* t = PySequence_Fast_GET_ITEM(tensors, k);
          good = THPVariable_Check(t);
          if (!good) break;
          const dpsgd_layer& L = static_cast<const dpsgd_layer*>(layers.buf)[k];
          // Sizes that the library refuses are not multiplied here.
          const bool small = L.d_in >= 1 && L.d_out >= 1 && L.d_in < (INT64_C(1) << 31) && L.d_out < (INT64_C(1) << 31);
          const int64_t entries = small ? L.d_in * L.d_out : -1;
          const at::Tensor& v = THPVariable_Unpack(t);
          good = plain(v, device) && static_cast<long>(v.scalar_type()) == element && v.is_contiguous() &&
                 v.numel() == (per_block ? 2 * ((entries + DPSGD_STATE_BLOCK - 1) / DPSGD_STATE_BLOCK) : entries);
          if (good) static_cast<uint64_t*>(to.buf)[k] = reinterpret_cast<uint64_t>(address_of(v));
        }
      };
      const bool whole = guarded(each);
      PyBuffer_Release(&to);
      if (whole) answer = PyBool_FromLong(good);
    }
    PyBuffer_Release(&layers);
  }
  Py_DECREF(tensors);
  return answer;
}

// Whether v has the shape (a, b, ...), or, for (-1, B, C, n), n entries in rows of C
// with B first. -1: `shape` is no tuple of numbers.
int fits(const at::Tensor& v, PyObject* shape) {
  if (!PyTuple_Check(shape)) return -1;
  const Py_ssize_t n = PyTuple_GET_SIZE(shape);
  long long s[8];
  if (n > 8) return -1;
  for (Py_ssize_t k = 0; k < n; ++k) {
    s[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, k));
    if (s[k] == -1 && PyErr_Occurred()) return -1;
  }
  if (n == 4 && s[0] == -1)
    return v.dim() >= 2 && v.size(0) == s[1] && v.size(-1) == s[2] && v.numel() == s[3];
  if (v.dim() != n) return 0;
  for (Py_ssize_t k = 0; k < n; ++k)
    if (v.size(k) != s[k]) return 0;
  return 1;
}

// take(device, tensor, shape, element, tensor, shape, element, ...): the addresses of
// contiguous tensors of these shapes and type codes (None for None) in a tuple, or the
// number of the first that is none.
PyObject* take(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args % 3 != 1) {
    PyErr_SetString(PyExc_TypeError, "take(device, tensor, shape, element, ...)");
    return nullptr;
  }
  const long device = PyLong_AsLong(args[0]);
  if (device == -1 && PyErr_Occurred()) return nullptr;
  const Py_ssize_t n = n_args / 3;
  PyObject* got = PyTuple_New(n);
  if (!got) return nullptr;
  for (Py_ssize_t k = 0; k < n; ++k) {
    PyObject* t = args[1 + 3 * k];
    PyObject* address = Py_None;
    if (t == Py_None) {
      Py_INCREF(address);
    } else {
      const long element = PyLong_AsLong(args[3 + 3 * k]);
      int good = !PyErr_Occurred() && THPVariable_Check(t);
      address = nullptr;
      if (good) {
        guarded([&] {
          const at::Tensor& v = THPVariable_Unpack(t);
          good = plain(v, device) && static_cast<long>(v.scalar_type()) == element && v.is_contiguous();
          if (good) good = fits(v, args[2 + 3 * k]);
          if (good == 1) address = PyLong_FromVoidPtr(address_of(v));
        });
      }
      if (!address) {
        Py_DECREF(got);
        if (PyErr_Occurred()) return nullptr;
        return PyLong_FromSsize_t(k);
      }
    }
    PyTuple_SET_ITEM(got, k, address);
  }
  return got;
}

// logits(device, tensor): (address, B, T, V, entries from row to row, type code) of
// logits [B, T, V] whose rows are evenly spaced and whose entries are neighbours, or
// None.
PyObject* logits(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 2) {
    PyErr_SetString(PyExc_TypeError, "logits(device, tensor)");
    return nullptr;
  }
  const long device = PyLong_AsLong(args[0]);
  if (device == -1 && PyErr_Occurred()) return nullptr;
  if (!THPVariable_Check(args[1])) Py_RETURN_NONE;
  PyObject* answer = nullptr;
  guarded([&] {
    const at::Tensor& v = THPVariable_Unpack(args[1]);
    bool good = plain(v, device) && v.dim() == 3 && v.numel() != 0;
    if (good) {
      const int64_t B = v.size(0), T = v.size(1), V = v.size(2);
      const int64_t stride = T > 1 ? v.stride(1) : (B > 1 ? v.stride(0) : V);
      good = (V == 1 || v.stride(2) == 1) && stride >= V && (B == 1 || T == 1 || v.stride(0) == T * v.stride(1));
      if (good)
        answer = Py_BuildValue("NLLLLi", PyLong_FromVoidPtr(address_of(v)), (long long)B, (long long)T,
                               (long long)V, (long long)stride, static_cast<int>(v.scalar_type()));
    }
    if (!good) {
      Py_INCREF(Py_None);
      answer = Py_None;
    }
  });
  return answer;
}

PyMethodDef methods[] = {
    {"addresses", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(addresses)), METH_FASTCALL,
     "Checks a list of tensors and writes their addresses."},
    {"take", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(take)), METH_FASTCALL,
     "Checks tensors one by one and returns their addresses."},
    {"logits", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(logits)), METH_FASTCALL,
     "Checks logits and returns their address and layout."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
