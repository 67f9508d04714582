// Checks a call's tensors and takes their addresses, for binding.py: what the
// Python attributes of ten tensors cost is as much as a kernel launch.
//
//   pointers(spec, t0, t1, ...)  spec: for each tensor its type ('i' int32, 'l'
//     int64, 'b' bf16, 'f' float32; a capital: None is allowed, a null address) and
//     its rank as a digit.  Every tensor is contiguous and on one GPU, the current
//     one.  Returns (device, address of t0, its sizes, address of t1, ...; for None
//     only a 0), or, as an int, the number of the first tensor that is none of that
//     (their count: on another device than the current one).
#define PY_SSIZE_T_CLEAN
#include <c10/hip/HIPFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool fits(const at::Tensor& t, char type, char rank) {
  type |= 0x20;
  const at::ScalarType want = type == 'i'   ? at::kInt
                              : type == 'l' ? at::kLong
                              : type == 'b' ? at::kBFloat16
                                            : at::kFloat;
  return t.is_cuda() && t.scalar_type() == want && t.dim() == rank - '0' && t.is_contiguous();
}

PyObject* pointers(PyObject*, PyObject* const* args, Py_ssize_t count) {
  const Py_ssize_t n = count - 1;
  if (n < 0 || !PyBytes_Check(args[0]) || PyBytes_GET_SIZE(args[0]) != 2 * n) {
    PyErr_SetString(PyExc_TypeError, "pointers: a spec of two characters for each tensor");
    return nullptr;
  }
  const char* spec = PyBytes_AS_STRING(args[0]);
  try {
    int device = -1;
    Py_ssize_t values = 1;
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* x = args[i + 1];
      if (x == Py_None && (spec[2 * i] & 0x20) == 0) {
        ++values;
        continue;
      }
      if (!THPVariable_Check(x)) return PyLong_FromSsize_t(i);
      const at::Tensor& t = THPVariable_Unpack(x);
      if (!fits(t, spec[2 * i], spec[2 * i + 1]) || (device >= 0 && device != t.get_device()))
        return PyLong_FromSsize_t(i);
      device = static_cast<int>(t.get_device());
      values += 1 + t.dim();
    }
    if (device < 0 || c10::hip::current_device() != device) return PyLong_FromSsize_t(n);
    PyObject* out = PyTuple_New(values);
    if (out == nullptr) return nullptr;
    Py_ssize_t at = 0;
    PyTuple_SET_ITEM(out, at++, PyLong_FromLong(device));
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* x = args[i + 1];
      if (x == Py_None) {
        PyTuple_SET_ITEM(out, at++, PyLong_FromLong(0));
        continue;
      }
      const at::Tensor& t = THPVariable_Unpack(x);
      PyTuple_SET_ITEM(out, at++, PyLong_FromVoidPtr(t.data_ptr()));
      for (const auto size : t.sizes()) PyTuple_SET_ITEM(out, at++, PyLong_FromLongLong(size));
    }
    return out;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {
    {"pointers", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(pointers)), METH_FASTCALL,
     "pointers(spec, *tensors)"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
