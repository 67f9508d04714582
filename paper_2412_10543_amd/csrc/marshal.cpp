// Checks a call's tensors and takes their addresses, for binding.py: what the
// Python attributes of ten tensors cost is as much as a kernel launch.
//
//   pointers(spec, t0, t1, ...)  spec: for each tensor its type ('i' int32, 'l'
//     int64, 'b' bf16, 'f' float32; a capital: None is allowed, a null address) and
//     its rank as a digit.  'u' is uint8.  'r' (bf16), 'g' (float32) and 'h' (either) are
//     rows: contiguous but for the step from one to the next, which is at least a row
//     and follows the sizes (for 'h' also whether it is float32).  Every tensor is
//     otherwise contiguous, and on one GPU, the current one.  Returns (device, address of t0, its
//     sizes, address of t1, ...; zeros for None), or, as an int, the number of the first
//     tensor that is none of that (their count: on another device than the current one).
#define PY_SSIZE_T_CLEAN
#include <c10/hip/HIPFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool is_rows(char type) { return type == 'r' || type == 'g' || type == 'h'; }

bool fits(const at::Tensor& t, char type, char rank) {
  const at::ScalarType want = type == 'i'                  ? at::kInt
                              : type == 'l'                ? at::kLong
                              : type == 'u'                ? at::kByte
                              : type == 'b' || type == 'r' ? at::kBFloat16
                                                           : at::kFloat;
  if (!t.is_cuda() || t.dim() != rank - '0' ||
      (t.scalar_type() != want && !(type == 'h' && t.scalar_type() == at::kBFloat16)))
    return false;
  if (!is_rows(type)) return t.is_contiguous();
  int64_t width = 1;
  for (int64_t i = t.dim() - 1; i > 0; --i) {
    if (t.size(i) != 1 && t.stride(i) != width) return false;
    width *= t.size(i);
  }
  return t.size(0) <= 1 || t.stride(0) >= width;
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
      const char type = spec[2 * i] | 0x20;
      values += 1 + (spec[2 * i + 1] - '0') + is_rows(type) + (type == 'h');
      if (x == Py_None && (spec[2 * i] & 0x20) == 0) continue;
      if (!THPVariable_Check(x)) return PyLong_FromSsize_t(i);
      const at::Tensor& t = THPVariable_Unpack(x);
      if (!fits(t, type, spec[2 * i + 1]) || (device >= 0 && device != t.get_device()))
        return PyLong_FromSsize_t(i);
      device = static_cast<int>(t.get_device());
    }
    if (device < 0 || c10::hip::current_device() != device) return PyLong_FromSsize_t(n);
    PyObject* out = PyTuple_New(values);
    if (out == nullptr) return nullptr;
    Py_ssize_t at = 0;
    PyTuple_SET_ITEM(out, at++, PyLong_FromLong(device));
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* x = args[i + 1];
      const char type = spec[2 * i] | 0x20;
      if (x == Py_None) {
        for (int n = 1 + (spec[2 * i + 1] - '0') + is_rows(type) + (type == 'h'); n > 0; --n)
          PyTuple_SET_ITEM(out, at++, PyLong_FromLong(0));
        continue;
      }
      const at::Tensor& t = THPVariable_Unpack(x);
      PyTuple_SET_ITEM(out, at++, PyLong_FromVoidPtr(t.data_ptr()));
      for (const auto size : t.sizes()) PyTuple_SET_ITEM(out, at++, PyLong_FromLongLong(size));
      if (is_rows(type)) PyTuple_SET_ITEM(out, at++, PyLong_FromLongLong(t.stride(0)));
      if (type == 'h')
        PyTuple_SET_ITEM(out, at++, PyLong_FromLong(t.scalar_type() == at::kFloat));
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
