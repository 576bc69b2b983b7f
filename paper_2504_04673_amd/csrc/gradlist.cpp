// A list of gradient tensors as struct sagnn_grad of the C header: address, address of the result, values, type.  Asked for one by
// one from Python these are ten questions a tensor at 70 ns each: 211 tensors 170 us, this way 4, of 41 for their clipping.
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>

// The torch that this is compiled against, found in the file before it is loaded: another one's tensors may lie otherwise.
extern "C" __attribute__((used)) const char sagnn_gradlist_torch[] = "sagnn_gradlist_torch=" SAGNN_TORCH;

namespace {

struct Row { int64_t in, out, n, dtype; };

bool usable(const at::Tensor& t) {
  return t.defined() && t.is_cuda() && t.layout() == c10::kStrided && (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16) &&
         t.is_contiguous();
}

// rows(gradients, results or None) -> bytes
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 2) return PyErr_Format(PyExc_TypeError, "rows(gradients, results): %zd arguments", n_args);
  PyObject *in = PySequence_Fast(args[0], "gradients: a sequence of tensors expected"), *out = nullptr, *bytes = nullptr;
  if (!in) return nullptr;
  if (args[1] != Py_None && !(out = PySequence_Fast(args[1], "out: a sequence of tensors expected"))) {
    Py_DECREF(in);
    return nullptr;
  }
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(in);
  const char* wrong = nullptr;
  if (out && PySequence_Fast_GET_SIZE(out) != n) wrong = "out: expected as many tensors as there are gradients";
  else bytes = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(Row));
  if (bytes) {
    char* to = PyBytes_AS_STRING(bytes);
    try {
      for (Py_ssize_t i = 0; i < n && !wrong; ++i) {
        PyObject *a = PySequence_Fast_GET_ITEM(in, i), *b = out ? PySequence_Fast_GET_ITEM(out, i) : a;
        if (!THPVariable_Check(a) || !THPVariable_Check(b)) {
          wrong = "gradients and out: tensors expected";
          break;
        }
        const at::Tensor &g = THPVariable_Unpack(a), &o = THPVariable_Unpack(b);
        if (!usable(g)) wrong = "gradients: expected contiguous float32 or bfloat16 CUDA/HIP tensors (there is no CPU path)";
        else if (a != b && (!usable(o) || o.scalar_type() != g.scalar_type() || o.sizes() != g.sizes()))
          wrong = "out: expected contiguous tensors like the gradients";
        if (wrong) break;
        const Row r = {(int64_t)(uintptr_t)g.data_ptr(), (int64_t)(uintptr_t)o.data_ptr(), g.numel(), g.scalar_type() == at::kBFloat16 ? 1 : 0};
        memcpy(to + i * sizeof(Row), &r, sizeof(Row));
      }
    } catch (const std::exception&) {
      wrong = "gradients and out: a tensor without memory";
    }
  }
  Py_DECREF(in);
  Py_XDECREF(out);
  if (wrong) {
    Py_XDECREF(bytes);
    PyErr_SetString(PyExc_ValueError, wrong);
    return nullptr;
  }
  return bytes;
}

PyMethodDef methods[] = {{"rows", (PyCFunction)(void (*)(void))rows, METH_FASTCALL, "rows(gradients, results or None) -> struct sagnn_grad of each, as bytes"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gradlist", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gradlist(void) { return PyModule_Create(&module); }
