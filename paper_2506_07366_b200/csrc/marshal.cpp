// Python module _marshal: checks a call's tensors and passes their addresses to an entry point of libmoegps.
//
// What binding.py does in Python with about half a microsecond for each tensor (type, shape, layout, address), for calls
// whose kernels take a few microseconds.  No arithmetic and no CUDA work of its own: a Call holds the address of a C entry
// point (include/moegps.h), the context and what each tensor has to be; calling it with (stream, tensors...) returns the
// entry point's code.  A tensor that is not what it has to be is handed to the Python check, which raises.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstddef>
#include <exception>
#include <memory>
#include <utility>
#include <vector>

namespace {

constexpr size_t kMaxTensors = 24;

struct Spec {
  at::ScalarType dtype;
  std::vector<int64_t> sizes;
  bool any_shape, optional;
};

struct Call {
  PyObject_HEAD
  vectorcallfunc vectorcall;
  void* entry;
  void* context;
  std::vector<Spec>* specs;
  PyObject* check;        // Python: check(tensor, *arguments[i]) returns or raises
  PyObject* arguments;
};

// entry(context, p[0], ..., p[N-1], stream)
template <size_t... I>
int invoke(void* entry, void* context, void* const* p, void* stream, std::index_sequence<I...>) {
  using Fn = int (*)(void*, decltype((void)I, (void*)nullptr)..., void*);
  return reinterpret_cast<Fn>(entry)(context, p[I]..., stream);
}
template <size_t N>
int invoke_n(void* entry, void* context, void* const* p, void* stream) {
  return invoke(entry, context, p, stream, std::make_index_sequence<N>());
}
using Invoker = int (*)(void*, void*, void* const*, void*);
template <size_t... N>
Invoker invoker(size_t n, std::index_sequence<N...>) {
  static constexpr Invoker table[] = {&invoke_n<N>...};
  return table[n];
}

bool matches(const Spec& s, PyObject* o, void** out) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != s.dtype || !t.is_contiguous()) return false;
  if (!s.any_shape && t.sizes() != c10::IntArrayRef(s.sizes)) return false;
  *out = t.data_ptr();
  return true;
}

// A stream argument as binding.py takes it: None (the current stream), a stream object or whatever int() makes a handle of.
bool stream_of(PyObject* o, void** out) {
  if (o == Py_None) {
    *out = c10::cuda::getCurrentCUDAStream().stream();
    return true;
  }
  PyObject* held = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, "cuda_stream");
  if (!held && PyErr_ExceptionMatches(PyExc_AttributeError)) {
    PyErr_Clear();
    held = Py_NewRef(o);
  }
  PyObject* handle = held ? PyNumber_Long(held) : nullptr;
  Py_XDECREF(held);
  if (!handle) {
    if (PyErr_ExceptionMatches(PyExc_TypeError))
      PyErr_Format(PyExc_AttributeError, "%R is neither a stream nor a stream's handle", o);
    return false;
  }
  *out = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  return !PyErr_Occurred();
}

PyObject* call(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* kwnames) {
  Call* c = reinterpret_cast<Call*>(self);
  const size_t n = c->specs->size();
  if ((size_t)PyVectorcall_NARGS(nargsf) != n + 1 || (kwnames && PyTuple_GET_SIZE(kwnames))) {
    PyErr_Format(PyExc_TypeError, "expected a stream and %zu tensors", n);
    return nullptr;
  }
  void *p[kMaxTensors] = {}, *stream = nullptr;
  try {
    for (size_t i = 0; i < n; ++i) {
      const Spec& s = (*c->specs)[i];
      PyObject* o = args[i + 1];
      if (o == Py_None && s.optional) continue;
      if (matches(s, o, &p[i])) continue;
      PyObject* rest = PyTuple_GET_ITEM(c->arguments, i);
      PyObject* one = PyTuple_Pack(1, o);
      PyObject* all = one ? PySequence_Concat(one, rest) : nullptr;
      Py_XDECREF(one);
      PyObject* r = all ? PyObject_Call(c->check, all, nullptr) : nullptr;
      Py_XDECREF(all);
      if (r) {
        Py_DECREF(r);
        PyErr_Format(PyExc_TypeError, "argument %zu was refused", i);
      }
      return nullptr;
    }
    if (!stream_of(args[0], &stream)) return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = invoker(n, std::make_index_sequence<kMaxTensors + 1>())(c->entry, c->context, p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// Call(entry address, context address, check, ((dtype, sizes or None, name, optional), ...))
PyObject* call_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long entry, context;
  PyObject *check, *arguments;
  if (!PyArg_ParseTuple(args, "KKOO!", &entry, &context, &check, &PyTuple_Type, &arguments)) return nullptr;
  auto specs = std::make_unique<std::vector<Spec>>();
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(arguments); ++i) {
    PyObject *dtype, *sizes;
    const char* name;
    int optional;
    if (!PyArg_ParseTuple(PyTuple_GET_ITEM(arguments, i), "OOsp", &dtype, &sizes, &name, &optional)) return nullptr;
    if (!THPDtype_Check(dtype)) {
      PyErr_SetString(PyExc_TypeError, "dtype expected");
      return nullptr;
    }
    Spec s{reinterpret_cast<THPDtype*>(dtype)->scalar_type, {}, sizes == Py_None, optional != 0};
    if (!s.any_shape) {
      PyObject* seq = PySequence_Fast(sizes, "sizes");
      if (!seq) return nullptr;
      for (Py_ssize_t k = 0; k < PySequence_Fast_GET_SIZE(seq); ++k)
        s.sizes.push_back(PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq, k)));
      Py_DECREF(seq);
      if (PyErr_Occurred()) return nullptr;
    }
    specs->push_back(std::move(s));
  }
  if (specs->size() > kMaxTensors) {
    PyErr_SetString(PyExc_ValueError, "too many tensors");
    return nullptr;
  }
  Call* c = reinterpret_cast<Call*>(type->tp_alloc(type, 0));
  if (!c) return nullptr;
  c->vectorcall = call;
  c->entry = reinterpret_cast<void*>(entry);
  c->context = reinterpret_cast<void*>(context);
  c->specs = specs.release();
  c->check = Py_NewRef(check);
  c->arguments = Py_NewRef(arguments);
  return reinterpret_cast<PyObject*>(c);
}

void call_dealloc(PyObject* self) {
  Call* c = reinterpret_cast<Call*>(self);
  delete c->specs;
  Py_XDECREF(c->check);
  Py_XDECREF(c->arguments);
  Py_TYPE(self)->tp_free(self);
}

PyTypeObject call_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", "Argument checks of the training step's calls.", -1, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  call_type.tp_name = "_marshal.Call";
  call_type.tp_basicsize = sizeof(Call);
  call_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL;
  call_type.tp_vectorcall_offset = offsetof(Call, vectorcall);
  call_type.tp_call = PyVectorcall_Call;
  call_type.tp_new = call_new;
  call_type.tp_dealloc = call_dealloc;
  if (PyType_Ready(&call_type) < 0) return nullptr;
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  // (the module depends on the layout of torch's objects: build.py and binding.py compare this with the installed version)
  if (PyModule_AddObjectRef(m, "Call", reinterpret_cast<PyObject*>(&call_type)) < 0 ||
      PyModule_AddStringConstant(m, "built_for", MOEGPS_BUILT_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
