// gpuos_binding.cpp -- what the functions on PyTorch tensors do for every call, as a CPython module against PyTorch's headers: a call's
// tensors as a key (everything about them but their addresses), and the launch of a descriptor with their addresses put in.
// From Python the key of eleven tensors takes 4 us and the addresses, the launch and the versions 4; here 0.6 and 3.9, of which the launch is 3.4.
#define PY_SSIZE_T_CLEAN
#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/gpuos.h"

namespace {

typedef int (*launch_t)(int32_t, const gpuos_cache_task*, void*, uint64_t, void*);

void put(std::string& to, int64_t v) { to.append(reinterpret_cast<const char*>(&v), sizeof v); }

// key(tensors): bytes; its first is 1 where gradients are recorded and one of the tensors requires one.
PyObject* key(PyObject*, PyObject* arg) {
  if (!PyTuple_Check(arg)) {
    PyErr_SetString(PyExc_TypeError, "a tuple of tensors");
    return nullptr;
  }
  try {
    std::string to(1, '\0');
    to.reserve(1024);
    bool grad = false;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(arg); ++i) {
      PyObject* o = PyTuple_GET_ITEM(arg, i);
      if (o == Py_None) {
        put(to, -1);
        continue;
      }
      if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_ValueError, "a tensor, not %s", Py_TYPE(o)->tp_name);
        return nullptr;
      }
      const at::Tensor& t = THPVariable_Unpack(o);
      if (t.layout() != at::kStrided) {
        PyErr_SetString(PyExc_ValueError, "a tensor without strides");
        return nullptr;
      }
      const c10::Device d = t.device();
      put(to, t.dim() | (int64_t)t.scalar_type() << 8 | (int64_t)(uint8_t)d.type() << 16 | (int64_t)(uint8_t)d.index() << 24 |
                  (int64_t)t.is_neg() << 32 | (int64_t)t.is_conj() << 33);
      const at::IntArrayRef sizes = t.sizes(), strides = t.strides();
      for (int64_t n : sizes) put(to, n);
      for (int64_t n : strides) put(to, n);
      grad = grad || t.requires_grad();
    }
    if (grad && c10::GradMode::is_enabled()) to[0] = 1;
    return PyBytes_FromStringAndSize(to.data(), (Py_ssize_t)to.size());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
    return nullptr;
  }
}

// launch(function, task, places, tensors, written, device, workspace, stream): the function's status.  task: a descriptor's bytes; places: for each of
// tensors the operand that it is, or -1; written: which of tensors are the caller's and have a new version behind the call.
PyObject* launch(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8 || !PyBytes_Check(a[1]) || PyBytes_GET_SIZE(a[1]) != (Py_ssize_t)sizeof(gpuos_cache_task) || !PyBytes_Check(a[2]) || !PyTuple_Check(a[3]) ||
      !PyBytes_Check(a[4]) || PyBytes_GET_SIZE(a[2]) != PyTuple_GET_SIZE(a[3])) {
    PyErr_SetString(PyExc_TypeError, "launch(function, task, places, tensors, written, device, workspace, stream)");
    return nullptr;
  }
  const launch_t function = reinterpret_cast<launch_t>(PyLong_AsVoidPtr(a[0]));
  const long device = PyLong_AsLong(a[5]);
  long long space = PyLong_AsLongLong(a[6]);
  void* stream = PyLong_AsVoidPtr(a[7]);
  if (PyErr_Occurred()) return nullptr;
  HANDLE_TH_ERRORS                                              // (out of memory, and what a dispatch mode raises, as from any other function of PyTorch's)
    gpuos_cache_task task;
    memcpy(&task, PyBytes_AS_STRING(a[1]), sizeof task);
    const char* places = PyBytes_AS_STRING(a[2]);
    const at::Tensor* some = nullptr;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[3]); ++i) {
      PyObject* o = PyTuple_GET_ITEM(a[3], i);
      if (places[i] < 0 || o == Py_None) continue;
      if (!THPVariable_Check(o) || places[i] >= GPUOS_MAX_CACHE_OPERANDS) {
        PyErr_SetString(PyExc_TypeError, "a tensor for each operand");
        return nullptr;
      }
      const at::Tensor& t = THPVariable_Unpack(o);
      void* p = t.data_ptr();
      if (!p && t.numel() != 0) {
        PyErr_SetString(PyExc_ValueError, "a tensor without memory (of a trace, say)");
        return nullptr;
      }
      task.operand[(int)places[i]].ptr = p;
      some = &t;
    }
    if (task.op == GPUOS_CACHE_ATTENTION && task.operand[0].ptr == task.operand[7].ptr && task.size[4] > 128) {
      const long long sums = (long long)GPUOS_CACHE_SUMS_BYTES(task.size[0], task.size[1], task.size[2], task.size[4]);
      if (space < sums) space = sums;
    }
    at::Tensor workspace;                                       // of the current stream: the allocator gives it to no other before that one is through
    if (space > 0 && some) workspace = at::empty({(int64_t)space}, some->options().dtype(at::kByte).requires_grad(false));
    const int rc = function((int32_t)device, &task, workspace.defined() ? workspace.data_ptr() : nullptr, (uint64_t)space, stream);
    if (rc == GPUOS_OK) {
      for (Py_ssize_t i = 0; i < PyBytes_GET_SIZE(a[4]); ++i) {
        const at::Tensor& t = THPVariable_Unpack(PyTuple_GET_ITEM(a[3], (Py_ssize_t)PyBytes_AS_STRING(a[4])[i]));
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();      // (tensors of inference mode have no versions)
      }
    }
    return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// like(tensor): an empty tensor of its shape, dtype and device, without strides of its own.
PyObject* like(PyObject*, PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a tensor");
    return nullptr;
  }
  HANDLE_TH_ERRORS
    const at::Tensor& t = THPVariable_Unpack(o);
    return THPVariable_Wrap(at::empty(t.sizes(), t.options().requires_grad(false)));
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"key", key, METH_O, "a call's tensors without their addresses"},
                         {"launch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(launch)), METH_FASTCALL, "a descriptor with its tensors' addresses"},
                         {"like", like, METH_O, "an empty tensor like one"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
