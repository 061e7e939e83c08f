// The forms of a call's tensors: all that a call's checks look at (type, device, sizes, strides), kept from the last
// call whose checks passed and compared with the next one's in a fraction of a microsecond, where the same
// comparison in Python takes longer than a small kernel.  Places in memory are not part of a form.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <memory>
#include <vector>

namespace {

struct Form {
  PyObject_HEAD
  std::vector<int64_t>* kept;      // null: nothing is
};

// Walks over the tensors' forms; `each` takes one number and says whether to go on.  -1: a Python error is set.
template <typename F>
int walk(PyObject* const* args, Py_ssize_t n, F&& each) {
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (args[i] == Py_None) {
      if (!each(-1)) return 0;
      continue;
    }
    if (!THPVariable_Check(args[i])) {
      PyErr_SetString(PyExc_TypeError, "a tensor or None is needed");
      return -1;
    }
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    const int64_t dims = t.dim();
    if (!each(static_cast<int64_t>(t.scalar_type()) << 8 | dims) || !each(static_cast<int64_t>(t.device().type()) << 8 | (t.device().index() & 255))) return 0;
    const auto sizes = t.sizes(), strides = t.strides();
    for (int64_t d = 0; d < dims; ++d)
      if (!each(sizes[d]) || !each(strides[d])) return 0;
  }
  return 1;
}

template <typename F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// keep(*tensors): from now on these are the kept forms; keep() forgets them.
PyObject* form_keep(Form* self, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    delete self->kept;
    self->kept = nullptr;
    if (n) {
      auto fresh = std::make_unique<std::vector<int64_t>>();
      if (walk(args, n, [&](int64_t v) { fresh->push_back(v); return true; }) < 0) return nullptr;
      self->kept = fresh.release();
    }
    Py_RETURN_NONE;
  });
}

// places(*tensors): a tuple of the tensors' addresses (0 for None) if their forms are the kept ones, else None.
PyObject* form_places(Form* self, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (!self->kept) Py_RETURN_NONE;
    const int64_t* at = self->kept->data();
    const int64_t* const end = at + self->kept->size();
    const int rc = walk(args, n, [&](int64_t v) { return at != end && *at++ == v; });
    if (rc < 0) return nullptr;
    if (rc == 0 || at != end) Py_RETURN_NONE;
    PyObject* places = PyTuple_New(n);
    if (!places) return nullptr;
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* place = nullptr;
      try {
        place = args[i] == Py_None ? PyLong_FromLong(0)
                                   : PyLong_FromSize_t(reinterpret_cast<size_t>(THPVariable_Unpack(args[i]).data_ptr()));
      } catch (...) {
        Py_DECREF(places);
        throw;
      }
      if (!place) {
        Py_DECREF(places);
        return nullptr;
      }
      PyTuple_SET_ITEM(places, i, place);
    }
    return places;
  });
}

PyObject* form_new(PyTypeObject* type, PyObject*, PyObject*) {
  Form* self = reinterpret_cast<Form*>(type->tp_alloc(type, 0));
  if (self) self->kept = nullptr;
  return reinterpret_cast<PyObject*>(self);
}

void form_free(Form* self) {
  delete self->kept;
  Py_TYPE(self)->tp_free(reinterpret_cast<PyObject*>(self));
}

PyMethodDef kMethods[] = {
    {"keep", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(form_keep)), METH_FASTCALL, "keep the forms of these tensors; none: forget"},
    {"places", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(form_places)), METH_FASTCALL, "addresses, if the forms are the kept ones; else None"},
    {nullptr, nullptr, 0, nullptr},
};

PyTypeObject kType = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_ans_form", "forms of a call's tensors", -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ans_form() {
  kType.tp_name = "_ans_form.Form";
  kType.tp_basicsize = sizeof(Form);
  kType.tp_flags = Py_TPFLAGS_DEFAULT;
  kType.tp_new = form_new;
  kType.tp_dealloc = reinterpret_cast<destructor>(form_free);
  kType.tp_methods = kMethods;
  if (PyType_Ready(&kType) < 0) return nullptr;
  PyObject* m = PyModule_Create(&kModule);
  if (!m) return nullptr;
  Py_INCREF(&kType);
  if (PyModule_AddObject(m, "Form", reinterpret_cast<PyObject*>(&kType)) < 0) {
    Py_DECREF(&kType);
    Py_DECREF(m);
    return nullptr;
  }
  if (PyModule_AddStringConstant(m, "MADE_FOR", ANS_MADE_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
