// The bindings' checks of a call's tensors, as a Python module: type, sizes, strides and device of a torch tensor are read where they are,
// not through five methods of the interpreter each (0.1 instead of 0.5 us a tensor, of which a call has 5 to 15 and a small kernel takes 3).
// A tensor that is what it has to be gives its address; whatever is not goes to the Python function of the same name, which says why.
// STEM_TORCH: the torch that it is compiled against (its version and commit), as tensors lie in memory as that one has them.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <initializer_list>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

enum { kValues, kWhole, kLines, kChecks };
PyObject* in_python[kChecks];                          // the functions that have the last word

PyObject* ask_python(int which, PyObject* const* args, Py_ssize_t n) {
    if (!in_python[which]) {
        PyErr_SetString(PyExc_RuntimeError, "begin() first");
        return nullptr;
    }
    return PyObject_Vectorcall(in_python[which], args, (size_t)n, nullptr);
}

// A plain tensor (or parameter) of dense values, or none
const at::Tensor* tensor_of(PyObject* x) {
    if (!THPVariable_CheckExact(x)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    return t.defined() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}
bool has_type(const at::Tensor& t, PyObject* dtype) {
    return THPDtype_Check(dtype) && reinterpret_cast<THPDtype*>(dtype)->scalar_type == t.scalar_type();
}
bool as_number(PyObject* x, int64_t* out) {
    if (!PyLong_CheckExact(x)) return false;
    int overflow = 0;
    *out = PyLong_AsLongLongAndOverflow(x, &overflow);
    return overflow == 0;
}
bool same(PyObject* tuple, c10::IntArrayRef numbers) {
    if (!PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) != (Py_ssize_t)numbers.size()) return false;
    for (size_t i = 0; i < numbers.size(); ++i) {
        int64_t x;
        if (!as_number(PyTuple_GET_ITEM(tuple, i), &x) || x != numbers[i]) return false;
    }
    return true;
}
// (type of contiguous numbers where none is named)
bool has_type_or_int32(const at::Tensor& t, PyObject* const* args, Py_ssize_t n, Py_ssize_t at) {
    return n > at ? has_type(t, args[at]) : t.scalar_type() == at::kInt;
}

// f says whether a tensor is what the arguments ask for; nothing that C++ throws leaves here.
template <typename F>
PyObject* address(int which, PyObject* const* args, Py_ssize_t n, Py_ssize_t device_at, F&& f) {
    const void* p = nullptr;
    bool good = false;
    try {
        int64_t device;
        if (const at::Tensor* t = n > device_at && as_number(args[device_at], &device) ? tensor_of(args[0]) : nullptr)
            if (t->get_device() == device && f(*t)) p = t->data_ptr(), good = true;
    } catch (...) {
        good = false;
    }
    return good ? PyLong_FromVoidPtr(const_cast<void*>(p)) : ask_python(which, args, n);
}

// values(t, like, name, dev): like is (sizes, strides, type), or None
PyObject* values(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n == 4 && args[1] == Py_None) Py_RETURN_NONE;
    return address(kValues, args, n, 3, [&](const at::Tensor& t) {
        PyObject* like = args[1];
        return n == 4 && PyTuple_Check(like) && PyTuple_GET_SIZE(like) == 3 && same(PyTuple_GET_ITEM(like, 0), t.sizes()) &&
               has_type(t, PyTuple_GET_ITEM(like, 2)) && (same(PyTuple_GET_ITEM(like, 1), t.strides()) || t.numel() == 0);
    });
}
// whole(t, n, name, dev, dtype = int32)
PyObject* whole(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return address(kWhole, args, n, 3, [&](const at::Tensor& t) {
        int64_t least;
        return n <= 5 && as_number(args[1], &least) && has_type_or_int32(t, args, n, 4) && t.numel() >= least && t.is_contiguous();
    });
}
// lines(t, n, each, name, dev, dtype = int32)
PyObject* lines(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return address(kLines, args, n, 4, [&](const at::Tensor& t) {
        int64_t least, each;                           // (two dimensions; what else may do is Python's matter)
        return n <= 6 && as_number(args[1], &least) && as_number(args[2], &each) && t.dim() == 2 && t.size(0) >= least && t.size(1) == each &&
               has_type_or_int32(t, args, n, 5) && t.is_contiguous();
    });
}

// begin(values, whole, lines): the Python functions
PyObject* begin(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != kChecks) {
        PyErr_SetString(PyExc_TypeError, "three functions are needed");
        return nullptr;
    }
    for (int i = 0; i < kChecks; ++i) {
        Py_INCREF(args[i]);
        Py_XDECREF(in_python[i]);
        in_python[i] = args[i];
    }
    Py_RETURN_NONE;
}

#define STEM_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {STEM_METHOD(values), STEM_METHOD(whole), STEM_METHOD(lines), STEM_METHOD(begin), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

// Whether the torch that is there is STEM_TORCH.
bool right_torch() {
    bool right = false;
    PyObject *torch = PyImport_ImportModule("torch"), *version = nullptr, *about = nullptr, *commit = nullptr, *here = nullptr;
    if (torch && (version = PyObject_GetAttrString(torch, "__version__")) && (about = PyObject_GetAttrString(torch, "version")) &&
        (commit = PyObject_GetAttrString(about, "git_version")) && (here = PyUnicode_FromFormat("%S %S", version, commit))) {
        right = PyUnicode_CompareWithASCIIString(here, STEM_TORCH) == 0;
        if (!right) PyErr_Format(PyExc_ImportError, "the checks of tensors are made for torch %s, and this is torch %U", STEM_TORCH, here);
    }
    for (PyObject* x : {torch, version, about, commit, here}) Py_XDECREF(x);
    return right;
}

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return right_torch() ? PyModule_Create(&module) : nullptr; }
