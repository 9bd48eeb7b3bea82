// tensor_lists.cpp -- a CPython module that reads the addresses, sizes and types of a list of tensors in one call, and counts their
// versions up in another.  The binding is ctypes otherwise; a step over hundreds of tensors in six lists spends half a millisecond on
// asking each of them in Python, several times its kernel's length (301 tensors: 575 us a step, 20 this way).
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <vector>

namespace {

// dtp_dtype, and what the binding alone tells apart
enum Code : int32_t { kBf16 = 0, kF32 = 1, kE4m3 = 2, kOther = -1 };

int32_t code_of(at::ScalarType t) {
    switch (t) {
        case at::kBFloat16: return kBf16;
        case at::kFloat: return kF32;
        case at::kFloat8_e4m3fn: return kE4m3;
        default: return kOther;
    }
}

template <typename T>
PyObject* bytes_of(const std::vector<T>& v) {
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(v.data()), static_cast<Py_ssize_t>(v.size() * sizeof(T)));
}

// read(name, tensors, device, like, per, distinct) -> (addresses, sizes, codes): bytes of uint64, int64 and int32.  All must be
// contiguous CUDA tensors of that device; with `like` (bytes of int64, else None) each has ceil(like / per) values; with
// `distinct` no two that hold values start at the same address.
PyObject* read_list(PyObject*, PyObject* args) {
    const char* name;
    PyObject *list, *like;
    int device, distinct;
    long long per;
    if (!PyArg_ParseTuple(args, "sO!iOLp", &name, &PyList_Type, &list, &device, &like, &per, &distinct)) return nullptr;
    const Py_ssize_t n = PyList_GET_SIZE(list);
    const int64_t* want = nullptr;
    if (like != Py_None) {
        if (!PyBytes_Check(like) || per < 1) {
            PyErr_SetString(PyExc_TypeError, "like must be bytes");
            return nullptr;
        }
        if (PyBytes_GET_SIZE(like) != n * static_cast<Py_ssize_t>(sizeof(int64_t))) {
            PyErr_Format(PyExc_ValueError, "%s must hold as many tensors as params, got %zd", name, n);
            return nullptr;
        }
        want = reinterpret_cast<const int64_t*>(PyBytes_AS_STRING(like));
    }
    std::vector<uint64_t> at(n);
    std::vector<int64_t> numel(n);
    std::vector<int32_t> code(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* o = PyList_GET_ITEM(list, i);
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "%s must hold tensors", name);
            return nullptr;
        }
        const at::TensorBase& t = THPVariable_Unpack(o);
        if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device || !t.is_contiguous()) {
            PyErr_Format(PyExc_ValueError, "%s must be contiguous CUDA tensors on one device", name);
            return nullptr;
        }
        numel[i] = t.numel();
        at[i] = reinterpret_cast<uint64_t>(t.const_data_ptr());
        code[i] = code_of(t.scalar_type());
        if (want && numel[i] != (want[i] + per - 1) / per) {
            PyErr_Format(PyExc_ValueError, "%s must have the sizes that go with params, got %lld values at %zd", name,
                         static_cast<long long>(numel[i]), i);
            return nullptr;
        }
    }
    if (distinct) {
        std::vector<uint64_t> held;
        for (Py_ssize_t i = 0; i < n; ++i)
            if (numel[i]) held.push_back(at[i]);
        std::sort(held.begin(), held.end());
        if (std::adjacent_find(held.begin(), held.end()) != held.end()) {
            PyErr_Format(PyExc_ValueError, "%s must not hold a tensor twice", name);
            return nullptr;
        }
    }
    return Py_BuildValue("(NNN)", bytes_of(at), bytes_of(numel), bytes_of(code));
}

PyObject* read(PyObject* self, PyObject* args) {
    try {
        return read_list(self, args);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// written(lists...): the tensors of the lists (where they hold some) have been written, which a graph that saved one must know.
// Tensors made in inference mode have no versions.
PyObject* written(PyObject*, PyObject* lists) {
    for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(lists); ++k) {
        PyObject* list = PyTuple_GET_ITEM(lists, k);
        if (!PyList_Check(list)) {
            PyErr_SetString(PyExc_TypeError, "written takes lists of tensors");
            return nullptr;
        }
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
            PyObject* o = PyList_GET_ITEM(list, i);
            if (!THPVariable_Check(o)) continue;
            const at::TensorBase& t = THPVariable_Unpack(o);
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
    }
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"read", read, METH_VARARGS, "addresses, sizes and types of a list of tensors"},
                         {"written", written, METH_VARARGS, "tells autograd that the tensors of some lists have been written"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_tensor_lists", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_lists() { return PyModule_Create(&module_def); }
