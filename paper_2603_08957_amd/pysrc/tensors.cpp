// Addresses, types and sizes of a list of torch tensors in one pass, for the calls
// that take many: asked of each tensor from Python, five properties of some hundred
// tensors cost more than the kernels that follow.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>

namespace {

// The list's items as a borrowed sequence, or null where it is none (no error set).
PyObject* items_of(PyObject* list) {
    PyObject* s = PySequence_Fast(list, "");
    if (!s) PyErr_Clear();
    return s;
}

// gather(tensors) -> (0, device, addresses, types, sizes): native int64, int32 and
// int64 arrays as bytes, types 0 for float32 and 1 for bfloat16, device -1 for no
// tensors.  Else (why, at): tensor `at` 1: is none, 2: is not on the first one's GPU,
// 3: is not contiguous, 4: has another type.
PyObject* gather(PyObject*, PyObject* list) {
    PyObject* s = items_of(list);
    if (!s) return Py_BuildValue("(ii)", 1, 0);
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(s);
    PyObject* addresses = PyBytes_FromStringAndSize(nullptr, n * 8);
    PyObject* types = PyBytes_FromStringAndSize(nullptr, n * 4);
    PyObject* sizes = PyBytes_FromStringAndSize(nullptr, n * 8);
    int why = addresses && types && sizes ? 0 : -1;
    Py_ssize_t at = 0;
    int64_t device = -1;
    if (!why) {
        int64_t* a = reinterpret_cast<int64_t*>(PyBytes_AS_STRING(addresses));
        int32_t* t = reinterpret_cast<int32_t*>(PyBytes_AS_STRING(types));
        int64_t* z = reinterpret_cast<int64_t*>(PyBytes_AS_STRING(sizes));
        try {
            for (; at < n && !why; at++) {
                PyObject* item = PySequence_Fast_GET_ITEM(s, at);
                if (!THPVariable_Check(item)) {
                    why = 1;
                    break;
                }
                const at::Tensor& x = THPVariable_Unpack(item);
                if (!x.is_cuda() || (at > 0 && x.get_device() != device)) why = 2;
                else if (x.layout() != at::kStrided || !x.is_contiguous()) why = 3;
                else if (x.scalar_type() != at::kFloat && x.scalar_type() != at::kBFloat16) why = 4;
                if (why) break;
                device = x.get_device();
                a[at] = int64_t(reinterpret_cast<intptr_t>(x.data_ptr()));
                t[at] = x.scalar_type() == at::kBFloat16;
                z[at] = x.numel();
            }
        } catch (const std::exception&) {  // (a tensor without memory of its own)
            why = 1;
        }
    }
    PyObject* r = why < 0 ? nullptr : why ? Py_BuildValue("(in)", why, at) : Py_BuildValue("(iLOOO)", 0, (long long)device, addresses, types, sizes);
    Py_XDECREF(addresses);
    Py_XDECREF(types);
    Py_XDECREF(sizes);
    Py_DECREF(s);
    return r;
}

// same_shapes(tensors, others) -> bool, of two lists that gather took.
PyObject* same_shapes(PyObject*, PyObject* args) {
    PyObject *x, *y;
    if (!PyArg_ParseTuple(args, "OO", &x, &y)) return nullptr;
    PyObject* s = items_of(x);
    PyObject* o = items_of(y);
    bool same = s && o && PySequence_Fast_GET_SIZE(s) == PySequence_Fast_GET_SIZE(o);
    try {
        for (Py_ssize_t i = 0; same && i < PySequence_Fast_GET_SIZE(s); i++) {
            PyObject *u = PySequence_Fast_GET_ITEM(s, i), *v = PySequence_Fast_GET_ITEM(o, i);
            same = THPVariable_Check(u) && THPVariable_Check(v) && THPVariable_Unpack(u).sizes() == THPVariable_Unpack(v).sizes();
        }
    } catch (const std::exception&) {
        same = false;
    }
    Py_XDECREF(s);
    Py_XDECREF(o);
    return PyBool_FromLong(same);
}

PyMethodDef methods[] = {{"gather", gather, METH_O, nullptr}, {"same_shapes", same_shapes, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
