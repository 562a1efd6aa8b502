// What the binding asks of torch tensors where asking from Python costs more than the
// kernel that follows: lists of some hundred tensors, and the tensors of calls that
// take microseconds.  Nothing is decided here but whether all is as it should be; what
// is not, the binding looks into itself, for its error.
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

// The tensor of an object, or null: strided, with memory of its own.
const at::Tensor* tensor_of(PyObject* x) {
    if (!THPVariable_Check(x)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    return t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}

// scores(x) -> (type, n, vocab, cols, row stride, tile stride, address, device) of
// scores on a GPU, [n, vocab] or in tiles [tiles, n, cols], whose last dimension is
// contiguous; None of anything else.
PyObject* scores(PyObject*, PyObject* x) try {
    const at::Tensor* t = tensor_of(x);
    if (!t || !t->is_cuda() || (t->dim() != 2 && t->dim() != 3) || (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16))
        Py_RETURN_NONE;
    const bool tiles = t->dim() == 3;
    const int64_t cols = t->size(-1), n = t->size(tiles ? 1 : 0);
    if (cols < 1 || (cols > 1 && t->stride(-1) != 1) || (tiles && t->size(0) < 1)) Py_RETURN_NONE;
    return Py_BuildValue("(iLLLLLLi)", int(t->scalar_type() == at::kBFloat16), (long long)n,
                         (long long)(tiles ? t->size(0) * cols : cols), (long long)cols, (long long)t->stride(tiles ? 1 : 0),
                         (long long)(tiles ? t->stride(0) : 0), (long long)reinterpret_cast<intptr_t>(t->data_ptr()),
                         int(t->get_device()));
} catch (const std::exception&) {
    Py_RETURN_NONE;
}

// vector(x, kind, device, n, row) -> its address, of a contiguous tensor [n] (row 0) or
// [n, row] on that GPU: kind 0 float32, 1 int32 or int64 (then negated for int32).  None
// of anything else.
PyObject* vector(PyObject*, PyObject* args) try {
    PyObject* x;
    int kind, device;
    long long n, row;
    if (!PyArg_ParseTuple(args, "OiiLL", &x, &kind, &device, &n, &row)) return nullptr;
    const at::Tensor* t = tensor_of(x);
    if (!t || !t->is_cuda() || t->get_device() != device || !t->is_contiguous() || t->dim() != (row ? 2 : 1) || t->size(0) != n ||
        (row && t->size(1) != row))
        Py_RETURN_NONE;
    const at::ScalarType s = t->scalar_type();
    if (kind == 0 ? s != at::kFloat : s != at::kInt && s != at::kLong) Py_RETURN_NONE;
    const long long at = (long long)reinterpret_cast<intptr_t>(t->data_ptr());
    return PyLong_FromLongLong(s == at::kInt ? -at : at);
} catch (const std::exception&) {
    Py_RETURN_NONE;
}

// views(flat, n, given, entropy, top) -> (stats [n, 2], lse [n], given: [n], entropy: [n],
// top: [n, top] and int32 [n, top]), None for what is not asked for, one after the other
// in the float32 tensor `flat`.
PyObject* views(PyObject*, PyObject* args) try {
    PyObject* x;
    long long n, top;
    int given, entropy;
    if (!PyArg_ParseTuple(args, "OLppL", &x, &n, &given, &entropy, &top)) return nullptr;
    if (!THPVariable_Check(x)) {
        PyErr_SetString(PyExc_TypeError, "a tensor wanted");
        return nullptr;
    }
    const at::Tensor& flat = THPVariable_Unpack(x);
    at::Tensor t[6];
    int64_t at = 0;
    auto part = [&](at::Tensor& t, int64_t row) {
        t = row ? flat.as_strided({n, row}, {row, 1}, at) : flat.as_strided({n}, {1}, at);
        at += n * (row ? row : 1);
    };
    part(t[0], 2);
    part(t[1], 0);
    if (given) part(t[2], 0);
    if (entropy) part(t[3], 0);
    if (top > 0) {
        part(t[4], top);
        part(t[5], top);
        t[5] = t[5].view(at::kInt);
    }
    PyObject* r = PyTuple_New(6);  // (None for a tensor that is not there)
    for (int i = 0; r && i < 6; i++) {
        PyObject* v = THPVariable_Wrap(t[i]);
        if (v) PyTuple_SET_ITEM(r, i, v);
        else Py_CLEAR(r);
    }
    return r;
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// written(a, b, ...): counts a version of each tensor, or of those of a list (None: none),
// as an operation in place does, so that a backward pass that saved one finds it changed.
// Tensors of inference mode, which nothing saves, have no count.
bool count_version(PyObject* x) {
    if (x == Py_None) return true;
    if (!THPVariable_Check(x)) return false;
    const at::Tensor& t = THPVariable_Unpack(x);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    return true;
}
PyObject* written(PyObject*, PyObject* args) try {
    bool all = true;
    for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(args); k++) {
        PyObject* x = PyTuple_GET_ITEM(args, k);
        if (!PyList_Check(x) && !PyTuple_Check(x)) {
            all = count_version(x) && all;
            continue;
        }
        for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(x); i++) all = count_version(PySequence_Fast_GET_ITEM(x, i)) && all;
    }
    if (all) Py_RETURN_NONE;
    PyErr_SetString(PyExc_TypeError, "tensors wanted");
    return nullptr;
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

PyMethodDef methods[] = {{"gather", gather, METH_O, nullptr},       {"same_shapes", same_shapes, METH_VARARGS, nullptr},
                         {"scores", scores, METH_O, nullptr},       {"vector", vector, METH_VARARGS, nullptr},
                         {"views", views, METH_VARARGS, nullptr},   {"written", written, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
