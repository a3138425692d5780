// Pointer tables of lists of tensors, for the binding's calls with a list per argument: the checks that binding.py spells out, without
// an interpreter's turn for every attribute of every tensor (eight workers and six lists: 17 us of a call that takes 5).  Anything out of
// the ordinary is answered with -1, and binding.py's own checks then say what it is.  That includes what a tensor throws when it is asked
// (a wrapper without memory of its own, under a transformation of functions for instance, has sizes but no address): the interpreter calls
// these functions by its C interface, which no exception may leave.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

constexpr at::ScalarType TYPES[] = {at::kFloat, at::kHalf, at::kBFloat16, at::kInt};

bool tensor_of(PyObject* o, long type, long device, const at::Tensor*& t)
{
    if (!THPVariable_Check(o)) return false;
    t = &THPVariable_Unpack(o);
    return t->layout() == at::kStrided && !t->is_nested() && t->scalar_type() == TYPES[type] && (t->is_cuda() ? t->get_device() : -1) == device;
}

// matrix(tensors, rows, columns, type, device, table address) -> distance of rows, 0 where no tensor has two, or -1
PyObject* matrix(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 6 || !PyList_Check(a[0]) || !PyList_Check(a[1]) || PyList_GET_SIZE(a[0]) != PyList_GET_SIZE(a[1])) return PyLong_FromLong(-1);
    const int64_t cols = PyLong_AsLongLong(a[2]);
    const long type = PyLong_AsLong(a[3]), device = PyLong_AsLong(a[4]);
    void** table = static_cast<void**>(PyLong_AsVoidPtr(a[5]));
    if (PyErr_Occurred()) return nullptr;
    if (type < 0 || type > 3 || !table) return PyLong_FromLong(-1);
    int64_t ld = -1;
    for (Py_ssize_t q = 0; q < PyList_GET_SIZE(a[0]); ++q) {
        const at::Tensor* t;
        const int64_t rows = PyLong_AsLongLong(PyList_GET_ITEM(a[1], q));
        if (PyErr_Occurred()) return nullptr;
        if (!tensor_of(PyList_GET_ITEM(a[0], q), type, device, t) || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols)
            return PyLong_FromLong(-1);
        table[q] = nullptr;
        if (rows == 0) continue;
        if (t->stride(1) != 1 && cols > 1) return PyLong_FromLong(-1);
        if (rows > 1 && t->stride(0) != ld) {
            if (ld >= 0 || t->stride(0) < cols) return PyLong_FromLong(-1);
            ld = t->stride(0);
        }
        table[q] = t->data_ptr();
        if (!table[q] && cols) return PyLong_FromLong(-1);
    }
    return PyLong_FromLongLong(ld < 0 ? 0 : ld);
}

// vectors(tensors or None each, numbers of elements, type, device, table address) -> 0 or -1
PyObject* vectors(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 5 || !PyList_Check(a[0]) || !PyList_Check(a[1]) || PyList_GET_SIZE(a[0]) != PyList_GET_SIZE(a[1])) return PyLong_FromLong(-1);
    const long type = PyLong_AsLong(a[2]), device = PyLong_AsLong(a[3]);
    void** table = static_cast<void**>(PyLong_AsVoidPtr(a[4]));
    if (PyErr_Occurred()) return nullptr;
    if (type < 0 || type > 3 || !table) return PyLong_FromLong(-1);
    for (Py_ssize_t q = 0; q < PyList_GET_SIZE(a[0]); ++q) {
        PyObject* o = PyList_GET_ITEM(a[0], q);
        table[q] = nullptr;
        if (o == Py_None) continue;
        const at::Tensor* t;
        const int64_t size = PyLong_AsLongLong(PyList_GET_ITEM(a[1], q));
        if (PyErr_Occurred()) return nullptr;
        if (!tensor_of(o, type, device, t) || t->numel() != size || !t->is_contiguous()) return PyLong_FromLong(-1);
        if (!size) continue;
        table[q] = t->data_ptr();
        if (!table[q]) return PyLong_FromLong(-1);
    }
    return PyLong_FromLong(0);
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) noexcept
{
    try {
        return F(self, a, n);
    } catch (...) {
        PyErr_Clear();          // a Python error on the way out of the tensor's own code is said again by binding.py's checks
        return PyLong_FromLong(-1);
    }
}

PyMethodDef methods[] = {{"matrix", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<matrix>)), METH_FASTCALL, nullptr},
                         {"vectors", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<vectors>)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tables", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tables() { return PyModule_Create(&module); }
