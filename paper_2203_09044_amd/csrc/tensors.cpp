// A look at a list of torch tensors: where each lies, how long it is, of which type and whether it is contiguous.  A plan of the
// server's update holds addresses, so every call has to know that its tensors are still those; from Python that is several calls a
// tensor (150 ns together; the addresses alone, in one call for the list, 28), here one pass over the list (7 ns a tensor: a step of
// 400 tensors of 1000 elements 38.0 us with the addresses alone looked at, 20.4 with everything).
#include <Python.h>
#include <string.h>

#include <torch/csrc/autograd/python_variable.h>

namespace {
struct Seen {
    const void *at;
    int64_t elems;
    int32_t type;
    uint8_t contiguous, device_type;
    int16_t device;
};
static_assert(sizeof(Seen) == 24, "no padding: records are compared byte by byte");

// false: no tensor, or one without memory of its own
bool see(PyObject *object, Seen &s)
{
    try {
        if (!THPVariable_Check(object)) return false;
        const at::Tensor &t = THPVariable_Unpack(object);
        if (!t.defined() || !t.has_storage()) return false;
        s = Seen{t.const_data_ptr(), t.numel(), (int32_t)t.scalar_type(), t.is_contiguous(), (uint8_t)t.device().type(),
                 (int16_t)t.device().index()};
        return true;
    } catch (...) {                               // a kind of tensor that does not tell
        return false;
    }
}

PyObject *look(PyObject *, PyObject *list)
{
    if (!PyList_Check(list)) {
        PyErr_SetString(PyExc_TypeError, "a list of tensors is needed");
        return nullptr;
    }
    const Py_ssize_t n = PyList_GET_SIZE(list);
    PyObject *out = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(Seen));
    for (Py_ssize_t k = 0; out && k < n; ++k) {
        Seen s;
        if (!see(PyList_GET_ITEM(list, k), s)) {
            Py_DECREF(out);
            PyErr_SetString(PyExc_ValueError, "tensors with memory of their own are needed");
            return nullptr;
        }
        memcpy(PyBytes_AS_STRING(out) + k * sizeof(Seen), &s, sizeof(Seen));
    }
    return out;
}

PyObject *same(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs != 2 || !PyList_Check(args[0]) || !PyBytes_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "a list of tensors and what look() returned are needed");
        return nullptr;
    }
    const Py_ssize_t n = PyList_GET_SIZE(args[0]);
    if (PyBytes_GET_SIZE(args[1]) != n * (Py_ssize_t)sizeof(Seen)) Py_RETURN_FALSE;
    const char *then = PyBytes_AS_STRING(args[1]);
    for (Py_ssize_t k = 0; k < n; ++k) {
        Seen s;
        if (!see(PyList_GET_ITEM(args[0], k), s) || memcmp(&s, then + k * sizeof(Seen), sizeof(Seen)) != 0) Py_RETURN_FALSE;
    }
    Py_RETURN_TRUE;
}

PyMethodDef methods[] = {
    {"look", look, METH_O, "look(list of tensors) -> bytes: what they are and where they lie"},
    {"same", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(same)), METH_FASTCALL,
     "same(list of tensors, bytes of look) -> whether they still are and lie as they did"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&module); }
