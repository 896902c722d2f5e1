// Pointer tables of a call's tensors for the ctypes binding.  Short calls take less time on the GPU than the interpreter needs to
// look at their tensors one by one, so the look is taken here.
//
//   addresses(device, ((name, dtype, shards, sizes), ...)) -> (keep, [address, ...]) or None
//
// `shards`: a list or tuple of tensors (the address is that of a table of their addresses, which lives in `keep`), one tensor
// (its own address) or None (None).  `sizes`: the elements of each, as a tuple of ints (one int for one tensor).  None as the result:
// something is not a contiguous tensor of that type and size in the memory of `device`, and the caller sees to it.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// The address of a tensor that is as it should be, or false
bool address_of(PyObject *o, at::ScalarType type, PyObject *size, long device, void **out) {
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.numel() != PyLong_AsLongLong(size) || !t.is_contiguous())
        return false;
    *out = t.data_ptr();
    return true;
}

PyObject *addresses(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    if (n_args != 2 || !PyTuple_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "addresses(device, ((name, dtype, shards, sizes), ...))");
        return nullptr;
    }
    try {
        const long device = PyLong_AsLong(args[0]);
        const Py_ssize_t n = PyTuple_GET_SIZE(args[1]);
        Py_ssize_t total = 0;
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject *item = PyTuple_GET_ITEM(args[1], i);
            if (!PyTuple_Check(item) || PyTuple_GET_SIZE(item) != 4 || !THPDtype_Check(PyTuple_GET_ITEM(item, 1))) Py_RETURN_NONE;
            if (PyTuple_Check(PyTuple_GET_ITEM(item, 3))) total += PyTuple_GET_SIZE(PyTuple_GET_ITEM(item, 3));
        }
        PyObject *keep = PyBytes_FromStringAndSize(nullptr, total * (Py_ssize_t)sizeof(void *));
        PyObject *out = keep ? PyList_New(n) : nullptr;
        if (!out) { Py_XDECREF(keep); return nullptr; }
        void **at = reinterpret_cast<void **>(PyBytes_AS_STRING(keep));
        bool right = true;
        for (Py_ssize_t i = 0; right && i < n; ++i) {
            PyObject *item = PyTuple_GET_ITEM(args[1], i), *shards = PyTuple_GET_ITEM(item, 2), *sizes = PyTuple_GET_ITEM(item, 3);
            const at::ScalarType type = reinterpret_cast<THPDtype *>(PyTuple_GET_ITEM(item, 1))->scalar_type;
            PyObject *value = nullptr;
            if (shards == Py_None) {
                value = Py_NewRef(Py_None);
            } else if (PyLong_Check(sizes)) {
                void *p = nullptr;
                right = address_of(shards, type, sizes, device, &p);
                if (right) value = PyLong_FromVoidPtr(p);
            } else if ((PyList_Check(shards) || PyTuple_Check(shards)) && PyTuple_Check(sizes) &&
                       PySequence_Fast_GET_SIZE(shards) == PyTuple_GET_SIZE(sizes)) {
                value = PyLong_FromVoidPtr(at);
                for (Py_ssize_t k = 0; right && k < PyTuple_GET_SIZE(sizes); ++k)
                    right = address_of(PySequence_Fast_GET_ITEM(shards, k), type, PyTuple_GET_ITEM(sizes, k), device, at++);
            } else {
                right = false;
            }
            if (!value) value = Py_NewRef(Py_None);
            PyList_SET_ITEM(out, i, value);
        }
        PyObject *result = right && !PyErr_Occurred() ? PyTuple_Pack(2, keep, out) : nullptr;
        Py_DECREF(keep);
        Py_DECREF(out);
        if (result || PyErr_Occurred()) return result;
        Py_RETURN_NONE;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {{"addresses", (PyCFunction)(void (*)(void))addresses, METH_FASTCALL, "addresses(device, named) -> (keep, addresses) or None"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
