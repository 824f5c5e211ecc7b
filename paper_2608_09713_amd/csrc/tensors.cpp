// note(tensors): what a call on them depends on, read at once: each tensor's address,
// bytes, element type, device and whether its elements lie one behind the other, as
// bytes that are equal as long as all of it is.  A tensor's storage, size or strides
// can be exchanged behind its Python object (`.data = ...`) with no trace but these,
// also at the same address.  Read through Python's attributes they take more of
// a step over many small tensors than its kernels (640 tensors: 119 us, the
// addresses alone 23, all of it by this 5).
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cstdint>
#include <cstring>

namespace {

struct Seen {
    int64_t address, bytes;
    int32_t type;  // (of None all of these are -1)
    int16_t device;
    int16_t contiguous;
};
static_assert(sizeof(Seen) == 24, "three words, with no bytes between the members");

// whether it is a tuple of tensors and Nones; sets the error if not
bool are_tensors(PyObject* tensors) {
    bool ok = PyTuple_Check(tensors);
    for (Py_ssize_t i = 0; ok && i < PyTuple_GET_SIZE(tensors); ++i) {
        PyObject* o = PyTuple_GET_ITEM(tensors, i);
        ok = o == Py_None || THPVariable_Check(o);
    }
    if (!ok) PyErr_SetString(PyExc_TypeError, "a tuple of tensors is needed");
    return ok;
}

PyObject* note(PyObject*, PyObject* tensors) {
    HANDLE_TH_ERRORS
    if (!are_tensors(tensors)) return nullptr;
    const Py_ssize_t n = PyTuple_GET_SIZE(tensors);
    THPObjectPtr out(PyBytes_FromStringAndSize(nullptr, n * Py_ssize_t(sizeof(Seen))));
    if (!out) return nullptr;
    char* to = PyBytes_AsString(out.get());
    for (Py_ssize_t i = 0; i < n; ++i, to += sizeof(Seen)) {
        Seen s{0, 0, -1, -1, -1};
        PyObject* o = PyTuple_GET_ITEM(tensors, i);
        if (o != Py_None) {
            const at::Tensor& t = THPVariable_Unpack(o);
            s.address = int64_t(reinterpret_cast<intptr_t>(t.data_ptr()));
            s.bytes = int64_t(t.nbytes());
            s.type = int32_t(t.scalar_type());
            s.device = int16_t(t.is_cpu() ? -1 : t.get_device());  // (as get_device gives in Python)
            s.contiguous = t.is_contiguous();
        }
        std::memcpy(to, &s, sizeof(s));
    }
    return out.release();
    END_HANDLE_TH_ERRORS
}

// changed(tensors): counts a change in place of each, so that autograd refuses a
// backward pass that saved one before.  (Tensors of inference mode have no count.)
PyObject* changed(PyObject*, PyObject* tensors) {
    HANDLE_TH_ERRORS
    if (!are_tensors(tensors)) return nullptr;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(tensors); ++i) {
        PyObject* o = PyTuple_GET_ITEM(tensors, i);
        if (o == Py_None) continue;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"note", note, METH_O, "Addresses, bytes, types, devices and layouts of a tuple of tensors."},
                         {"changed", changed, METH_O, "Counts a change in place of each tensor of a tuple."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
