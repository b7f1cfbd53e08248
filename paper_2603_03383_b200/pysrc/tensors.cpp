// What binding.py asks of tensors before their addresses go to the library, all of a call's in one step.  An attribute of a tensor costs the
// interpreter 50 to 70 ns, four of them for each of a call's ten tensors as much as the call itself (compaction 5.8 us with none looked at,
// 8.5 with all of them by attributes, 5.9 so).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

enum { BF16 = 0, I32 = 1, I64 = 2, F32 = 3, ANY = 4, FP8 = 5, TYPES = 7, OPTIONAL = 16, STRIDED = 32, LIKE_PREVIOUS = 64 };

bool is_kind(c10::ScalarType t, long kind) {
    using S = c10::ScalarType;
    switch (kind & TYPES) {
    case BF16: return t == S::BFloat16;
    case I32: return t == S::Int || t == S::UInt32;
    case I64: return t == S::Long || t == S::UInt64;
    case F32: return t == S::Float;
    case FP8: return t == S::Float8_e4m3fn;
    default: return true;
    }
}

// The address of x, or none: it is refused (or an exception is set).  *device: of the tensors so far, -2 in front of the first.
PyObject *address_of(PyObject *x, long kind, long long size, int *device, const at::Tensor **previous) {
    if (x == Py_None && (kind & OPTIONAL)) return Py_NewRef(Py_None);
    if (!THPVariable_Check(x)) return nullptr;
    try {
        const at::Tensor &t = THPVariable_Unpack(x);
        const int on = t.is_cuda() ? (int)t.device().index() : t.is_cpu() ? -1 : -3;
        if (*device == -2) *device = on;
        const at::Tensor *before = *previous;
        *previous = &t;
        if (on == -3 || on != *device || t.layout() != c10::kStrided || !is_kind(t.scalar_type(), kind) || t.numel() < size) return nullptr;
        if (!(kind & STRIDED) && !t.is_contiguous()) return nullptr;
        if ((kind & LIKE_PREVIOUS) && !(before && t.sizes() == before->sizes())) return nullptr;
        return PyLong_FromVoidPtr(const_cast<void *>(t.const_data_ptr()));
    } catch (const std::exception &e) {         // (a tensor without storage, say)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// addresses(tensor, kind, size, tensor, kind, size, ...) -> (device index, address, address, ...)
// kind: an element type, + OPTIONAL (None is passed on), + STRIDED (else contiguous), + LIKE_PREVIOUS (of the sizes of the tensor in front of it)
// size: elements at least (buffers may be made for more sequences than a call has)
// All tensors are on one device, which is a CUDA device or, as -1, the host.  Where something is not so: the place of the first such tensor.
PyObject *addresses(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    const Py_ssize_t n = n_args / 3;
    if (n < 1 || n_args % 3) {
        PyErr_SetString(PyExc_TypeError, "addresses: (tensor, kind, size) expected");
        return nullptr;
    }
    PyObject *out = PyTuple_New(n + 1);
    if (!out) return nullptr;
    int device = -2;
    const at::Tensor *previous = nullptr;
    for (Py_ssize_t i = 0; i < n; ++i) {
        const long kind = PyLong_AsLong(args[3 * i + 1]);
        const long long size = PyLong_AsLongLong(args[3 * i + 2]);
        PyObject *address = PyErr_Occurred() ? nullptr : address_of(args[3 * i], kind, size, &device, &previous);
        if (!address) {
            Py_DECREF(out);
            return PyErr_Occurred() ? nullptr : PyLong_FromSsize_t(i);
        }
        PyTuple_SET_ITEM(out, i + 1, address);
    }
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(device));
    return out;
}

PyMethodDef methods[] = {{"addresses", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(addresses)), METH_FASTCALL,
                          "(tensor, kind, size) triples -> (device, addresses ...), or the index of the first tensor that is refused"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() {
    return PyModule_Create(&module);
}
