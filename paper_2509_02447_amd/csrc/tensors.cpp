// What a list of tensors says of itself, for the binding (AdamW._pointers): host code, a CPython module.  Asked from Python, a tensor's type, size, place, order and address are
// five calls, 0.23 us together, and a step over several hundred tensors waits for its checks (the norm of 600: 141 us, so 13.5).
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

namespace {

// pointers(tensors, sizes, dtype) -> bytearray of 64-bit addresses, 0 for None.  tensors: a sequence; sizes: a buffer of as many int64; what is there must be a tensor of
// `dtype` with that many elements, contiguous and on the GPU: AssertionError.
PyObject *pointers(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    if (n_args != 3 || !THPDtype_Check(args[2])) {
        PyErr_SetString(PyExc_TypeError, "pointers(tensors, sizes, dtype)");
        return nullptr;
    }
    const at::ScalarType type = reinterpret_cast<THPDtype *>(args[2])->scalar_type;
    THPObjectPtr list(PySequence_Fast(args[0], "a list of tensors"));
    if (!list) return nullptr;
    Py_buffer sizes;
    if (PyObject_GetBuffer(args[1], &sizes, PyBUF_SIMPLE)) return nullptr;
    const Py_ssize_t n = sizes.len / (Py_ssize_t)sizeof(int64_t);
    const int64_t *const size = static_cast<const int64_t *>(sizes.buf);
    PyObject *out = nullptr;
    const char *wrong = nullptr;
    if (PySequence_Fast_GET_SIZE(list.get()) != n) {
        wrong = "one gradient (or None) for each tensor";
    } else if ((out = PyByteArray_FromStringAndSize(nullptr, std::max<Py_ssize_t>(1, n) * 8))) {
        uint64_t *const to = reinterpret_cast<uint64_t *>(PyByteArray_AS_STRING(out));
        to[0] = 0;
        try {
            for (Py_ssize_t i = 0; i < n && !wrong; ++i) {
                PyObject *const item = PySequence_Fast_GET_ITEM(list.get(), i);
                to[i] = 0;
                if (item == Py_None) continue;
                const at::Tensor *const t = THPVariable_Check(item) ? &THPVariable_Unpack(item) : nullptr;
                if (t && t->scalar_type() == type && t->is_cuda() && t->layout() == at::kStrided && t->numel() == size[i] && t->is_contiguous()) to[i] = reinterpret_cast<uint64_t>(t->const_data_ptr());
                else wrong = "gradients must have the plan's type and sizes, be contiguous and on the GPU";
            }
        } catch (...) {
            PyBuffer_Release(&sizes);
            Py_DECREF(out);
            throw;
        }
    }
    PyBuffer_Release(&sizes);
    if (wrong) {
        Py_CLEAR(out);
        PyErr_SetString(PyExc_AssertionError, wrong);
    }
    return out;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"pointers", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(pointers)), METH_FASTCALL, "Addresses of tensors that are as they have to be."}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
