// tensors.cpp -- what the Python binding asks of a tensor, in one call a tensor instead
// of one a property (37 to 120 ns each on the GB300's host, five to a tensor).
//
// Each function answers None where the tensor is not plainly what is asked for: a
// subclass, another type, shape, device or layout.  The binding's own checks then
// say what is wrong, or take it after all; so nothing here raises.
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

// A strided cuda tensor (no subclass but Parameter), or null.
const at::Tensor *cuda_tensor(PyObject *obj) {
    if (!THPVariable_CheckExact(obj)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(obj);
    return t.defined() && t.is_cuda() && t.layout() == c10::kStrided ? &t : nullptr;
}

bool has_dtype(const at::Tensor &t, PyObject *dtype) {
    return reinterpret_cast<PyObject *>(torch::getTHPDtype(t.scalar_type())) == dtype;
}

// t's sizes are the n integers of `args`
bool has_sizes(const at::Tensor &t, PyObject *const *args, Py_ssize_t n) {
    if (t.dim() != n) return false;
    for (Py_ssize_t i = 0; i < n; ++i)
        if (!PyLong_Check(args[i]) || t.size(i) != PyLong_AsLongLong(args[i])) {
            PyErr_Clear();
            return false;
        }
    return true;
}

// (dev: its number)
const at::Tensor *asked_for(PyObject *const *args, Py_ssize_t n) {
    if (n < 3 || !PyLong_Check(args[2])) return nullptr;
    const at::Tensor *t = cuda_tensor(args[0]);
    if (!t || !has_dtype(*t, args[1]) || !has_sizes(*t, args + 3, n - 3)) return nullptr;
    const long dev = PyLong_AsLong(args[2]);
    if (dev != t->get_device()) {
        PyErr_Clear();
        return nullptr;
    }
    return t;
}

// flat(tensor, dtype, dev, *sizes): its address, where it is contiguous
PyObject *flat(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        const at::Tensor *t = asked_for(args, n);
        if (t && t->is_contiguous()) return PyLong_FromVoidPtr(t->data_ptr());
    } catch (...) {
    }
    Py_RETURN_NONE;
}

// rows(tensor, dtype, dev, tokens, heads, dim): the bytes of a parason_rows, where
// elements are contiguous and the start and both strides are multiples of 16 bytes
PyObject *rows(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        const at::Tensor *t = n == 6 ? asked_for(args, n) : nullptr;
        if (t && t->stride(2) == 1) {
            struct {
                void *data;
                int64_t token_stride, head_stride;
            } r = {t->data_ptr(), t->stride(0), t->stride(1)};
            const int64_t step = 16 / static_cast<int64_t>(t->element_size());
            if (reinterpret_cast<uintptr_t>(r.data) % 16 == 0 && r.token_stride % step == 0 && r.head_stride % step == 0)
                return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(&r), sizeof(r));
        }
    } catch (...) {
    }
    Py_RETURN_NONE;
}

// alike(a, b): (dtype, dev, address of a, address of b, shape) of two contiguous tensors
// with the same dtype, device and shape
PyObject *alike(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        const at::Tensor *a = n == 2 ? cuda_tensor(args[0]) : nullptr, *b = a ? cuda_tensor(args[1]) : nullptr;
        if (b && a->scalar_type() == b->scalar_type() && a->get_device() == b->get_device() &&
            a->sizes() == b->sizes() && a->is_contiguous() && b->is_contiguous()) {
            PyObject *shape = PyTuple_New(a->dim());
            if (!shape) return nullptr;
            for (int64_t i = 0; i < a->dim(); ++i) {
                PyObject *x = PyLong_FromLongLong(a->size(i));
                if (!x) {
                    Py_DECREF(shape);
                    return nullptr;
                }
                PyTuple_SET_ITEM(shape, i, x);
            }
            return Py_BuildValue("(OiKKN)", torch::getTHPDtype(a->scalar_type()), static_cast<int>(a->get_device()),
                                 static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(a->data_ptr())),
                                 static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(b->data_ptr())), shape);
        }
    } catch (...) {
    }
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"flat", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(flat)), METH_FASTCALL, nullptr},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows)), METH_FASTCALL, nullptr},
    {"alike", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(alike)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
