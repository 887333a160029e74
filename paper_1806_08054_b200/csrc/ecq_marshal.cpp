// Tensors to the pointers, strides and types of the C ABI, as binding.py does in Python: the same checks and
// messages, at a tenth of a microsecond for each tensor instead of 0.6 to 1.  A call on small matrices has up
// to nine of them and takes a few microseconds on the GPU.
#include <Python.h>

#include <cstdint>

#include <ATen/detail/CUDAHooksInterface.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

struct Matrix {                          // ecq_act8_matrix of ecq.h
    void* data;
    uint64_t stride;
    void* scales;
    int32_t dtype, pad;
};

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// The tensor of a matrix, and of a pair its scales.
bool parts(PyObject* m, const at::Tensor*& q, const at::Tensor*& scales, bool& pair) {
    pair = PyTuple_CheckExact(m) || PyList_CheckExact(m);
    scales = nullptr;
    if (!pair) return (q = tensor(m)) != nullptr;
    if (PySequence_Fast_GET_SIZE(m) != 2) return false;
    q = tensor(PySequence_Fast_GET_ITEM(m, 0));
    scales = tensor(PySequence_Fast_GET_ITEM(m, 1));
    return q && scales;
}

PyObject* refuse(const char* format, PyObject* name) {
    PyErr_Format(PyExc_ValueError, format, name);
    return nullptr;
}

// matrix(m, name, rows, cols, device): the bytes of an ecq_act8_matrix, or None for None
PyObject* matrix(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "matrix takes five arguments");
        return nullptr;
    }
    if (args[0] == Py_None) Py_RETURN_NONE;
    const long long rows = PyLong_AsLongLong(args[2]), cols = PyLong_AsLongLong(args[3]), device = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *q, *scales;
    bool pair;
    if (!parts(args[0], q, scales, pair)) return refuse("%U must be float32, bfloat16 or float16, or a pair (q, scales)", args[1]);
    Matrix out = {};
    const at::ScalarType type = q->scalar_type();
    if (pair) {
        out.dtype = type == at::kFloat8_e4m3fn ? 3 : type == at::kFloat8_e5m2 ? 4 : -1;
        if (out.dtype < 0 || scales->scalar_type() != at::kByte || !scales->is_contiguous() || scales->get_device() != device ||
            scales->numel() < ((rows + 127) >> 7) * ((cols + 511) >> 9) * 512)
            return refuse("%U must be (float8_e4m3fn or float8_e5m2, uint8 scales of ecq_act8_scale_bytes), both on the current CUDA "
                          "device", args[1]);
        out.scales = scales->data_ptr();
    } else {
        out.dtype = type == at::kFloat ? 0 : type == at::kBFloat16 ? 1 : type == at::kHalf ? 2 : -1;
        if (out.dtype < 0) return refuse("%U must be float32, bfloat16 or float16, or a pair (q, scales)", args[1]);
    }
    if (q->get_device() != device) return refuse("%U must be on the current CUDA device (there is no CPU path)", args[1]);
    if (q->dim() != 2 || q->size(0) != rows || q->size(1) != cols) {
        PyErr_Format(PyExc_ValueError, "%U must be %lld x %lld", args[1], rows, cols);
        return nullptr;
    }
    const int64_t stride = q->stride(0), step = q->stride(1);
    if ((step != 1 && cols > 1) || (stride < cols && rows > 1)) return refuse("%U must have contiguous rows that do not overlap", args[1]);
    out.data = q->data_ptr();
    out.stride = (uint64_t)(rows > 1 ? stride : (cols + 15) & ~15ll);
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&out), sizeof out);
}

// size(m, name): rows, columns and the current device
PyObject* size(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "size takes two arguments");
        return nullptr;
    }
    const at::Tensor *q, *scales;
    bool pair;
    if (!parts(args[0], q, scales, pair)) return refuse("%U must be a tensor or a pair (q, scales)", args[1]);
    if (!q->is_cuda()) return refuse("%U must be on the current CUDA device (there is no CPU path)", args[1]);
    if (q->dim() != 2) return refuse("%U must have two dimensions", args[1]);
    return Py_BuildValue("LLi", (long long)q->size(0), (long long)q->size(1), (int)at::detail::getCUDAHooks().getCurrentDevice());
}

// vector(t, dtype, n, name, device): its address, or None for None
PyObject* vector(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 5 || !THPDtype_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "vector takes a tensor, a type, a length, a name and a device");
        return nullptr;
    }
    if (args[0] == Py_None) Py_RETURN_NONE;
    const long long length = PyLong_AsLongLong(args[2]), device = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* t = tensor(args[0]);
    if (!t || t->scalar_type() != reinterpret_cast<THPDtype*>(args[1])->scalar_type || t->get_device() != device || t->numel() != length ||
        !t->is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%U must be %lld contiguous entries of %S on the current CUDA device", args[3], length, args[1]);
        return nullptr;
    }
    return PyLong_FromVoidPtr(t->data_ptr());
}

// What torch throws (a tensor without storage) comes back as an exception of Python.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    try {
        return F(self, args, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {
    {"matrix", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<matrix>)), METH_FASTCALL, nullptr},
    {"size", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<size>)), METH_FASTCALL, nullptr},
    {"vector", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<vector>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
