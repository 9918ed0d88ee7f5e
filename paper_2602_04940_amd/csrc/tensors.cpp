// Tables of tensors for the C ABI, for lists too long to be read from Python attribute by
// attribute (five calls of 40 ns each on hundreds of tensors: 200 us beside 40 us on the GPU).
// A module of one function, built next to the library; it holds no computation.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ts3.h"

namespace {

// The tensor at o as row fields; false with a Python exception set where it may not be one.
bool read_tensor(PyObject *o, const char *what, const void **data, int64_t *n, int32_t *dtype, int *device) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
        return false;
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    const auto type = t.scalar_type();
    if (!t.is_cuda() || !t.is_contiguous() || (type != at::kFloat && type != at::kBFloat16)) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous cuda float32 or bfloat16 tensor", what);
        return false;
    }
    *data = t.data_ptr();
    *n = t.numel();
    *dtype = type == at::kFloat ? TS3_FP32 : TS3_BF16;
    *device = t.device().index();
    return true;
}

// clip_table(grads, out or None) -> (ts3_clip_tensor rows as bytes, device index or -1)
PyObject *clip_table(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    if (nargs != 2) {
        PyErr_SetString(PyExc_TypeError, "clip_table(grads, out)");
        return nullptr;
    }
    PyObject *grads = PySequence_Fast(args[0], "gradients must be a sequence of tensors");
    if (!grads) return nullptr;
    PyObject *out = args[1] == Py_None ? nullptr : PySequence_Fast(args[1], "outputs must be a sequence of tensors");
    PyObject *rows = nullptr, *result = nullptr;
    int device = -1;
    try {
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(grads);
        if (out && PySequence_Fast_GET_SIZE(out) != count) {
            PyErr_Format(PyExc_ValueError, "%zd output tensors expected, not %zd", count, PySequence_Fast_GET_SIZE(out));
        } else if (args[1] == Py_None || out) {
            rows = PyBytes_FromStringAndSize(nullptr, count * (Py_ssize_t)sizeof(ts3_clip_tensor));
            ts3_clip_tensor *r = rows ? reinterpret_cast<ts3_clip_tensor *>(PyBytes_AS_STRING(rows)) : nullptr;
            bool ok = rows != nullptr;
            for (Py_ssize_t i = 0; ok && i < count; ++i) {
                int dev = 0;
                r[i].reserved = 0;
                ok = read_tensor(PySequence_Fast_GET_ITEM(grads, i), "a gradient", &r[i].src, &r[i].n, &r[i].dtype, &dev);
                if (!ok) break;
                if (i == 0) device = dev;
                r[i].dst = const_cast<void *>(r[i].src);
                bool same = dev == device;
                if (out) {
                    const void *dst = nullptr;
                    int64_t n = 0;
                    int32_t dtype = 0;
                    ok = read_tensor(PySequence_Fast_GET_ITEM(out, i), "an output", &dst, &n, &dtype, &dev);
                    if (!ok) break;
                    r[i].dst = const_cast<void *>(dst);
                    same = same && dev == device;
                    if (n != r[i].n || dtype != r[i].dtype) {
                        PyErr_SetString(PyExc_ValueError, "an output tensor must have its gradient's type and size");
                        ok = false;
                    }
                }
                if (ok && !same) {
                    PyErr_SetString(PyExc_ValueError, "gradients must be on one device");
                    ok = false;
                }
            }
            if (ok) result = Py_BuildValue("Oi", rows, device);
        }
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        result = nullptr;
    }
    Py_XDECREF(rows);
    Py_XDECREF(out);
    Py_DECREF(grads);
    return result;
}

PyMethodDef methods[] = {{"clip_table", (PyCFunction)(void (*)())clip_table, METH_FASTCALL, "Rows of ts3_clip_tensor."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&module); }
