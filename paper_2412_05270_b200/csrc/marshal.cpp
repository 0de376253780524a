// What the binding asks of tensors, in one call each: an attribute of a tensor costs 50 to 200 ns from Python, and a call on small tensors
// asks for dozens (65 vectors of an AdamW step: 80 us; through pack(): 3 us).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

namespace {

// (the exact types first: asking whether an object is an instance costs 50 ns)
bool is_tensor(PyObject* x) { return THPVariable_CheckTypeExact(Py_TYPE(x)) || THPVariable_Check(x); }

int type_code(const at::Tensor& t)
{
    switch (t.scalar_type()) {
        case at::kFloat: return 0;
        case at::kBFloat16: return 1;
        case at::kInt: return 2;
        case at::kLong: return 3;
        case at::kByte: return 4;
        default: return -1;
    }
}

long device_index(const at::Tensor& t) { return t.is_cuda() ? (long)t.get_device() : -1L; }

// (address, device index or -1, type code, dimensions, sizes and strides of the first two, contiguous)
PyObject* describe(PyObject*, PyObject* arg)
{
    if (!is_tensor(arg)) {
        PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
        return nullptr;
    }
    try {
        const at::Tensor& t = THPVariable_Unpack(arg);
        if (t.layout() != at::kStrided) {
            PyErr_SetString(PyExc_ValueError, "a strided tensor is wanted");
            return nullptr;
        }
        const auto size = t.sizes();
        const auto stride = t.strides();
        const long n = (long)size.size();
        return Py_BuildValue("Klillllli", (unsigned long long)(uintptr_t)t.data_ptr(), device_index(t), type_code(t), n, n > 0 ? (long)size[0] : 1L,
                             n > 1 ? (long)size[1] : 1L, n > 0 ? (long)stride[0] : 1L, n > 1 ? (long)stride[1] : 1L, (int)t.is_contiguous());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
}

PyObject* refuse(const char* what, const char* why)
{
    PyErr_SetString(PyExc_ValueError, (std::string(what) + " " + why).c_str());
    return nullptr;
}

// Whether a tensor, or a tuple of whole numbers, has these sizes.
bool same_shape(PyObject* other, at::IntArrayRef sizes)
{
    if (!PyTuple_Check(other)) return is_tensor(other) && THPVariable_Unpack(other).sizes().equals(sizes);
    if ((size_t)PyTuple_GET_SIZE(other) != sizes.size()) return false;
    for (size_t i = 0; i < sizes.size(); ++i) {
        const long long n = PyLong_AsLongLong(PyTuple_GET_ITEM(other, (Py_ssize_t)i));
        if (n != (long long)sizes[i]) {
            PyErr_Clear();
            return false;
        }
    }
    return true;
}

// pack(what, tensors, like, device): addresses (uint64), lengths (int64) and types (int32, 0 = float32, 1 = bfloat16) of a list of contiguous
// CUDA tensors as bytes, their device and how many there are.  None: address 0.  like: a list of the shapes (tuples) or tensors whose shapes they must
// have, or None; device: the index they must be on, or -1.
PyObject* pack(PyObject*, PyObject* args)
{
    const char* what;
    PyObject *tensors, *like;
    long device;
    if (!PyArg_ParseTuple(args, "sOOl", &what, &tensors, &like, &device)) return nullptr;
    PyObject* list = PySequence_Fast(tensors, "a list of tensors is wanted");
    if (!list) return nullptr;
    PyObject* shapes = like == Py_None ? nullptr : PySequence_Fast(like, "a list of tensors is wanted");
    if (like != Py_None && !shapes) {
        Py_DECREF(list);
        return nullptr;
    }
    PyObject* result = nullptr;
    try {
        result = [&]() -> PyObject* {
            const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
            if (shapes && PySequence_Fast_GET_SIZE(shapes) != n) return refuse(what, "must be as many as there are parameters");
            std::vector<uint64_t> address((size_t)n, 0);
            std::vector<int64_t> length((size_t)n, 0);
            std::vector<int32_t> type((size_t)n, 0);
            long live = 0;
            for (Py_ssize_t i = 0; i < n; ++i) {
                PyObject* item = PySequence_Fast_GET_ITEM(list, i);
                if (item == Py_None) continue;
                if (!is_tensor(item)) return refuse(what, "must be tensors");
                const at::Tensor& t = THPVariable_Unpack(item);
                if (!t.is_cuda() || t.layout() != at::kStrided || !t.is_contiguous()) return refuse(what, "must be contiguous CUDA tensors");
                const int code = type_code(t);
                if (code != 0 && code != 1) return refuse(what, "must be bfloat16 or float32");
                if (device < 0) device = device_index(t);
                if (device_index(t) != device) return refuse("the tensors of a call, out and workspace among them,", "must be on one device");
                if (shapes) {
                    PyObject* other = PySequence_Fast_GET_ITEM(shapes, i);
                    if (!same_shape(other, t.sizes())) return refuse(what, "must have their parameters' shapes");
                }
                address[(size_t)i] = (uint64_t)(uintptr_t)t.data_ptr();
                length[(size_t)i] = t.numel();
                type[(size_t)i] = code;
                ++live;
            }
            return Py_BuildValue("y#y#y#ll", (const char*)address.data(), (Py_ssize_t)(n * 8), (const char*)length.data(), (Py_ssize_t)(n * 8),
                                 (const char*)type.data(), (Py_ssize_t)(n * 4), device, live);
        }();
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    }
    Py_XDECREF(shapes);
    Py_DECREF(list);
    return result;
}

// changed(tensors, where): tells autograd that a call has written to them, so that a saved one is not used for a gradient; where: a list of as many
// (tensors whose place in it is None were left alone), or None.  A None among the tensors is left out.
PyObject* changed(PyObject*, PyObject* args)
{
    PyObject *tensors, *where;
    if (!PyArg_ParseTuple(args, "OO", &tensors, &where)) return nullptr;
    PyObject* list = PySequence_Fast(tensors, "a list of tensors is wanted");
    if (!list) return nullptr;
    PyObject* written = where == Py_None ? nullptr : PySequence_Fast(where, "a list is wanted");
    if (where != Py_None && !written) {
        Py_DECREF(list);
        return nullptr;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* item = PySequence_Fast_GET_ITEM(list, i);
        if (!is_tensor(item)) continue;
        if (written && (i >= PySequence_Fast_GET_SIZE(written) || PySequence_Fast_GET_ITEM(written, i) == Py_None)) continue;
        const at::Tensor& t = THPVariable_Unpack(item);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
    Py_XDECREF(written);
    Py_DECREF(list);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    { "describe", describe, METH_O, "(address, device index or -1, type code, dimensions, size 0, size 1, stride 0, stride 1, contiguous)" },
    { "pack", pack, METH_VARARGS, "(addresses, lengths, types, device, tensors that are not None)" },
    { "changed", changed, METH_VARARGS, "autograd is told that the tensors (those whose place in the second list is not None) were written" },
    { nullptr, nullptr, 0, nullptr },
};

PyModuleDef module = { PyModuleDef_HEAD_INIT, "_marshal", "What the binding asks of tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr };

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
