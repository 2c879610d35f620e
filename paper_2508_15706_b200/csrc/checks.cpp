// The checks that inner.py makes of every tensor it hands to the library, compiled: in Python they cost as much as the rest of a
// small call.  A Python extension module over torch's C++ tensors; what is wrong is reported through a Python function (`refuse`) that
// puts the message together.  It reads the objects of one torch and one Python: `built_for` names them, and the package refuses others.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>

namespace {

PyObject* g_refuse = nullptr;

// refuse(what, tensor, wanted) raises; the null that a failing call returns is passed on.  `wanted` is owned here.
PyObject* refused(PyObject* what, PyObject* tensor, PyObject* wanted) {
    if (!wanted) return nullptr;
    PyObject* r = g_refuse ? PyObject_CallFunctionObjArgs(g_refuse, what, tensor, wanted, nullptr) : nullptr;
    Py_DECREF(wanted);
    if (r || !g_refuse) {
        Py_XDECREF(r);
        PyErr_SetString(PyExc_RuntimeError, "set_refuse takes a function that raises");
    }
    return nullptr;
}

bool is_dtype(const at::Tensor& x, PyObject* dtype) { return THPDtype_Check(dtype) && reinterpret_cast<THPDtype*>(dtype)->scalar_type == x.scalar_type(); }

// The entry as Python calls it: a C++ exception (a tensor without strides or storage, say) becomes a RuntimeError here.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return F(args, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

bool integers(PyObject* const* args, int n, long long* out) {
    for (int i = 0; i < n; ++i) {
        out[i] = PyLong_AsLongLong(args[i]);
        if (out[i] == -1 && PyErr_Occurred()) return false;
    }
    return true;
}

// ptr(tensor or None, device, numel, dtype, what) -> address or None
PyObject* ptr(PyObject* const* args, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "ptr(tensor, device, numel, dtype, what)");
        return nullptr;
    }
    if (args[0] == Py_None) Py_RETURN_NONE;
    long long v[2];
    if (!integers(args + 1, 2, v)) return nullptr;
    if (THPVariable_Check(args[0])) {
        const at::Tensor& x = THPVariable_Unpack(args[0]);
        if (x.get_device() == v[0] && x.is_cuda() && is_dtype(x, args[3]) && x.is_contiguous() && x.numel() >= v[1]) return PyLong_FromVoidPtr(x.data_ptr());
    }
    return refused(args[4], args[0], PyUnicode_FromFormat("a contiguous CUDA tensor of %S on device %lld with at least %lld elements", args[3], v[0], v[1]));
}

PyObject* address_and(void* p, long long ld) {
    PyObject* address = PyLong_FromVoidPtr(p);
    PyObject* stride = PyLong_FromLongLong(ld);
    PyObject* both = address && stride ? PyTuple_New(2) : nullptr;
    if (!both) {
        Py_XDECREF(address);
        Py_XDECREF(stride);
        return nullptr;
    }
    PyTuple_SET_ITEM(both, 0, address);
    PyTuple_SET_ITEM(both, 1, stride);
    return both;
}

// rows(matrix or None, device, rows, cols, dtype, what) -> (address, row stride)
PyObject* rows(PyObject* const* args, Py_ssize_t n) {
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "rows(tensor, device, rows, cols, dtype, what)");
        return nullptr;
    }
    if (args[0] == Py_None) return Py_BuildValue("Oi", Py_None, 0);
    long long v[3];
    if (!integers(args + 1, 3, v)) return nullptr;
    if (THPVariable_Check(args[0])) {
        const at::Tensor& x = THPVariable_Unpack(args[0]);
        if (x.get_device() == v[0] && x.is_cuda() && is_dtype(x, args[4]) && x.dim() == 2 && x.size(0) == v[1] && x.size(1) == v[2] && (v[2] == 1 || x.stride(1) == 1) &&
            (v[1] <= 1 || x.stride(0) >= v[2]))
            return address_and(x.data_ptr(), v[1] > 1 ? x.stride(0) : v[2]);
    }
    return refused(args[5], args[0], PyUnicode_FromFormat("a CUDA tensor [%lld, %lld] of %S on device %lld with unit column stride and rows apart", v[1], v[2], args[4], v[0]));
}

// heads(x, out, device, batch, seq, head_dim, dtype, what) -> the bytes of a sl_rotary_heads
PyObject* heads(PyObject* const* args, Py_ssize_t n) {
    if (n != 8) {
        PyErr_SetString(PyExc_TypeError, "heads(x, out, device, batch, seq, head_dim, dtype, what)");
        return nullptr;
    }
    long long v[4];
    if (!integers(args + 2, 4, v)) return nullptr;
    struct {
        const void* in;
        const void* out;
        int64_t heads, stride[6];  // batch, token, head of the input, then of the output
    } h;
    for (int k = 0; k < 2; ++k) {
        bool fits = false;
        if (THPVariable_Check(args[k])) {
            const at::Tensor& x = THPVariable_Unpack(args[k]);
            fits = x.get_device() == v[0] && x.is_cuda() && is_dtype(x, args[6]) && x.dim() == 4 && x.size(0) == v[1] && x.size(1) == v[2] && x.size(3) == v[3] &&
                   (v[3] <= 1 || x.stride(3) == 1) && (k == 0 || x.size(2) == h.heads);
            if (fits) {
                (k ? h.out : h.in) = x.data_ptr();
                h.heads = x.size(2);
                for (int d = 0; d < 3; ++d) h.stride[3 * k + d] = x.stride(d);
            }
        }
        if (!fits)
            return refused(args[7], args[k], PyUnicode_FromFormat("a CUDA tensor [%lld, %lld, heads, %lld] of %S on device %lld with a unit stride inside a head, an output with the heads of its input",
                                                                  v[1], v[2], v[3], args[6], v[0]));
    }
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&h), sizeof(h));
}

PyObject* set_refuse(PyObject*, PyObject* f) {
    Py_XINCREF(f);
    Py_XSETREF(g_refuse, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"ptr", (PyCFunction)(void (*)(void))entry<ptr>, METH_FASTCALL, nullptr},
                         {"rows", (PyCFunction)(void (*)(void))entry<rows>, METH_FASTCALL, nullptr},
                         {"heads", (PyCFunction)(void (*)(void))entry<heads>, METH_FASTCALL, nullptr},
                         {"set_refuse", set_refuse, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_checks", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef BUILT_FOR
#error "BUILT_FOR names the torch and the Python that this is compiled for"
#endif

extern "C" PyObject* PyInit__checks() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
