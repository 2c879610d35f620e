// The checks that inner.py makes of every tensor it hands to the library, and the tensors it makes where several outputs are left out,
// compiled: in Python they cost as much as the rest of a small call.  A Python extension module over torch's C++ tensors; what is wrong is reported through a Python function (`refuse`) that
// puts the message together.  It reads the objects of one torch and one Python: `built_for` names them, and the package refuses others.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>

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

// The entry as Python calls it: a C++ exception (a tensor without strides or storage, say) becomes a RuntimeError here, memory that is not there torch's
// own error for it.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return F(args, n);
    } catch (const c10::OutOfMemoryError& e) {
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());  // (else the error of the lookup stands)
        Py_XDECREF(type);
        Py_XDECREF(torch);
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

// tokens(x or None, device, tokens, heads, head_dim, dtype, what) -> (address, token stride, head stride) of [tokens, heads, head_dim], or of
// [batch, seq, heads, head_dim] whose sequences lie one behind the other
PyObject* tokens(PyObject* const* args, Py_ssize_t n) {
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "tokens(x, device, tokens, heads, head_dim, dtype, what)");
        return nullptr;
    }
    if (args[0] == Py_None) return Py_BuildValue("Oii", Py_None, 0, 0);
    long long v[4];
    if (!integers(args + 1, 4, v)) return nullptr;
    if (THPVariable_Check(args[0])) {
        const at::Tensor& x = THPVariable_Unpack(args[0]);
        const int64_t dim = x.dim();
        if (x.get_device() == v[0] && x.is_cuda() && is_dtype(x, args[5]) && (dim == 3 || dim == 4) && x.size(dim - 2) == v[2] && x.size(dim - 1) == v[3] && (v[3] <= 1 || x.stride(dim - 1) == 1)) {
            const int64_t seq = x.size(dim - 3), batch = dim == 4 ? x.size(0) : 1;
            if (batch * seq == v[1] && (v[1] == 0 || batch == 1 || seq == 1 || x.stride(0) == seq * x.stride(1))) {
                const long long token = batch > 1 && seq == 1 ? x.stride(0) : x.stride(dim - 3);
                return Py_BuildValue("NLL", PyLong_FromVoidPtr(x.data_ptr()), token, (long long)x.stride(dim - 2));
            }
        }
    }
    return refused(args[6], args[0], PyUnicode_FromFormat("a CUDA tensor [%lld tokens, %lld, %lld] of %S on device %lld with a unit stride inside a head (or [batch, seq, ...], sequences one behind the other)",
                                                          v[1], v[2], v[3], args[5], v[0]));
}

// empties(device, dtype, rows, cols, dtype, rows, cols, ..) -> tuple of new tensors [rows, cols] on a CUDA device; cols < 0: [rows].  All of them lie in
// one piece of memory, which takes the allocator one visit (1 us each otherwise) and lives as long as any of them.
PyObject* empties(PyObject* const* args, Py_ssize_t n) {
    constexpr int kMost = 16;
    const int count = (int)(n / 3);
    if (n < 4 || n % 3 != 1 || count > kMost) {
        PyErr_SetString(PyExc_TypeError, "empties(device, dtype, rows, cols, ..), at most 16 tensors");
        return nullptr;
    }
    long long dev, v[kMost][2];
    int64_t at_byte[kMost], bytes = 0;
    at::ScalarType types[kMost];
    if (!integers(args, 1, &dev)) return nullptr;
    for (int i = 0; i < count; ++i) {
        PyObject* const* a = args + 1 + 3 * i;
        if (!THPDtype_Check(a[0])) {
            PyErr_SetString(PyExc_TypeError, "empties: a dtype, rows and cols for every tensor");
            return nullptr;
        }
        if (!integers(a + 1, 2, v[i])) return nullptr;
        types[i] = reinterpret_cast<THPDtype*>(a[0])->scalar_type;
        const int64_t most = (1ll << 50) / (int64_t)c10::elementSize(types[i]), across = v[i][1] < 0 ? 1 : v[i][1];  // (2^50 bytes a tensor: their sum stays within 64 bits)
        if (v[i][0] < 0 || (across > 0 && v[i][0] > most / across)) {
            PyErr_SetString(PyExc_ValueError, "empties: sizes out of range");
            return nullptr;
        }
        at_byte[i] = bytes;
        bytes += (v[i][0] * across * (int64_t)c10::elementSize(types[i]) + 255) / 256 * 256;
    }
    const at::Tensor all = at::empty({bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, (at::DeviceIndex)dev));
    PyObject* out = PyTuple_New(count);
    if (!out) return nullptr;
    for (int i = 0; i < count; ++i) {
        PyObject* t = nullptr;
        try {
            at::Tensor x = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(types[i]));
            c10::TensorImpl* impl = x.unsafeGetTensorImpl();
            impl->set_storage_offset(at_byte[i] / (int64_t)c10::elementSize(types[i]));
            if (v[i][1] < 0) impl->set_sizes_contiguous({v[i][0]});
            else impl->set_sizes_contiguous({v[i][0], v[i][1]});
            t = THPVariable_Wrap(x);
        } catch (...) {
            Py_DECREF(out);
            throw;  // (into entry())
        }
        if (!t) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i, t);
    }
    return out;
}

PyObject* set_refuse(PyObject*, PyObject* f) {
    Py_XINCREF(f);
    Py_XSETREF(g_refuse, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"ptr", (PyCFunction)(void (*)(void))entry<ptr>, METH_FASTCALL, nullptr},
                         {"rows", (PyCFunction)(void (*)(void))entry<rows>, METH_FASTCALL, nullptr},
                         {"heads", (PyCFunction)(void (*)(void))entry<heads>, METH_FASTCALL, nullptr},
                         {"tokens", (PyCFunction)(void (*)(void))entry<tokens>, METH_FASTCALL, nullptr},
                         {"empties", (PyCFunction)(void (*)(void))entry<empties>, METH_FASTCALL, nullptr},
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
