// The library's entries and the checks of their tensors as functions of a Python module, for calls whose kernels take less time than
// their arguments' way through ctypes (18 arguments: 2 us there, 0.2 here).
//
// An entry takes its C arguments in order: an int or None for a pointer, an int for a number, a float, and for a description
// (dst_fp8_t and its like, or an array of dst_tensor_t) whatever exposes its memory, a ctypes structure, or None.  It returns the status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include "dst_step.h"

namespace {

// a Python argument as a C argument of type T; `bad` where it is none (a Python error is set)
template <typename T> struct Arg {                           // integers and floating point
    T value{};
    bool bad = false;
    explicit Arg(PyObject* o) {
        if (PyErr_Occurred()) { bad = true; return; }        // (another argument's)
        if constexpr (std::is_floating_point_v<T>) {
            const double v = PyFloat_AsDouble(o);
            bad = v == -1. && PyErr_Occurred();
            value = static_cast<T>(v);
        } else if constexpr (std::is_unsigned_v<T>) {
            const unsigned long long v = PyLong_AsUnsignedLongLong(o);
            bad = v == ~0ull && PyErr_Occurred();
            value = static_cast<T>(v);
        } else {
            const long long v = PyLong_AsLongLong(o);
            bad = v == -1 && PyErr_Occurred();
            if (!bad && (v < std::numeric_limits<T>::min() || v > std::numeric_limits<T>::max())) {
                PyErr_SetString(PyExc_OverflowError, "argument does not fit 32 bits");
                bad = true;
            }
            value = static_cast<T>(v);
        }
    }
};
template <typename T> constexpr bool kDescription = std::is_same_v<T, dst_fp8_t> || std::is_same_v<T, dst_fp4_t> || std::is_same_v<T, dst_tensor_t> || std::is_same_v<T, dst_dropout_t>;
template <typename T> struct Arg<T*> {                       // addresses
    T* value = nullptr;
    bool bad = false;
    Py_buffer view{};
    explicit Arg(PyObject* o) {
        if (PyErr_Occurred()) { bad = true; return; }
        if (o == Py_None) return;
        if constexpr (kDescription<std::remove_const_t<T>>) {
            if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) { bad = true; return; }
            constexpr bool list = std::is_same_v<std::remove_const_t<T>, dst_tensor_t>;
            if (list ? view.len % sizeof(T) != 0 : view.len != (Py_ssize_t)sizeof(T)) {
                PyErr_SetString(PyExc_TypeError, "a description of another kind");
                bad = true;
            }
            value = static_cast<T*>(view.buf);
        } else {
            value = static_cast<T*>(PyLong_AsVoidPtr(o));
            bad = !value && PyErr_Occurred();
        }
    }
    Arg(const Arg&) = delete;
    ~Arg() { if (view.obj) PyBuffer_Release(&view); }
};

template <auto F> struct Entry;
template <typename... A, int (*F)(A...)> struct Entry<F> {
    template <size_t... I> static PyObject* run(PyObject* const* given, std::index_sequence<I...>) {
        std::tuple<Arg<A>...> args(given[I]...);
        if ((std::get<I>(args).bad || ...)) return nullptr;
        int status;
        Py_BEGIN_ALLOW_THREADS
        status = F(std::get<I>(args).value...);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    }
    static PyObject* call(PyObject*, PyObject* const* given, Py_ssize_t n) {
        if (n != (Py_ssize_t)sizeof...(A)) return PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", (Py_ssize_t)sizeof...(A), n);
        return run(given, std::index_sequence_for<A...>{});
    }
};

// ---- tensors ----------------------------------------------------------------------
int type_of(const at::Tensor& t) {
    return t.scalar_type() == at::kFloat ? DST_F32 : t.scalar_type() == at::kBFloat16 ? DST_BF16 : -1;
}
PyObject* dtype_name(PyObject* tensor) { return PyObject_GetAttrString(tensor, "dtype"); }
bool number(PyObject* o, long long& v) { v = PyLong_AsLongLong(o); return !(v == -1 && PyErr_Occurred()); }

PyObject* not_a(PyObject* tensor, PyObject* name, const char* what) {
    if (PyObject* d = dtype_name(tensor)) { PyErr_Format(PyExc_TypeError, "%U must be %s, got %S", name, what, d); Py_DECREF(d); }
    return nullptr;
}
const at::Tensor* tensor_of(PyObject* o, PyObject* name) {
    if (!PyUnicode_Check(name)) { PyErr_SetString(PyExc_TypeError, "a name must be a string"); return nullptr; }
    if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "%U must be a tensor, got %s", name, Py_TYPE(o)->tp_name); return nullptr; }
    return &THPVariable_Unpack(o);
}
bool elsewhere(const at::Tensor& t, long long device) {
    if (t.get_device() == device) return false;
    PyErr_SetString(PyExc_ValueError, "all tensors must live on the same device");
    return true;
}

// matrix(tensor, rows, cols, device, name): (pointer, leading dimension, type) of a [rows, cols] matrix with contiguous rows
PyObject* matrix(PyObject*, PyObject* const* a, Py_ssize_t n) {
    long long rows, cols, device;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments, not %zd", n);
    if (!number(a[1], rows) || !number(a[2], cols) || !number(a[3], device)) return nullptr;
    const at::Tensor* const t = tensor_of(a[0], a[4]);
    if (!t) return nullptr;
    try {
        const int type = type_of(*t);
        if (type < 0) return not_a(a[0], a[4], "float32 or bfloat16");
        if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) {
            if (PyObject* s = PyObject_GetAttrString(a[0], "shape")) { PyErr_Format(PyExc_ValueError, "%U must be [%lld, %lld], got %S", a[4], rows, cols, s); Py_DECREF(s); }
            return nullptr;
        }
        if (elsewhere(*t, device)) return nullptr;
        long long ld = t->stride(0);
        const long long step = t->stride(1);
        if ((step != 1 && cols > 1) || ld < cols) {           // (the stride of a single column means nothing)
            if (rows > 1 || (step != 1 && cols > 1)) return PyErr_Format(PyExc_ValueError, "%U must have contiguous rows that do not overlap", a[4]);
            ld = cols;
        }
        PyObject* const out = PyTuple_New(3);
        if (!out) return nullptr;
        PyTuple_SET_ITEM(out, 0, PyLong_FromVoidPtr(t->data_ptr()));
        PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(ld));
        PyTuple_SET_ITEM(out, 2, PyLong_FromLong(type));
        return out;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// a tensor of a type; a new error otherwise
const at::Tensor* typed(PyObject* o, PyObject* dtype, PyObject* name) {
    const at::Tensor* const t = tensor_of(o, name);
    if (!t) return nullptr;
    PyObject* const is = dtype_name(o);                      // (one object for each type)
    if (!is) return nullptr;
    Py_DECREF(is);
    if (is == dtype) return t;
    PyErr_Format(PyExc_TypeError, "%U must be %S, got %S", name, dtype, is);
    return nullptr;
}

// vector(tensor or None, n, dtype, device, name): pointer of n contiguous elements, or None
PyObject* vector(PyObject*, PyObject* const* a, Py_ssize_t n) {
    long long elements, device;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments, not %zd", n);
    if (a[0] == Py_None) Py_RETURN_NONE;
    if (!number(a[1], elements) || !number(a[3], device)) return nullptr;
    try {
        const at::Tensor* const t = typed(a[0], a[2], a[4]);
        if (!t) return nullptr;
        if (t->dim() != 1 || t->size(0) != elements || !t->is_contiguous()) return PyErr_Format(PyExc_ValueError, "%U must be contiguous [%lld]", a[4], elements);
        return elsewhere(*t, device) ? nullptr : PyLong_FromVoidPtr(t->data_ptr());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// table(tensor, rows, dtype, device, name): (pointer, columns) of a contiguous matrix
PyObject* table(PyObject*, PyObject* const* a, Py_ssize_t n) {
    long long rows, device;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments, not %zd", n);
    if (!number(a[1], rows) || !number(a[3], device)) return nullptr;
    try {
        const at::Tensor* const t = typed(a[0], a[2], a[4]);
        if (!t) return nullptr;
        if (t->dim() != 2 || t->size(0) != rows || !t->is_contiguous()) return PyErr_Format(PyExc_ValueError, "%U must be contiguous [%lld, n]", a[4], rows);
        return elsewhere(*t, device) ? nullptr : Py_BuildValue("(NL)", PyLong_FromVoidPtr(t->data_ptr()), (long long)t->size(1));
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define DST_ENTRY(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(Entry<NAME>::call)), METH_FASTCALL, nullptr}
#define DST_CHECK(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    DST_CHECK(matrix), DST_CHECK(vector), DST_CHECK(table),
    DST_ENTRY(dst_dropout), DST_ENTRY(dst_embed), DST_ENTRY(dst_quantize_fp8), DST_ENTRY(dst_matmul_fp8), DST_ENTRY(dst_linear_fp8),
    DST_ENTRY(dst_quantize_fp4), DST_ENTRY(dst_matmul_fp4), DST_ENTRY(dst_linear_fp4), DST_ENTRY(dst_sample),
    DST_ENTRY(dst_logprob), DST_ENTRY(dst_logprob_loss), DST_ENTRY(dst_logprob_backward), DST_ENTRY(dst_rmsnorm), DST_ENTRY(dst_rmsnorm_backward),
    DST_ENTRY(dst_grad_norm), DST_ENTRY(dst_clip),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Entries of libdst_b200.so and the checks of their tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
