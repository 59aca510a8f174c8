// Argument marshalling of the calls that a serving loop makes for every layer of every step.  Through
// ctypes and Python attribute look-ups a call of eight tensors costs 4 us for its checks and 1.7 us for
// its twenty arguments, more than its launch; here it costs a fraction of that.  The checks are the
// same: a tensor of another type, shape, device or layout is refused before anything is launched.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <tuple>
#include <type_traits>
#include <utility>

#include "chiron_kv.h"

namespace {

PyObject *attr_text(PyObject *t, const char *name)
{
    PyObject *a = PyObject_GetAttrString(t, name);
    PyObject *s = a ? PyObject_Str(a) : nullptr;
    Py_XDECREF(a);
    if (!s) {
        PyErr_Clear();
        s = PyUnicode_FromString("?");
    }
    return s;
}

// ValueError: `what` must be `wanted` of this shape on this device, and what the argument is instead.
PyObject *refuse(PyObject *t, PyObject *what, PyObject *wanted, long device, PyObject *const *shape, Py_ssize_t dims)
{
    if (!THPVariable_Check(t)) {
        PyErr_Format(PyExc_ValueError, "%S must be a tensor, got %R", what, t);
        return nullptr;
    }
    PyObject *want = PyTuple_New(dims);
    if (!want) return nullptr;
    for (Py_ssize_t i = 0; i < dims; ++i) {
        Py_INCREF(shape[i]);
        PyTuple_SET_ITEM(want, i, shape[i]);
    }
    PyObject *dtype = attr_text(t, "dtype"), *got = attr_text(t, "shape"), *where = attr_text(t, "device");
    PyObject *strides = PyObject_CallMethod(t, "stride", nullptr);
    if (!strides) PyErr_Clear();
    PyErr_Format(PyExc_ValueError, "%S must be %S of shape %S on cuda:%ld, got %S %S (strides %S) on %S", what, wanted, want,
                 device, dtype, got, strides ? strides : Py_None, where);
    Py_XDECREF(strides);
    Py_DECREF(want);
    Py_DECREF(dtype);
    Py_DECREF(got);
    Py_DECREF(where);
    return nullptr;
}

// Whether `test` holds of the tensor.  A sparse, nested or functional tensor throws when it is asked for strides or an
// address: it does not fit.
template <typename Test>
bool holds(const at::Tensor &v, Test test) noexcept
{
    try {
        return test(v);
    } catch (...) {
        return false;
    }
}

bool fits(const at::Tensor &v, long device, PyObject *const *shape, Py_ssize_t dims)
{
    if (!v.is_cuda() || v.get_device() != device || v.dim() != dims) return false;
    for (Py_ssize_t i = 0; i < dims; ++i)
        if (v.size(i) != PyLong_AsLongLong(shape[i])) return false;
    return true;
}

// on(device, tensor, dtype, what, *shape): the address of a contiguous tensor of this type and shape there.
PyObject *on(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n < 4) {
        PyErr_SetString(PyExc_TypeError, "on(device, tensor, dtype, what, *shape)");
        return nullptr;
    }
    const long device = PyLong_AsLong(args[0]);
    if (THPVariable_Check(args[1]) && THPDtype_Check(args[2])) {
        const at::ScalarType type = reinterpret_cast<THPDtype *>(args[2])->scalar_type;
        void *at = nullptr;
        if (holds(THPVariable_Unpack(args[1]), [&](const at::Tensor &v) {
                if (v.scalar_type() != type || !fits(v, device, args + 4, n - 4) || !v.is_contiguous()) return false;
                at = v.data_ptr();
                return true;
            }))
            return PyLong_FromVoidPtr(at);
    }
    if (PyErr_Occurred()) return nullptr;
    PyObject *wanted = PyUnicode_FromFormat("a contiguous %S tensor", args[2]);
    if (!wanted) return nullptr;
    refuse(args[1], args[3], wanted, device, args + 4, n - 4);
    Py_DECREF(wanted);
    return nullptr;
}

// rows_on(device, tensor, what, tokens, heads, d): (address, stride between tokens) of bf16 rows that are contiguous
// within a token.
PyObject *rows_on(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "rows_on(device, tensor, what, tokens, heads, d)");
        return nullptr;
    }
    const long device = PyLong_AsLong(args[0]);
    if (THPVariable_Check(args[1])) {
        void *at = nullptr;
        long long stride = 0;
        if (holds(THPVariable_Unpack(args[1]), [&](const at::Tensor &v) {
                if (v.scalar_type() != at::kBFloat16 || !fits(v, device, args + 3, 3) || v.stride(2) != 1 ||
                    (v.stride(1) != v.size(2) && v.size(1) != 1))
                    return false;
                at = v.data_ptr();
                stride = v.stride(0);
                return true;
            }))
            return Py_BuildValue("(NL)", PyLong_FromVoidPtr(at), stride);
    }
    if (PyErr_Occurred()) return nullptr;
    PyObject *wanted = PyUnicode_FromString("bfloat16 rows, contiguous within a token,");
    if (!wanted) return nullptr;
    refuse(args[1], args[2], wanted, device, args + 3, 3);
    Py_DECREF(wanted);
    return nullptr;
}

// probs_on(device, tensor, dtype, what, batch, count, vocab): (address, stride between rows) of evenly spaced rows of
// probabilities.  The stride of a dimension of size 1 means nothing: one row a request lies as far from the next as
// the requests do.
PyObject *probs_on(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "probs_on(device, tensor, dtype, what, batch, count, vocab)");
        return nullptr;
    }
    const long device = PyLong_AsLong(args[0]);
    if (THPVariable_Check(args[1]) && THPDtype_Check(args[2])) {
        const at::ScalarType type = reinterpret_cast<THPDtype *>(args[2])->scalar_type;
        void *at = nullptr;
        long long stride = 0;
        if (holds(THPVariable_Unpack(args[1]), [&](const at::Tensor &v) {
                if (v.scalar_type() != type || !fits(v, device, args + 4, 3) || (v.stride(2) != 1 && v.size(2) != 1)) return false;
                stride = v.size(1) != 1 ? v.stride(1) : v.size(0) != 1 ? v.stride(0) : v.size(2);
                if (v.size(0) != 1 && v.size(1) > 1 && v.stride(0) != v.size(1) * stride) return false;
                at = v.data_ptr();
                return true;
            }))
            return Py_BuildValue("(NL)", PyLong_FromVoidPtr(at), stride);
    }
    if (PyErr_Occurred()) return nullptr;
    PyObject *wanted = PyUnicode_FromFormat("evenly spaced %S rows", args[2]);
    if (!wanted) return nullptr;
    refuse(args[1], args[3], wanted, device, args + 4, 3);
    Py_DECREF(wanted);
    return nullptr;
}

// A Python number as an argument of the C ABI: an address (None: NULL), an int32, an int64, a size or a float.
template <typename T>
T argument(PyObject *x)
{
    if constexpr (std::is_pointer_v<T>) return x == Py_None ? nullptr : static_cast<T>(PyLong_AsVoidPtr(x));
    else if constexpr (std::is_same_v<T, float>) return (float)PyFloat_AsDouble(x);
    else if constexpr (std::is_same_v<T, size_t>) return PyLong_AsSize_t(x);
    else {
        const long long v = PyLong_AsLongLong(x);
        if (v != (long long)(T)v) PyErr_SetString(PyExc_OverflowError, "an argument does not fit 32 bits");
        return (T)v;
    }
}

// One wrapper per function: its arguments in order, the status returned.  Other Python threads run meanwhile: with
// the launch queue full, a launch blocks until the GPU has caught up.
template <typename... P, size_t... I>
PyObject *call(int32_t (*fn)(P...), PyObject *const *args, std::index_sequence<I...>)
{
    const std::tuple<P...> values{argument<P>(args[I])...};
    if (PyErr_Occurred()) return nullptr;
    int32_t status;
    Py_BEGIN_ALLOW_THREADS
    status = std::apply(fn, values);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

template <typename... P>
PyObject *call(int32_t (*fn)(P...), PyObject *const *args, Py_ssize_t n, const char *name)
{
    if (n != (Py_ssize_t)sizeof...(P)) {
        PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, (Py_ssize_t)sizeof...(P), n);
        return nullptr;
    }
    return call(fn, args, std::index_sequence_for<P...>{});
}

#define CKV_WRAP(name) \
    PyObject *py_##name(PyObject *, PyObject *const *args, Py_ssize_t n) { return call(name, args, n, #name); }
CKV_WRAP(kv_append_rope)
CKV_WRAP(kv_index_update)
CKV_WRAP(kv_index_values)
CKV_WRAP(decode_select_pages)
CKV_WRAP(decode_attention_pages)
CKV_WRAP(decode_attention_sparse)
CKV_WRAP(draft_verify)
CKV_WRAP(kv8_append)
CKV_WRAP(kv8_gather)
CKV_WRAP(kv8_attention)
CKV_WRAP(decode_attention_window)
CKV_WRAP(kv_pages_assign)
CKV_WRAP(kv_pages_release)
CKV_WRAP(logits_process)

#define CKV_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"on", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(on)), METH_FASTCALL, "Address of a tensor after its checks."},
    {"rows_on", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows_on)), METH_FASTCALL, "Address and token stride of rows."},
    {"probs_on", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(probs_on)), METH_FASTCALL, "Address and row stride of probabilities."},
    CKV_METHOD(kv_append_rope), CKV_METHOD(kv_index_update), CKV_METHOD(kv_index_values), CKV_METHOD(decode_select_pages),
    CKV_METHOD(decode_attention_pages), CKV_METHOD(decode_attention_sparse), CKV_METHOD(draft_verify),
    CKV_METHOD(kv8_append), CKV_METHOD(kv8_gather), CKV_METHOD(kv8_attention), CKV_METHOD(decode_attention_window),
    CKV_METHOD(kv_pages_assign), CKV_METHOD(kv_pages_release), CKV_METHOD(logits_process),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of libchiron_kv.so.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
