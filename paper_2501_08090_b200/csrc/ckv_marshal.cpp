// Argument marshalling of the calls that a serving loop makes for every layer of every step.  Through
// ctypes and Python attribute look-ups a call of eight tensors costs 4 us for its checks and 1.7 us for
// its twenty arguments, more than its launch; here it costs a fraction of that.  The checks are the
// same: a tensor of another type, shape, device or layout is refused before anything is launched.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
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
CKV_WRAP(logits_process)

// The calls of a step whose state stays on the GPU take their tensors here: a method's dozen checks one by one through
// Python cost 1.3 us, a third of the call.  Arguments: handle, address of the configuration, device, then the method's own in order.
struct Step {
    ckv_pool *pool;
    const ckv_config *c;
    long device;
    PyObject *const *args;              // the method's own
    long long batch = 0;
    bool ok = true;                     // false: an exception is set

    Step(PyObject *const *all)
        : pool(argument<ckv_pool *>(all[0])), c(argument<const ckv_config *>(all[1])), device(PyLong_AsLong(all[2])), args(all + 3) {}

    // Not asked once an exception is set: the check may call into Python, and would throw.
    const at::Tensor *tensor(PyObject *t) const noexcept
    {
        if (!ok || t == Py_None || PyErr_Occurred()) return nullptr;
        try {
            return THPVariable_Check(t) ? &THPVariable_Unpack(t) : nullptr;
        } catch (...) {
            return nullptr;
        }
    }

    void refused(PyObject *t, const char *what, const char *wanted, std::initializer_list<long long> shape)
    {
        ok = false;
        if (PyErr_Occurred()) return;
        PyObject *sizes[5] = {}, *name = PyUnicode_FromString(what), *kind = PyUnicode_FromString(wanted);
        Py_ssize_t n = 0;
        for (long long x : shape) sizes[n++] = PyLong_FromLongLong(x);
        bool built = name && kind;
        for (Py_ssize_t i = 0; i < n; ++i) built = built && sizes[i];
        if (built) refuse(t, name, kind, device, sizes, n);
        for (Py_ssize_t i = 0; i < n; ++i) Py_XDECREF(sizes[i]);
        Py_XDECREF(name);
        Py_XDECREF(kind);
    }

    bool fits(const at::Tensor &v, std::initializer_list<long long> shape) const
    {
        if (!v.is_cuda() || v.get_device() != device || v.dim() != (long long)shape.size()) return false;
        int64_t i = 0;
        for (long long x : shape)
            if (v.size(i++) != x) return false;
        return true;
    }

    // The address of a contiguous tensor of this type and shape.
    template <typename T>
    T *on(PyObject *t, at::ScalarType type, const char *type_name, const char *what, std::initializer_list<long long> shape)
    {
        if (!ok) return nullptr;
        void *at = nullptr;
        const at::Tensor *v = tensor(t);
        if (v && holds(*v, [&](const at::Tensor &x) {
                if (x.scalar_type() != type || !fits(x, shape) || !x.is_contiguous()) return false;
                at = x.data_ptr();
                return true;
            }))
            return static_cast<T *>(at);
        refused(t, what, type_name, shape);
        return nullptr;
    }
    int32_t *ints(PyObject *t, const char *what, std::initializer_list<long long> shape)
    {
        return on<int32_t>(t, at::kInt, "a contiguous torch.int32 tensor", what, shape);
    }
    int32_t *ints_or_none(PyObject *t, const char *what, std::initializer_list<long long> shape) { return t == Py_None ? nullptr : ints(t, what, shape); }

    // bf16 rows that are contiguous within a token, and their stride.
    uint16_t *rows(PyObject *t, const char *what, long long tokens, long long heads, int64_t &stride)
    {
        if (!ok) return nullptr;
        void *at = nullptr;
        const at::Tensor *v = tensor(t);
        if (v && holds(*v, [&](const at::Tensor &x) {
                if (x.scalar_type() != at::kBFloat16 || !fits(x, {tokens, heads, c->head_dim}) || x.stride(2) != 1 ||
                    (x.stride(1) != x.size(2) && x.size(1) != 1))
                    return false;
                at = x.data_ptr();
                stride = x.stride(0);
                return true;
            }))
            return static_cast<uint16_t *>(at);
        refused(t, what, "bfloat16 rows, contiguous within a token,", {tokens, heads, c->head_dim});
        return nullptr;
    }

    // Elements of a tensor, or its size along a dimension; 0 of anything else, which its own check refuses.
    long long numel(PyObject *t) const
    {
        long long n = 0;
        const at::Tensor *v = tensor(t);
        if (v) holds(*v, [&](const at::Tensor &x) { n = x.numel(); return true; });
        return n;
    }
    long long size(PyObject *t, int64_t dim) const
    {
        long long n = 0;
        const at::Tensor *v = tensor(t);
        if (v) holds(*v, [&](const at::Tensor &x) { n = x.dim() > dim ? x.size(dim) : 0; return true; });
        return n;
    }

    int32_t *tables(PyObject *block_tables, PyObject *seq_lens, int32_t *&lens)
    {
        batch = numel(seq_lens);
        if (batch > 0x7fffffffll) PyErr_SetString(PyExc_OverflowError, "the batch does not fit 32 bits");
        lens = ints(seq_lens, "seq_lens", {batch});
        return ints(block_tables, "block_tables", {batch, c->max_pages_per_req});
    }

    template <typename Call>
    PyObject *run(Call call)
    {
        if (!ok || PyErr_Occurred()) return nullptr;
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    }
};

// block_tables, seq_lens, new_tokens, free_pages, free_count, lens_out, count_out, step_lens, new_start, slots, stream
PyObject *step_pages_assign(Step s)
{
    int32_t *lens, *tables = s.tables(s.args[0], s.args[1], lens);
    int32_t *amounts = s.ints(s.args[2], "new_tokens", {s.batch}), *free_pages = s.ints(s.args[3], "free_pages", {s.c->num_pages});
    int32_t *count = s.ints(s.args[4], "free_count", {1}), *lens_out = s.ints(s.args[5], "lens_out", {s.batch});
    int32_t *count_out = s.ints(s.args[6], "count_out", {1}), *step_lens = s.ints_or_none(s.args[7], "step_lens", {s.batch});
    int32_t *new_start = s.ints_or_none(s.args[8], "new_start", {s.batch + 1});
    const long long n_slots = s.numel(s.args[9]);
    int64_t *slots = s.args[9] == Py_None ? nullptr : s.on<int64_t>(s.args[9], at::kLong, "a contiguous torch.int64 tensor", "slots", {n_slots});
    void *stream = argument<void *>(s.args[10]);
    if (n_slots > 0x7fffffffll) PyErr_SetString(PyExc_OverflowError, "slots does not fit 32 bits");
    return s.run([&] {
        return kv_pages_assign(s.pool, (int32_t)s.batch, tables, lens, amounts, free_pages, count, lens_out, count_out, step_lens, new_start,
                               n_slots > 0 ? slots : nullptr, (int32_t)n_slots, stream);
    });
}

// block_tables, seq_lens, keep_lens, free_pages, free_count, lens_out, count_out, stream
PyObject *step_pages_release(Step s)
{
    int32_t *lens, *tables = s.tables(s.args[0], s.args[1], lens);
    int32_t *amounts = s.ints(s.args[2], "keep_lens", {s.batch}), *free_pages = s.ints(s.args[3], "free_pages", {s.c->num_pages});
    int32_t *count = s.ints(s.args[4], "free_count", {1}), *lens_out = s.ints(s.args[5], "lens_out", {s.batch});
    int32_t *count_out = s.ints(s.args[6], "count_out", {1});
    void *stream = argument<void *>(s.args[7]);
    return s.run([&] { return kv_pages_release(s.pool, (int32_t)s.batch, tables, lens, amounts, free_pages, count, lens_out, count_out, stream); });
}

// layer, block_tables, seq_lens, k_new, v_new, q, q_out, inv_freq, new_start, interleaved, scale, stream
PyObject *step_kv8_append(Step s)
{
    const int32_t layer = argument<int32_t>(s.args[0]);
    int32_t *lens, *tables = s.tables(s.args[1], s.args[2], lens);
    const long long tokens = s.size(s.args[3], 0), half = s.numel(s.args[7]);
    if ((s.args[5] == Py_None) != (s.args[6] == Py_None)) {
        PyErr_SetString(PyExc_ValueError, "q and q_out go together");
        return nullptr;
    }
    int64_t q_stride = 0, k_stride = 0, v_stride = 0, out_stride = 0;
    const bool queries = s.args[5] != Py_None;
    uint16_t *q = queries ? s.rows(s.args[5], "q", tokens, s.c->num_q_heads, q_stride) : nullptr;
    uint16_t *q_out = queries ? s.rows(s.args[6], "q_out", tokens, s.c->num_q_heads, out_stride) : nullptr;
    uint16_t *k = s.rows(s.args[3], "k_new", tokens, s.c->num_kv_heads, k_stride), *v = s.rows(s.args[4], "v_new", tokens, s.c->num_kv_heads, v_stride);
    float *inv_freq = s.args[7] == Py_None ? nullptr : s.on<float>(s.args[7], at::kFloat, "a contiguous torch.float32 tensor", "inv_freq", {half});
    int32_t *new_start = s.ints_or_none(s.args[8], "new_start", {s.batch + 1});
    const int interleaved = PyObject_IsTrue(s.args[9]);
    const float scale = argument<float>(s.args[10]);
    void *stream = argument<void *>(s.args[11]);
    if (tokens > 0x7fffffffll || half > 0x3fffffffll) PyErr_SetString(PyExc_OverflowError, "a size does not fit 32 bits");
    return s.run([&] {
        return kv8_append(s.pool, layer, (int32_t)s.batch, (int32_t)tokens, tables, lens, new_start, inv_freq, (int32_t)(2 * half), interleaved, scale,
                          q, q_stride, k, k_stride, v, v_stride, q_out, out_stride, stream);
    });
}

// layer, block_tables, seq_lens, k, v, start, stream
PyObject *step_kv8_gather(Step s)
{
    const int32_t layer = argument<int32_t>(s.args[0]);
    int32_t *lens, *tables = s.tables(s.args[1], s.args[2], lens);
    const long long tokens = s.size(s.args[3], 0);
    int64_t k_stride = 0, v_stride = 0;
    uint16_t *k = s.rows(s.args[3], "k", tokens, s.c->num_kv_heads, k_stride), *v = s.rows(s.args[4], "v", tokens, s.c->num_kv_heads, v_stride);
    int32_t *start = s.ints_or_none(s.args[5], "start", {s.batch + 1});
    void *stream = argument<void *>(s.args[6]);
    if (tokens > 0x7fffffffll) PyErr_SetString(PyExc_OverflowError, "a size does not fit 32 bits");
    return s.run([&] { return kv8_gather(s.pool, layer, (int32_t)s.batch, (int32_t)tokens, tables, lens, start, k, k_stride, v, v_stride, stream); });
}

// layer, block_tables, seq_lens, q, out, window, sink, stream
template <decltype(kv8_attention) *kCall>
PyObject *step_attention(Step s)
{
    const int32_t layer = argument<int32_t>(s.args[0]);
    int32_t *lens, *tables = s.tables(s.args[1], s.args[2], lens);
    const at::Tensor *given = s.tensor(s.args[3]);
    const bool one = given && holds(*given, [](const at::Tensor &x) { return x.dim() == 3; });   // [batch][Hq][d]
    const long long q_len = one ? 1 : s.size(s.args[3], 1), heads = s.c->num_q_heads, d = s.c->head_dim;
    constexpr const char *kType = "a contiguous torch.bfloat16 tensor";
    auto at = [&](PyObject *t, const char *what) {
        return one ? s.on<void>(t, at::kBFloat16, kType, what, {s.batch, heads, d}) : s.on<void>(t, at::kBFloat16, kType, what, {s.batch, q_len, heads, d});
    };
    void *q = at(s.args[3], "q"), *out = at(s.args[4], "out");
    const int32_t window = argument<int32_t>(s.args[5]), sink = argument<int32_t>(s.args[6]);
    void *stream = argument<void *>(s.args[7]);
    if (q_len > 0x7fffffffll) PyErr_SetString(PyExc_OverflowError, "a size does not fit 32 bits");
    return s.run([&] { return kCall(s.pool, layer, (int32_t)s.batch, (int32_t)q_len, tables, lens, q, out, window, sink, stream); });
}

template <PyObject *(*kStep)(Step), Py_ssize_t kOwn>
PyObject *step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 3 + kOwn) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, got %zd", 3 + kOwn, n);
        return nullptr;
    }
    const Step s(args);
    return PyErr_Occurred() ? nullptr : kStep(s);
}

#define CKV_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
#define CKV_STEP(name, fn, own) \
    {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(step<fn, own>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"on", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(on)), METH_FASTCALL, "Address of a tensor after its checks."},
    {"rows_on", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows_on)), METH_FASTCALL, "Address and token stride of rows."},
    {"probs_on", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(probs_on)), METH_FASTCALL, "Address and row stride of probabilities."},
    CKV_METHOD(kv_append_rope), CKV_METHOD(kv_index_update), CKV_METHOD(kv_index_values), CKV_METHOD(decode_select_pages),
    CKV_METHOD(decode_attention_pages), CKV_METHOD(decode_attention_sparse), CKV_METHOD(draft_verify),
    CKV_METHOD(logits_process),
    CKV_STEP("pages_assign", step_pages_assign, 11), CKV_STEP("pages_release", step_pages_release, 8), CKV_STEP("kv8_append", step_kv8_append, 12),
    CKV_STEP("kv8_gather", step_kv8_gather, 7), CKV_STEP("kv8_attention", step_attention<kv8_attention>, 8),
    CKV_STEP("decode_attention_window", step_attention<decode_attention_window>, 8),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of libchiron_kv.so.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
