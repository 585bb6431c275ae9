// Argument marshalling of the serving step's entry points (skv_rope_append, skv_plan_step, skv_plan_release,
// skv_decode_attn_window, skv_prefill_attn_window) as a CPython extension: reads the tensors' types, shapes, devices and
// pointers directly and calls the C entry point, whose address binding.py hands over.  These calls run for a few
// microseconds on the GPU, and asking the same of the tensors from Python, then passing 15 to 20 arguments through ctypes, takes 7
// to 9 on the host.
// A function returns the entry point's status, or None where anything is not as the plain case has it (another type, shape
// or device, a stream of the caller's, an integer out of range, a handle that is closed), or where asking throws (a tensor
// without memory, no device): binding.py then goes through its own checks, which say what is wrong or make the call.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "../../include/skv.h"

namespace {

decltype(&skv_is_owner) is_owner;
decltype(&skv_rope_append) rope_append_entry;
decltype(&skv_plan_step) plan_step_entry;
decltype(&skv_plan_release) plan_release_entry;
decltype(&skv_decode_attn_window) decode_window_entry;
decltype(&skv_prefill_attn_window) prefill_window_entry;

// The arguments of one call, in order; `ok` turns false at the first that is not plain.
struct Args {
    PyObject *const *a;
    Py_ssize_t n;
    Py_ssize_t i = 0;
    bool ok = true;
    int device = -1;
    skv_cache *cache = nullptr;
    void *stream = nullptr;

    PyObject *next() { return i < n ? a[i++] : (ok = false, Py_None); }
    void *handle()
    {
        PyObject *o = next();
        if (!PyLong_CheckExact(o)) return ok = false, nullptr;
        void *p = PyLong_AsVoidPtr(o);
        if (!p) PyErr_Clear(), ok = false;
        return p;
    }
    int integer()
    {
        PyObject *o = next();
        int overflow = 0;
        const long v = PyLong_CheckExact(o) ? PyLong_AsLongAndOverflow(o, &overflow) : (ok = false, 0);
        if (overflow || v != (long)(int)v) ok = false;
        return (int)v;
    }
    float real()
    {
        PyObject *o = next();
        if (!PyFloat_CheckExact(o)) return ok = false, 0.f;
        return (float)PyFloat_AS_DOUBLE(o);
    }
    const at::Tensor *tensor(at::ScalarType type)
    {
        PyObject *o = next();
        if (!THPVariable_Check(o)) return ok = false, nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != device) ok = false;
        return &t;
    }
    // (after a refusal the checks go on, so that no caller reads through a null pointer)
    const at::Tensor *dense(at::ScalarType type, int dims)
    {
        const at::Tensor *t = tensor(type);
        if (t && (t->dim() != dims || !t->is_contiguous())) ok = false;
        for (int64_t size : ok ? t->sizes() : at::IntArrayRef())
            if (type != at::kByte && size > 0x7FFFFFFF) ok = false;
        return ok ? t : nullptr;
    }
    // cache handle and pool: the pool's device has to be the current one, and gives the stream
    void begin()
    {
        cache = static_cast<skv_cache *>(handle());
        PyObject *pool = next();
        if (!ok || !THPVariable_Check(pool)) {
            ok = false;
            return;
        }
        device = THPVariable_Unpack(pool).get_device();
        if (device < 0 || device != c10::cuda::current_device()) ok = false;
        else stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    }
    bool end()                         // the last argument: the caller's stream
    {
        return next() == Py_None && ok && i == n;
    }
};

// The entry point's status; its arguments are all evaluated before the interpreter is let go, since looking at a tensor may throw.
template <class Entry, class... A>
PyObject *status_of(Entry entry, A... args)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(args...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// A method as Python calls it: no C++ exception may pass through its frames.
template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *declining(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    try {
        return F(self, a, n);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

template <class T>
T *ptr(const at::Tensor *t) { return static_cast<T *>(t->data_ptr()); }

// (cache, pool, head_dim, layer, Q, page_table, seq_lens, out, workspace, window, sinks, scale, stream)
PyObject *decode_attn_window(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Args x{a, n};
    x.begin();
    const int head_dim = x.integer(), layer = x.integer();
    const at::Tensor *q = x.dense(at::kBFloat16, 3), *table = x.dense(at::kInt, 2), *lens = x.dense(at::kInt, 1), *out = x.dense(at::kBFloat16, 3),
                     *work = x.dense(at::kByte, 1);
    const int window = x.integer(), sinks = x.integer();
    const float scale = x.real();
    if (!x.end() || q->size(2) != head_dim || out->sizes() != q->sizes() || table->size(0) != q->size(0) || lens->size(0) != q->size(0)) Py_RETURN_NONE;
    const int batch = (int)q->size(0), heads = (int)q->size(1), width = (int)table->size(1);
    return status_of(decode_window_entry, x.cache, layer, ptr<void>(q), ptr<int32_t>(table), ptr<int32_t>(lens), ptr<void>(out), batch, heads, width, window,
                     sinks, scale, ptr<void>(work), (size_t)work->numel(), x.stream);
}

// (cache, pool, head_dim, layer, Q, cu_q_lens, page_table, seq_lens, out, max_q_len, window, sinks, scale, stream)
PyObject *prefill_attn_window(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Args x{a, n};
    x.begin();
    const int head_dim = x.integer(), layer = x.integer();
    const at::Tensor *q = x.dense(at::kBFloat16, 3), *cu = x.dense(at::kInt, 1), *table = x.dense(at::kInt, 2), *lens = x.dense(at::kInt, 1),
                     *out = x.dense(at::kBFloat16, 3);
    const int most = x.integer(), window = x.integer(), sinks = x.integer();
    const float scale = x.real();
    if (!x.end() || q->size(2) != head_dim || out->sizes() != q->sizes() || table->size(0) != lens->size(0) || cu->size(0) != lens->size(0) + 1)
        Py_RETURN_NONE;
    const int batch = (int)lens->size(0), heads = (int)q->size(1), width = (int)table->size(1);
    return status_of(prefill_window_entry, x.cache, layer, ptr<void>(q), ptr<int32_t>(cu), ptr<int32_t>(table), ptr<int32_t>(lens), ptr<void>(out), batch, most,
                     heads, width, window, sinks, scale, x.stream);
}

// rows [n][heads][dim] whose heads are dense and whose rows may be further apart; their distance in elements, or -1
int64_t row_stride(const at::Tensor *t, int64_t n, int64_t heads, int64_t dim)
{
    if (!t || t->dim() != 3 || t->size(0) != n || t->size(1) != heads || t->size(2) != dim) return -1;
    const int64_t row = n <= 1 ? heads * dim : t->stride(0);        // (a single row's stride says nothing)
    if (n > 0 && heads > 0 && (t->stride(2) != 1 || (heads > 1 && t->stride(1) != dim) || row < heads * dim)) return -1;
    return row;
}

// (cache, pool, head_dim, kv_heads, n_axes, layer, rope, Q, Q_out, K, V, positions, slot_map, stream)
PyObject *rope_append(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    Args x{a, n_args};
    x.begin();
    const int head_dim = x.integer(), kv_heads = x.integer(), n_axes = x.integer(), layer = x.integer();
    const skv_rope *rope = static_cast<const skv_rope *>(x.handle());
    const at::Tensor *q = x.tensor(at::kBFloat16), *q_out = x.tensor(at::kBFloat16);
    if (!x.ok) Py_RETURN_NONE;
    const bool owner = is_owner(x.cache, layer) == 1;
    const at::Tensor *k = nullptr, *v = nullptr, *slots = nullptr;
    if (owner) {
        k = x.tensor(at::kBFloat16);
        v = x.tensor(at::kBFloat16);
    } else x.i += 2;
    const at::Tensor *pos = x.tensor(at::kInt);
    if (owner) slots = x.dense(at::kLong, 1);
    else x.i += 1;
    if (!x.end() || q->dim() != 3 || pos->dim() < 1 || pos->dim() > 2) Py_RETURN_NONE;
    const int64_t n = pos->size(-1), axes = pos->dim() == 2 ? pos->size(0) : 1, heads = q->size(1);
    if (axes != n_axes || (n > 1 && pos->stride(-1) != 1) || heads > 0x7FFFFFFF) Py_RETURN_NONE;
    const int64_t qs = row_stride(q, n, heads, head_dim), os = row_stride(q_out, n, heads, head_dim);
    const int64_t ks = owner ? row_stride(k, n, kv_heads, head_dim) : 0, vs = owner ? row_stride(v, n, kv_heads, head_dim) : 0;
    if (qs < 0 || os < 0 || ks < 0 || vs < 0 || (owner && slots->size(0) != n)) Py_RETURN_NONE;
    return status_of(rope_append_entry, x.cache, layer, rope, ptr<void>(q), qs, ptr<void>(q_out), os, owner ? ptr<void>(k) : nullptr, ks,
                     owner ? ptr<void>(v) : nullptr, vs, ptr<int32_t>(pos), axes > 1 ? pos->stride(0) : n,
                     owner ? ptr<int64_t>(slots) : nullptr, n, (int)heads, x.stream);
}

// (cache, pool, page_table, seq_lens, new_lens, free_pages, n_free, slot_map, cu_q_lens, seq_lens_out, n_free_out, positions, stream)
PyObject *plan_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Args x{a, n};
    x.begin();
    const at::Tensor *table = x.dense(at::kInt, 2), *lens = x.dense(at::kInt, 1), *news = x.dense(at::kInt, 1), *pages = x.dense(at::kInt, 1),
                     *n_free = x.dense(at::kInt, 1), *slots = x.dense(at::kLong, 1), *cu = x.dense(at::kInt, 1), *lens_out = x.dense(at::kInt, 1),
                     *free_out = x.dense(at::kInt, 1), *pos = nullptr;
    if (x.i < n && a[x.i] == Py_None) ++x.i;
    else pos = x.dense(at::kInt, 1);
    if (!x.end()) Py_RETURN_NONE;
    const int64_t batch = lens->size(0);
    if (table->size(0) != batch || news->size(0) != batch || lens_out->size(0) != batch || cu->size(0) != batch + 1 || n_free->size(0) != 1 ||
        free_out->size(0) != 1 || (pos && pos->size(0) < slots->size(0)))
        Py_RETURN_NONE;
    return status_of(plan_step_entry, x.cache, ptr<int32_t>(table), (int)table->size(1), ptr<int32_t>(lens), ptr<int32_t>(news), (int)batch, ptr<int32_t>(pages),
                     (int)pages->size(0), ptr<int32_t>(n_free), slots->size(0), ptr<int64_t>(slots), pos ? ptr<int32_t>(pos) : nullptr,
                     ptr<int32_t>(cu), ptr<int32_t>(lens_out), ptr<int32_t>(free_out), x.stream);
}

// (cache, pool, page_table, first_page, end_page, free_pages, n_free, n_free_out, stream)
PyObject *plan_release(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Args x{a, n};
    x.begin();
    const at::Tensor *table = x.dense(at::kInt, 2), *first = x.dense(at::kInt, 1), *end = x.dense(at::kInt, 1), *pages = x.dense(at::kInt, 1),
                     *n_free = x.dense(at::kInt, 1), *free_out = x.dense(at::kInt, 1);
    if (!x.end()) Py_RETURN_NONE;
    const int64_t batch = table->size(0);
    if (first->size(0) != batch || end->size(0) != batch || n_free->size(0) != 1 || free_out->size(0) != 1) Py_RETURN_NONE;
    return status_of(plan_release_entry, x.cache, ptr<int32_t>(table), (int)table->size(1), ptr<int32_t>(first), ptr<int32_t>(end), (int)batch,
                     ptr<int32_t>(pages), (int)pages->size(0), ptr<int32_t>(n_free), ptr<int32_t>(free_out), x.stream);
}

// connect(address, ...): the entry points of the loaded library, in the order of the declarations above
PyObject *connect(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "connect: six addresses");
        return nullptr;
    }
    for (int i = 0; i < 6; ++i)
        if (!(p[i] = PyLong_AsVoidPtr(a[i]))) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "connect: a null address");
            return nullptr;
        }
    is_owner = reinterpret_cast<decltype(is_owner)>(p[0]);
    rope_append_entry = reinterpret_cast<decltype(rope_append_entry)>(p[1]);
    plan_step_entry = reinterpret_cast<decltype(plan_step_entry)>(p[2]);
    plan_release_entry = reinterpret_cast<decltype(plan_release_entry)>(p[3]);
    decode_window_entry = reinterpret_cast<decltype(decode_window_entry)>(p[4]);
    prefill_window_entry = reinterpret_cast<decltype(prefill_window_entry)>(p[5]);
    Py_RETURN_NONE;
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(declining<f>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"connect", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(connect)), METH_FASTCALL, nullptr},
                         METHOD(decode_attn_window), METHOD(prefill_attn_window), METHOD(rope_append), METHOD(plan_step),
                         METHOD(plan_release), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", SKV_TORCH_VERSION) != 0) {     // (whose headers say how a tensor lies in memory)
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
