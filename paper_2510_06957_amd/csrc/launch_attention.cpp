// The native half of the binding's cache of keys and values and of attention (tst_attention.h), part of the Python module _launch: calls as programs ordinarily
// make them, on torch's current stream, with nothing given but the operands.  It saves host time: 64 tokens appended took 18 us from Python, of which the GPU
// works 6, through structs of ctypes.
//
// Each function returns None, without having done anything, for whatever is not plain or does not fit, and for what the library refuses; the caller then goes the long
// way, which refuses it with the message that belongs to it.  An error of the GPU is raised here.
#include "launch_internal.h"

#include <torch/csrc/Dtype.h>

#include <cmath>

#include "tst_attention.h"

namespace launch {
namespace {

decltype(&tst_kv_append) g_append;
decltype(&tst_kv_read) g_read;
decltype(&tst_kv_attention_workspace_bytes) g_cached_bytes;
decltype(&tst_kv_attention) g_cached;
decltype(&tst_attention) g_prompt;
PyObject *g_error, *g_cache_class;   // TstgemmError, KvCache
PyObject *s_raw, *s_device_index, *s_tensors;

// A tensor of torch's own class with memory of its own on device dev, which holds its values as they are.
const at::Tensor *plain(PyObject *o, int dev)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.is_neg() || t.get_device() != dev) return nullptr;
    return &t;
}
int type_of(at::ScalarType t) { return t == at::kFloat ? TST_F32 : t == at::kBFloat16 ? TST_BF16 : t == at::kHalf ? TST_F16 : -1; }

// [tokens, heads, size] whose heads' entries lie together.
const at::Tensor *heads(PyObject *o, int dev, tst_heads_t *out)
{
    const at::Tensor *t = plain(o, dev);
    if (t == nullptr || t->dim() != 3 || type_of(t->scalar_type()) < 0 || t->size(0) > TST_MAX_TOKENS || t->size(1) < 1 || t->size(1) > TST_MAX_HEADS || t->size(2) < 1 ||
        t->size(2) > TST_MAX_HEAD_SIZE || (t->size(2) > 1 && t->stride(2) != 1))
        return nullptr;
    *out = tst_heads_t{t->data_ptr(), t->size(0) > 1 ? t->stride(0) : 0, t->size(1) > 1 ? t->stride(1) : 0};
    return t;
}
const int32_t *int32(PyObject *o, int dev, int64_t n)
{
    const at::Tensor *t = plain(o, dev);
    return t != nullptr && t->scalar_type() == at::kInt && t->dim() == 1 && t->size(0) == n && t->is_contiguous() ? static_cast<const int32_t *>(t->data_ptr()) : nullptr;
}
const at::Tensor *angles(PyObject *o, int dev)
{
    const at::Tensor *t = plain(o, dev);
    return t != nullptr && t->scalar_type() == at::kFloat && t->dim() == 2 && t->is_contiguous() && t->size(0) >= 1 && t->size(0) <= INT_MAX && t->size(1) >= 1 &&
                   t->size(1) <= TST_MAX_HEAD_SIZE
               ? t : nullptr;
}

// A cache and the sequences of a call; ok only if all of it fits.
struct Call {
    const tst_kv_cache_t *cache = nullptr;
    tst_sequences_t s{};
    bool ok = false;
    // The struct has the tensors' addresses: they have to be where they were.
    bool as_it_was(PyObject *c) const
    {
        PyObject *tensors = PyObject_GetAttr(c, s_tensors);
        const void *const at[4] = {cache->k_codes, cache->v_codes, cache->k_scale, cache->v_scale};
        bool same = tensors != nullptr && PyTuple_CheckExact(tensors) && PyTuple_GET_SIZE(tensors) == 4;
        for (int i = 0; same && i < 4; ++i) {
            PyObject *t = PyTuple_GET_ITEM(tensors, i);
            same = THPVariable_Check(t) && THPVariable_Unpack(t).data_ptr() == at[i];
        }
        Py_XDECREF(tensors);
        PyErr_Clear();
        return same;
    }
    Call(PyObject *c, PyObject *pages, PyObject *lens, PyObject *offsets, int64_t tokens, int dev)
    {
        unsigned long long raw = 0, index = 0;
        if ((PyObject *)Py_TYPE(c) != g_cache_class || !int_attr(c, s_raw, &raw) || !int_attr(c, s_device_index, &index) || raw == 0 || (int)index != dev) return;
        cache = reinterpret_cast<const tst_kv_cache_t *>(raw);
        if (!as_it_was(c)) return;
        const at::Tensor *p = plain(pages, dev);
        if (p == nullptr || p->scalar_type() != at::kInt || p->dim() != 2 || p->size(0) > TST_MAX_SEQUENCES || p->size(1) < 1 || p->size(1) > INT_MAX ||
            (p->size(1) > 1 && p->stride(1) != 1))
            return;
        const int64_t S = p->size(0);
        const int32_t *l = int32(lens, dev, S), *o = nullptr;
        if (l == nullptr || (offsets != Py_None && (o = int32(offsets, dev, S + 1)) == nullptr) || tokens > TST_MAX_TOKENS || (o == nullptr && tokens != S)) return;
        s = tst_sequences_t{sizeof(tst_sequences_t), (int)S, (int)tokens, o, l, static_cast<const int32_t *>(p->data_ptr()), (int)p->size(1), S > 1 ? p->stride(0) : p->size(1)};
        ok = true;
    }
};

at::Tensor make(at::IntArrayRef shape, at::ScalarType type, int dev)
{
    return at::empty(shape, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)dev)));
}
void *stream_of(int dev) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)dev).stream(); }

PyObject *raise(int rc, const char *name)
{
    PyObject *e = PyObject_CallFunction(g_error, "is", rc, name);
    if (e != nullptr) PyErr_SetObject(g_error, e);
    Py_XDECREF(e);
    return nullptr;
}

template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, const char *usage, F call)
{
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, usage);
        return nullptr;
    }
    try {
        if (g_error == nullptr || modes_set()) Py_RETURN_NONE;
        return call(c10::hip::current_device());
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
// The factor of logits, or 1 / sqrt(size); NaN for what is none.
float scale_of(PyObject *o, int64_t size)
{
    if (o == Py_None) return (float)(1 / std::sqrt((double)size));
    return PyFloat_CheckExact(o) ? (float)PyFloat_AS_DOUBLE(o) : NAN;
}
PyObject *or_none(at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(std::move(t));
    Py_RETURN_NONE;
}

PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, "kv_append(cache, K, V, pages, lens, offsets, Q, cos, sin, interleaved, keys)", [&](int dev) -> PyObject * {
        tst_heads_t k, v, q{};
        const at::Tensor *kt = heads(a[1], dev, &k), *vt = heads(a[2], dev, &v), *qt = nullptr;
        if (kt == nullptr || vt == nullptr || vt->scalar_type() != kt->scalar_type() || vt->sizes() != kt->sizes() || !PyBool_Check(a[9]) || !PyBool_Check(a[10])) Py_RETURN_NONE;
        const Call c(a[0], a[3], a[4], a[5], kt->size(0), dev);
        if (!c.ok || kt->size(1) != c.cache->heads || kt->size(2) != c.cache->head_size) Py_RETURN_NONE;
        tst_rotation_t r{};
        if (a[7] != Py_None) {
            const at::Tensor *cs = angles(a[7], dev), *sn = angles(a[8], dev);
            if (cs == nullptr || sn == nullptr || cs->sizes() != sn->sizes()) Py_RETURN_NONE;
            r = tst_rotation_t{sizeof(tst_rotation_t), static_cast<const float *>(cs->data_ptr()), static_cast<const float *>(sn->data_ptr()), (int)cs->size(0), (int)cs->size(1),
                               a[9] == Py_True};
        } else if (a[8] != Py_None || a[6] != Py_None || a[10] == Py_True) Py_RETURN_NONE;
        if (a[6] != Py_None) {
            qt = heads(a[6], dev, &q);
            if (qt == nullptr || qt->scalar_type() != kt->scalar_type() || qt->size(0) != kt->size(0) || qt->size(2) != kt->size(2)) Py_RETURN_NONE;
        }
        at::Tensor q_out, k_out;
        int rc;
        {
            WithoutGil released;
            if (qt) q_out = make(qt->sizes(), qt->scalar_type(), dev);
            if (a[10] == Py_True) k_out = make(kt->sizes(), kt->scalar_type(), dev);
            rc = g_append(c.cache, &c.s, type_of(kt->scalar_type()), &k, &v, qt ? &q : nullptr, qt ? (int)qt->size(1) : 0, r.cos ? &r : nullptr, qt ? q_out.data_ptr() : nullptr,
                          k_out.defined() ? k_out.data_ptr() : nullptr, stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_kv_append");
        if (rc != 0) Py_RETURN_NONE;
        return Py_BuildValue("NN", or_none(q_out), or_none(k_out));
    });
}

PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, "kv_read(cache, pages, lens, tokens, offsets, dtype)", [&](int dev) -> PyObject * {
        if (!PyLong_CheckExact(a[3])) Py_RETURN_NONE;
        const long long tokens = PyLong_AsLongLong(a[3]);
        if (PyErr_Occurred() || tokens < 0) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const Call c(a[0], a[1], a[2], a[4], tokens, dev);
        const at::ScalarType type = a[5] == Py_None ? at::kBFloat16 : THPDtype_Check(a[5]) ? reinterpret_cast<THPDtype *>(a[5])->scalar_type : at::kByte;
        if (!c.ok || type_of(type) < 0) Py_RETURN_NONE;
        at::Tensor k, v;
        int rc;
        {
            WithoutGil released;
            k = make({tokens, c.cache->heads, c.cache->head_size}, type, dev);
            v = make({tokens, c.cache->heads, c.cache->head_size}, type, dev);
            rc = g_read(c.cache, &c.s, type_of(type), k.data_ptr(), v.data_ptr(), stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_kv_read");
        if (rc != 0) Py_RETURN_NONE;
        return Py_BuildValue("NN", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
    });
}

PyObject *kv_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, "kv_attention(Q, cache, pages, lens, offsets, scale)", [&](int dev) -> PyObject * {
        tst_heads_t q;
        const at::Tensor *qt = heads(a[0], dev, &q);
        if (qt == nullptr) Py_RETURN_NONE;
        const Call c(a[1], a[2], a[3], a[4], qt->size(0), dev);
        const float scale = scale_of(a[5], qt->size(2));
        size_t bytes = 0;
        if (!c.ok || qt->size(2) != c.cache->head_size || !(scale <= 0x1p127f && scale >= -0x1p127f) || g_cached_bytes(c.cache, &c.s, (int)qt->size(1), &bytes) != 0) Py_RETURN_NONE;
        at::Tensor y, ws;
        int rc;
        {
            WithoutGil released;
            y = make(qt->sizes(), qt->scalar_type(), dev);
            if (bytes) ws = make({(int64_t)bytes}, at::kByte, dev);
            rc = g_cached(&q, type_of(qt->scalar_type()), (int)qt->size(1), c.cache, &c.s, scale, y.data_ptr(), bytes ? ws.data_ptr() : nullptr, bytes, stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_kv_attention");
        if (rc != 0) Py_RETURN_NONE;
        return THPVariable_Wrap(std::move(y));
    });
}

PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, "attention(Q, K, V, offsets, scale)", [&](int dev) -> PyObject * {
        tst_heads_t q, k, v;
        const at::Tensor *qt = heads(a[0], dev, &q), *kt = heads(a[1], dev, &k), *vt = heads(a[2], dev, &v), *o = plain(a[3], dev);
        if (qt == nullptr || kt == nullptr || vt == nullptr || kt->scalar_type() != qt->scalar_type() || vt->scalar_type() != qt->scalar_type() || kt->size(0) != qt->size(0) ||
            kt->size(2) != qt->size(2) || vt->sizes() != kt->sizes() || o == nullptr || o->dim() != 1 || o->size(0) < 1 || o->size(0) > TST_MAX_SEQUENCES + 1)
            Py_RETURN_NONE;
        const int32_t *offsets = int32(a[3], dev, o->size(0));
        const float scale = scale_of(a[4], qt->size(2));
        if (offsets == nullptr || !(scale <= 0x1p127f && scale >= -0x1p127f)) Py_RETURN_NONE;
        at::Tensor y;
        int rc;
        {
            WithoutGil released;
            y = make(qt->sizes(), qt->scalar_type(), dev);
            rc = g_prompt(&q, &k, &v, type_of(qt->scalar_type()), (int)qt->size(1), (int)kt->size(1), (int)qt->size(2), offsets, (int)o->size(0) - 1, (int)qt->size(0), scale,
                          y.data_ptr(), stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_attention");
        if (rc != 0) Py_RETURN_NONE;
        return THPVariable_Wrap(std::move(y));
    });
}

// bind_attention(addresses of the five in the loaded library, TstgemmError, KvCache)
PyObject *bind_attention(PyObject *, PyObject *args)
{
    unsigned long long p[5];
    PyObject *error, *cache;
    if (!PyArg_ParseTuple(args, "KKKKKOO", &p[0], &p[1], &p[2], &p[3], &p[4], &error, &cache)) return nullptr;
    g_append = reinterpret_cast<decltype(g_append)>(p[0]);
    g_read = reinterpret_cast<decltype(g_read)>(p[1]);
    g_cached_bytes = reinterpret_cast<decltype(g_cached_bytes)>(p[2]);
    g_cached = reinterpret_cast<decltype(g_cached)>(p[3]);
    g_prompt = reinterpret_cast<decltype(g_prompt)>(p[4]);
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_INCREF(cache);
    Py_XSETREF(g_cache_class, cache);
    Py_RETURN_NONE;
}

PyCFunction fast(PyObject *(*f)(PyObject *, PyObject *const *, Py_ssize_t)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

}  // namespace

PyMethodDef attention_methods[] = {{"kv_append", fast(kv_append), METH_FASTCALL, nullptr},       {"kv_read", fast(kv_read), METH_FASTCALL, nullptr},
                                   {"kv_attention", fast(kv_attention), METH_FASTCALL, nullptr}, {"attention", fast(attention), METH_FASTCALL, nullptr},
                                   {"bind_attention", bind_attention, METH_VARARGS, nullptr},    {nullptr, nullptr, 0, nullptr}};

bool attention_init()
{
    s_raw = PyUnicode_InternFromString("_raw");
    s_device_index = PyUnicode_InternFromString("_device_index");
    s_tensors = PyUnicode_InternFromString("_tensors");
    return s_raw != nullptr && s_device_index != nullptr && s_tensors != nullptr;
}

}  // namespace launch
