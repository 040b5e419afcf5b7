// The native half of the binding's operators around the ternary product (tst_ops.h), part of the Python module _launch: the calls as
// programs ordinarily make them, with nothing given but the operands, on torch's current stream.  It saves host time: log probabilities of one
// row took 22 us from Python, of which the GPU works 16, through five allocations and ctypes.
//
// Each function returns None, without having done anything, for whatever is not plain or does not fit, and for what the library refuses; the
// caller then goes the long way, which refuses it with the message that belongs to it.  An error of the GPU is raised here.
#include "launch_internal.h"

#include <torch/csrc/Dtype.h>

#include "tst_ops.h"

namespace launch {
namespace {

decltype(&tst_w8_gemm) g_gemm;
decltype(&tst_w8_linear_workspace_bytes) g_linear_bytes;
decltype(&tst_w8_linear) g_linear;
decltype(&tst_moe_workspace_bytes) g_moe_bytes;
decltype(&tst_moe) g_moe;
decltype(&tst_logprobs_workspace_bytes) g_logprobs_bytes;
decltype(&tst_logprobs) g_logprobs;
PyObject *g_error;   // TstgemmError
PyObject *g_w8_class, *g_moe_class;   // W8 and Moe
PyObject *s_K, *s_N, *s_count, *s_packed, *s_scale, *s_raw, *s_device_index;

// A tensor of torch's own class with memory of its own on the current device, which holds its values as they are.
const at::Tensor *plain(PyObject *o, int dev)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.is_neg() || t.get_device() != dev) return nullptr;
    return &t;
}
const at::Tensor *dense(PyObject *o, int dev, at::ScalarType type)
{
    const at::Tensor *t = plain(o, dev);
    return t != nullptr && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}
// A matrix of contiguous rows that do not overlap; *stride: entries from row to row.
const at::Tensor *rows(PyObject *o, int dev, int64_t *stride)
{
    const at::Tensor *t = plain(o, dev);
    if (t == nullptr || t->dim() != 2 || t->size(0) > INT_MAX || t->size(1) > INT_MAX || t->size(1) < 1) return nullptr;
    *stride = t->size(0) > 1 ? t->stride(0) : t->size(1);
    return (t->size(1) > 1 && t->stride(1) != 1) || *stride < t->size(1) ? nullptr : t;
}
int type_of(at::ScalarType t) { return t == at::kFloat ? TST_F32 : t == at::kBFloat16 ? TST_BF16 : t == at::kHalf ? TST_F16 : -1; }

at::Tensor make(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like)
{
    return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}
void *stream_of(int dev) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)dev).stream(); }

PyObject *raise(int rc, const char *name)
{
    PyObject *e = PyObject_CallFunction(g_error, "is", rc, name);
    if (e != nullptr) PyErr_SetObject(g_error, e);
    Py_XDECREF(e);
    return nullptr;
}

struct Layer {
    unsigned long long K = 0, N = 0;
    const void *packed = nullptr;
    const float *scale = nullptr, *b = nullptr;
    bool ok = false;
    Layer(PyObject *w, PyObject *bias, int dev)
    {
        unsigned long long count = 0;
        if ((PyObject *)Py_TYPE(w) != g_w8_class || !int_attr(w, s_count, &count) || count != 1 || !int_attr(w, s_K, &K) || !int_attr(w, s_N, &N) || K < 1 ||
            K > INT_MAX - 64 || N < 1 || N > INT_MAX - 16)
            return;
        const int64_t bytes = ((int64_t)K + 63) / 64 * 64 * (((int64_t)N + 15) / 16 * 16);   // tst_w8_bytes()
        PyObject *p = PyObject_GetAttr(w, s_packed), *s = PyObject_GetAttr(w, s_scale);   // (w keeps them)
        const at::Tensor *pt = p ? dense(p, dev, at::kByte) : nullptr, *st = s ? dense(s, dev, at::kFloat) : nullptr;
        if (pt && st && pt->numel() == bytes && st->numel() == (int64_t)N) {
            packed = pt->data_ptr();
            scale = static_cast<const float *>(st->data_ptr());
            ok = true;
        }
        Py_XDECREF(p);
        Py_XDECREF(s);
        PyErr_Clear();
        if (ok && bias != Py_None) {
            const at::Tensor *t = dense(bias, dev, at::kFloat);
            ok = t != nullptr && t->dim() == 1 && t->numel() == (int64_t)N;
            if (ok) b = static_cast<const float *>(t->data_ptr());
        }
    }
};

template <typename F> PyObject *guarded(PyObject *const *, Py_ssize_t n, Py_ssize_t want, const char *usage, F call)
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

PyObject *w8_gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(a, n, 5, "w8_gemm(Q, scale, w, b, dtype)", [&](int dev) -> PyObject * {
        int64_t stride = 0;
        const at::Tensor *q = rows(a[0], dev, &stride), *s = dense(a[1], dev, at::kFloat);
        if (q == nullptr || q->scalar_type() != at::kChar || s == nullptr || s->dim() != 1 || s->numel() != q->size(0)) Py_RETURN_NONE;
        const Layer w(a[2], a[3], dev);
        if (!w.ok || q->size(1) != (int64_t)w.K) Py_RETURN_NONE;
        at::ScalarType type = at::kFloat;
        if (a[4] != Py_None) {
            if (!THPDtype_Check(a[4])) Py_RETURN_NONE;
            type = reinterpret_cast<THPDtype *>(a[4])->scalar_type;
        }
        if (type_of(type) < 0) Py_RETURN_NONE;
        at::Tensor y;
        int rc;
        {
            WithoutGil released;
            y = make({q->size(0), (int64_t)w.N}, type, *q);
            rc = g_gemm(static_cast<const int8_t *>(q->data_ptr()), stride, static_cast<const float *>(s->data_ptr()), w.packed, w.scale, w.b,
                        y.data_ptr(), type_of(type), (int)q->size(0), (int)w.K, (int)w.N, stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_w8_gemm");
        if (rc != 0) Py_RETURN_NONE;
        return THPVariable_Wrap(std::move(y));
    });
}

PyObject *w8_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(a, n, 3, "w8_linear(X, w, b)", [&](int dev) -> PyObject * {
        int64_t stride = 0;
        const at::Tensor *x = rows(a[0], dev, &stride);
        if (x == nullptr || type_of(x->scalar_type()) < 0) Py_RETURN_NONE;
        const Layer w(a[1], a[2], dev);
        if (!w.ok || x->size(1) != (int64_t)w.K) Py_RETURN_NONE;
        const int M = (int)x->size(0), K = (int)w.K;
        size_t bytes = 0;
        if (g_linear_bytes(M, K, &bytes) != 0) Py_RETURN_NONE;
        at::Tensor y, ws;
        int rc;
        {
            WithoutGil released;
            y = make({M, (int64_t)w.N}, x->scalar_type(), *x);
            ws = make({(int64_t)bytes}, at::kByte, *x);
            rc = g_linear(x->data_ptr(), type_of(x->scalar_type()), stride, w.packed, w.scale, w.b, y.data_ptr(), M, K, (int)w.N, ws.data_ptr(),
                          bytes, stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_w8_linear");
        if (rc != 0) Py_RETURN_NONE;
        return THPVariable_Wrap(std::move(y));
    });
}

PyObject *moe(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(a, n, 4, "moe(X, moe, top_k, normalize)", [&](int dev) -> PyObject * {
        unsigned long long raw = 0, index = 0;
        int64_t stride = 0;
        const at::Tensor *x = rows(a[0], dev, &stride);
        if (x == nullptr || (PyObject *)Py_TYPE(a[1]) != g_moe_class || !int_attr(a[1], s_raw, &raw) || !int_attr(a[1], s_device_index, &index) || raw == 0 || (int)index != dev ||
            !PyLong_CheckExact(a[2]) || !PyBool_Check(a[3]))
            Py_RETURN_NONE;
        const tst_moe_t *m = reinterpret_cast<const tst_moe_t *>(raw);
        const long top = PyLong_AsLong(a[2]);
        if (PyErr_Occurred() || top < 1 || top > TST_MOE_MAX_TOP || type_of(x->scalar_type()) != m->type || x->size(1) != m->width) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int T = (int)x->size(0);
        size_t bytes = 0;
        if (g_moe_bytes(m, T, (int)top, &bytes) != 0) Py_RETURN_NONE;
        at::Tensor y, ids, p, ws;
        int rc;
        {
            WithoutGil released;
            y = make({T, m->width}, x->scalar_type(), *x);
            ids = make({T, top}, at::kInt, *x);
            p = make({T, top}, at::kFloat, *x);
            ws = make({(int64_t)bytes}, at::kByte, *x);
            rc = g_moe(x->data_ptr(), stride, m, (int)top, a[3] == Py_True, y.data_ptr(), static_cast<int32_t *>(ids.data_ptr()),
                       static_cast<float *>(p.data_ptr()), T, ws.data_ptr(), bytes, stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_moe");
        if (rc != 0) Py_RETURN_NONE;
        return Py_BuildValue("NNN", THPVariable_Wrap(std::move(y)), THPVariable_Wrap(std::move(ids)), THPVariable_Wrap(std::move(p)));
    });
}

PyObject *logprobs(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(a, n, 3, "logprobs(logits, tokens, top)", [&](int dev) -> PyObject * {
        int64_t stride = 0;
        const at::Tensor *z = rows(a[0], dev, &stride);
        if (z == nullptr || type_of(z->scalar_type()) < 0 || !PyLong_CheckExact(a[2])) Py_RETURN_NONE;
        const long top = PyLong_AsLong(a[2]);
        if (PyErr_Occurred() || top < 0 || top > TST_LOGPROBS_MAX_TOP) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int R = (int)z->size(0), V = (int)z->size(1);
        const at::Tensor *t = nullptr;
        int token_bytes = 8, C = 0;
        if (a[1] != Py_None) {
            t = plain(a[1], dev);
            if (t == nullptr || (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) || (t->dim() != 1 && t->dim() != 2) ||
                t->size(0) != R || !t->is_contiguous() || (t->dim() == 2 && t->size(1) > TST_LOGPROBS_MAX_TOKENS))
                Py_RETURN_NONE;
            token_bytes = t->scalar_type() == at::kInt ? 4 : 8;
            C = t->dim() == 1 ? 1 : (int)t->size(1);
        }
        size_t bytes = 0;
        if (g_logprobs_bytes(R, V, (int)top, &bytes) != 0) Py_RETURN_NONE;
        at::Tensor of_token, entropy, ids, of_top, ws;
        int rc;
        {
            WithoutGil released;
            of_token = t == nullptr ? make({R, 0}, at::kFloat, *z) : make(t->sizes(), at::kFloat, *z);
            entropy = make({R}, at::kFloat, *z);
            ids = make({R, top}, at::kInt, *z);
            of_top = make({R, top}, at::kFloat, *z);
            if (bytes) ws = make({(int64_t)bytes}, at::kByte, *z);
            rc = g_logprobs(z->data_ptr(), type_of(z->scalar_type()), stride, t ? t->data_ptr() : nullptr, token_bytes, C, (int)top,
                            static_cast<float *>(of_token.data_ptr()), static_cast<float *>(entropy.data_ptr()),
                            static_cast<int32_t *>(ids.data_ptr()), static_cast<float *>(of_top.data_ptr()), R, V,
                            bytes ? ws.data_ptr() : nullptr, bytes, stream_of(dev));
        }
        if (rc == TSTGEMM_EHIP) return raise(rc, "tst_logprobs");
        if (rc != 0) Py_RETURN_NONE;
        return Py_BuildValue("NNNN", THPVariable_Wrap(std::move(of_token)), THPVariable_Wrap(std::move(entropy)), THPVariable_Wrap(std::move(ids)),
                             THPVariable_Wrap(std::move(of_top)));
    });
}

// bind_ops(addresses of the seven in the loaded library, TstgemmError, W8, Moe)
PyObject *bind_ops(PyObject *, PyObject *args)
{
    unsigned long long p[7];
    PyObject *error, *w8, *moe_class;
    if (!PyArg_ParseTuple(args, "KKKKKKKOOO", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &error, &w8, &moe_class)) return nullptr;
    g_gemm = reinterpret_cast<decltype(g_gemm)>(p[0]);
    g_linear_bytes = reinterpret_cast<decltype(g_linear_bytes)>(p[1]);
    g_linear = reinterpret_cast<decltype(g_linear)>(p[2]);
    g_moe_bytes = reinterpret_cast<decltype(g_moe_bytes)>(p[3]);
    g_moe = reinterpret_cast<decltype(g_moe)>(p[4]);
    g_logprobs_bytes = reinterpret_cast<decltype(g_logprobs_bytes)>(p[5]);
    g_logprobs = reinterpret_cast<decltype(g_logprobs)>(p[6]);
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_INCREF(w8);
    Py_XSETREF(g_w8_class, w8);
    Py_INCREF(moe_class);
    Py_XSETREF(g_moe_class, moe_class);
    Py_RETURN_NONE;
}

PyCFunction fast(PyObject *(*f)(PyObject *, PyObject *const *, Py_ssize_t)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

}  // namespace

PyMethodDef ops_methods[] = {{"w8_gemm", fast(w8_gemm), METH_FASTCALL, nullptr},     {"w8_linear", fast(w8_linear), METH_FASTCALL, nullptr},
                             {"moe", fast(moe), METH_FASTCALL, nullptr},             {"logprobs", fast(logprobs), METH_FASTCALL, nullptr},
                             {"bind_ops", bind_ops, METH_VARARGS, nullptr},          {nullptr, nullptr, 0, nullptr}};

bool ops_init()
{
    PyObject **const names[] = {&s_K, &s_N, &s_count, &s_packed, &s_scale, &s_raw, &s_device_index};
    const char *const texts[] = {"K", "N", "count", "packed", "scale", "_raw", "device_index"};
    for (int i = 0; i < 7; ++i)
        if ((*names[i] = PyUnicode_InternFromString(texts[i])) == nullptr) return false;
    return true;
}

}  // namespace launch
