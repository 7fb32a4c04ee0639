// The way of the operators that mix tokens from Python into the library: tensors' addresses and sizes are read, outputs and workspaces
// taken from torch, and the library called, without a step through the interpreter.  By ctypes a call cost the host 19 to 24 us, more than
// the kernels of a single token's step take.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>

#include <climits>
#include <cmath>
#include <cstdint>

#include "idf.h"

namespace {

int (*norm_rotate_fn)(const idf_norm_rotate_args *, void *);
int (*window_workspace_fn)(const idf_window_args *, size_t *);
int (*window_fn)(const idf_window_args *, void *);
int (*decay_workspace_fn)(const idf_decay_args *, size_t *);
int (*decay_fn)(const idf_decay_args *, void *);

PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) { PyErr_SetString(PyExc_TypeError, "five addresses"); return nullptr; }
    void *p[5];
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    norm_rotate_fn = reinterpret_cast<decltype(norm_rotate_fn)>(p[0]);
    window_workspace_fn = reinterpret_cast<decltype(window_workspace_fn)>(p[1]);
    window_fn = reinterpret_cast<decltype(window_fn)>(p[2]);
    decay_workspace_fn = reinterpret_cast<decltype(decay_workspace_fn)>(p[3]);
    decay_fn = reinterpret_cast<decltype(decay_fn)>(p[4]);
    Py_RETURN_NONE;
}

// Thrown where arguments are not of the usual kinds, or wrong: the call then goes the long way round, which converts them or raises.
struct Unusual {};

void need(bool ok)
{
    if (!ok) throw Unusual();
}

const at::Tensor *tensor(PyObject *o)
{
    if (o == Py_None) return nullptr;
    need(THPVariable_CheckExact(o));
    const at::Tensor &t = THPVariable_Unpack(o);
    need(!t.requires_grad() || !c10::GradMode::is_enabled());                // (refused there: there is no backward pass)
    return &t;
}

int precision(const at::Tensor &t)
{
    need(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16);
    return t.scalar_type() == at::kFloat ? IDF_PREC_F32 : IDF_PREC_BF16;
}

// Packed tokens [token][head][value], as they are; aligned: rows that begin at multiples of 16 bytes.
idf_tokens rows(const at::Tensor &t, const at::Tensor &like, bool aligned)
{
    need(t.is_cuda() && t.layout() == at::kStrided && t.dim() == 3 && t.scalar_type() == like.scalar_type() && t.device() == like.device() && (t.stride(2) == 1 || t.size(2) <= 1));
    idf_tokens r{t.data_ptr(), t.stride(0), t.stride(1)};
    const int64_t vl = 16 / (int64_t)t.element_size();
    need(!aligned || ((uintptr_t)r.base % 16 == 0 && r.token_stride % vl == 0 && r.head_stride % vl == 0));
    return r;
}

// A contiguous tensor of this type on the device of another, or nullptr.
template <class T> T *plain(const at::Tensor *t, at::ScalarType type, int64_t n, const at::Tensor &like)
{
    if (!t) return nullptr;
    need(t->scalar_type() == type && t->device() == like.device() && t->is_contiguous() && t->dim() == 1 && (n < 0 || t->size(0) == n));
    return static_cast<T *>(t->data_ptr());
}

int64_t whole(PyObject *o)
{
    need(PyLong_CheckExact(o));
    const int64_t v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) { PyErr_Clear(); throw Unusual(); }
    return v;
}
int small(PyObject *o)
{
    const int64_t v = whole(o);
    need(v >= INT_MIN && v <= INT_MAX);
    return (int)v;
}
double real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) { PyErr_Clear(); throw Unusual(); }
    return v;
}

template <class A> int call(int (*fn)(const A *, void *), const A &a, void *stream)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&a, stream);
    Py_END_ALLOW_THREADS
    return rc;
}

// Outputs: the caller's, or new ones.
at::Tensor output(const at::Tensor *given, at::IntArrayRef shape, const at::Tensor &like)
{
    if (given) {
        need(given->sizes() == shape);
        return *given;
    }
    return at::empty(shape, like.options());
}

// Every entry: what the library returned if that is an error, None where the arguments go the long way round, else the outputs.
template <class F> PyObject *entry(F f)
{
    try {
        return f();
    } catch (const Unusual &) {
        Py_RETURN_NONE;
    } catch (...) {                                // (tensors without memory of their own, no memory left: the long way says so)
        if (PyErr_Occurred()) PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// norm_rotate(stream, q, k, positions, frequencies, interleaved, amplitude, q_weight, k_weight, eps, q_out, k_out)
PyObject *norm_rotate(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 12 || !norm_rotate_fn) { PyErr_SetString(PyExc_TypeError, "norm_rotate takes 12 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *q = tensor(args[1]), *k = tensor(args[2]), *pos = tensor(args[3]), *freq = tensor(args[4]);
        need(q && k && pos && freq);
        idf_norm_rotate_args a{};
        a.precision = precision(*q);
        a.q = rows(*q, *q, false);
        a.k = rows(*k, *q, false);
        need(k->size(0) == q->size(0) && k->size(2) == q->size(2) && q->size(1) <= INT_MAX && k->size(1) <= INT_MAX && q->size(2) <= INT_MAX && freq->numel() <= 1024);
        a.heads_q = (int)q->size(1);
        a.heads_k = (int)k->size(1);
        a.head_dim = (int)q->size(2);
        a.n_tokens = q->size(0);
        a.rotary_dim = 2 * (int)freq->numel();
        a.positions = plain<int64_t>(pos, at::kLong, a.n_tokens, *q);
        a.frequencies = plain<double>(freq, at::kDouble, -1, *q);
        a.interleaved = small(args[5]);
        a.amplitude = real(args[6]);
        a.q_weight = plain<float>(tensor(args[7]), at::kFloat, a.head_dim, *q);
        a.k_weight = plain<float>(tensor(args[8]), at::kFloat, a.head_dim, *q);
        a.eps = (float)real(args[9]);
        const c10::DeviceGuard guard(q->device());
        const at::Tensor q_out = output(tensor(args[10]), q->sizes(), *q), k_out = output(tensor(args[11]), k->sizes(), *q);
        a.q_out = rows(q_out, *q, false);
        a.k_out = rows(k_out, *q, false);
        const int rc = call(norm_rotate_fn, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        PyObject *both = PyTuple_New(2);
        if (!both) throw Unusual();
        PyTuple_SET_ITEM(both, 0, args[10] != Py_None ? Py_NewRef(args[10]) : THPVariable_Wrap(q_out));
        PyTuple_SET_ITEM(both, 1, args[11] != Py_None ? Py_NewRef(args[11]) : THPVariable_Wrap(k_out));
        return both;
    });
}

// What both attentions have in common behind q, k and v: segments by offsets, or of one length.
template <class A> void segments(A &a, const at::Tensor &q, const at::Tensor *offsets, PyObject *max_tokens, int64_t count)
{
    if (offsets) {
        a.offsets = plain<int64_t>(offsets, at::kLong, -1, q);
        need(offsets->numel() >= 1 && offsets->numel() - 1 <= INT_MAX);
        a.n_segments = (int)offsets->numel() - 1;
        a.max_tokens = whole(max_tokens);
    } else {
        need(count > 0 && count <= INT_MAX && a.n_tokens % count == 0);
        a.n_segments = (int)count;
        a.max_tokens = a.n_tokens / count;
    }
}

// window_attend(stream, q, k, v, k_ring, v_ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out)
PyObject *window_attend(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 14 || !window_fn) { PyErr_SetString(PyExc_TypeError, "window_attend takes 14 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *q = tensor(args[1]), *k = tensor(args[2]), *v = tensor(args[3]), *k_ring = tensor(args[4]), *v_ring = tensor(args[5]);
        const at::Tensor *starts = tensor(args[6]), *offsets = tensor(args[10]), *ids = tensor(args[12]);
        need(q && k && v && !k_ring == !v_ring);
        idf_window_args a{};
        a.precision = precision(*q);
        a.q = rows(*q, *q, true);
        a.k = rows(*k, *q, true);
        a.v = rows(*v, *q, true);
        need(k->sizes() == v->sizes() && k->size(0) == q->size(0) && k->size(2) == q->size(2) && q->size(1) <= INT_MAX && k->size(1) <= INT_MAX && q->size(2) <= INT_MAX);
        a.heads_q = (int)q->size(1);
        a.heads_kv = (int)k->size(1);
        a.head_dim = (int)q->size(2);
        a.n_tokens = q->size(0);
        if (k_ring) {
            for (const at::Tensor *r : {k_ring, v_ring})
                need(r->dim() == 4 && r->scalar_type() == q->scalar_type() && r->device() == q->device() && r->is_contiguous() && r->size(2) == k->size(1) && r->size(3) == k->size(2) && r->size(0) <= INT_MAX);
            need(k_ring->sizes() == v_ring->sizes());
            a.n_streams = (int)k_ring->size(0);
            a.slots = k_ring->size(1);
            a.k_ring = k_ring->data_ptr();
            a.v_ring = v_ring->data_ptr();
        }
        const int64_t count = ids ? ids->numel() : starts ? starts->numel() : k_ring ? a.n_streams : 1;
        segments(a, *q, offsets, args[11], count);
        need(!(ids || starts) || a.n_segments == count);
        if (!k_ring) a.n_streams = a.n_segments;
        a.starts = plain<int64_t>(starts, at::kLong, a.n_segments, *q);
        a.stream_ids = plain<int32_t>(ids, at::kInt, a.n_segments, *q);
        a.window = small(args[7]);
        a.sinks = small(args[8]);
        a.scale = args[9] == Py_None ? (float)(1.0 / std::sqrt((double)a.head_dim)) : (float)real(args[9]);
        const c10::DeviceGuard guard(q->device());
        const at::Tensor out = output(tensor(args[13]), q->sizes(), *q);
        a.out = rows(out, *q, true);
        int rc = window_workspace_fn(&a, &a.workspace_bytes);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        at::Tensor ws;                             // (held until the work is enqueued)
        if (a.workspace_bytes) {
            ws = at::empty({(int64_t)a.workspace_bytes}, q->options().dtype(at::kByte));
            a.workspace = ws.data_ptr();
        }
        rc = call(window_fn, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        return args[13] != Py_None ? Py_NewRef(args[13]) : THPVariable_Wrap(out);
    });
}

// decay_attend(stream, q, k, v, log_decay, state, state_out, scale, offsets, max_tokens, n_segments, stream_ids, out)
PyObject *decay_attend(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 13 || !decay_fn) { PyErr_SetString(PyExc_TypeError, "decay_attend takes 13 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *q = tensor(args[1]), *k = tensor(args[2]), *v = tensor(args[3]), *log_decay = tensor(args[4]), *in = tensor(args[5]), *to = tensor(args[6]);
        const at::Tensor *offsets = tensor(args[8]), *ids = tensor(args[11]);
        need(q && k && v && log_decay);
        idf_decay_args a{};
        a.precision = precision(*q);
        a.q = rows(*q, *q, true);
        a.k = rows(*k, *q, true);
        a.v = rows(*v, *q, true);
        need(k->size(0) == q->size(0) && v->size(0) == q->size(0) && k->size(1) == v->size(1) && k->size(2) == q->size(2) && q->size(1) <= INT_MAX && k->size(1) <= INT_MAX && q->size(2) <= INT_MAX && v->size(2) <= INT_MAX);
        a.heads_q = (int)q->size(1);
        a.heads_kv = (int)k->size(1);
        a.dim_k = (int)q->size(2);
        a.dim_v = (int)v->size(2);
        a.n_tokens = q->size(0);
        a.log_decay = plain<float>(log_decay, at::kFloat, a.heads_kv, *q);
        int64_t streams = -1;
        for (const at::Tensor *s : {in, to}) {
            if (!s) continue;
            need(s->dim() == 4 && s->scalar_type() == at::kFloat && s->device() == q->device() && s->is_contiguous() && s->size(1) == k->size(1) && s->size(2) == q->size(2) && s->size(3) == v->size(2));
            need((streams < 0 || streams == s->size(0)) && s->size(0) <= INT_MAX);
            streams = s->size(0);
        }
        a.state_in = in ? static_cast<const float *>(in->data_ptr()) : nullptr;
        a.state_out = to ? static_cast<float *>(to->data_ptr()) : nullptr;
        const bool told = ids || args[10] != Py_None;
        const int64_t count = ids ? ids->numel() : args[10] != Py_None ? whole(args[10]) : streams >= 0 ? streams : 1;
        segments(a, *q, offsets, args[9], count);
        need(!told || a.n_segments == count);
        a.n_streams = streams >= 0 ? (int)streams : a.n_segments;
        a.stream_ids = plain<int32_t>(ids, at::kInt, a.n_segments, *q);
        a.scale = args[7] == Py_None ? (float)(1.0 / std::sqrt((double)a.dim_k)) : (float)real(args[7]);
        const c10::DeviceGuard guard(q->device());
        const at::Tensor out = output(tensor(args[12]), {a.n_tokens, a.heads_q, a.dim_v}, *q);
        a.out = rows(out, *q, true);
        int rc = decay_workspace_fn(&a, &a.workspace_bytes);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        at::Tensor ws;
        if (a.workspace_bytes) {
            ws = at::empty({(int64_t)a.workspace_bytes}, q->options().dtype(at::kByte));
            a.workspace = ws.data_ptr();
        }
        rc = call(decay_fn, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        return args[12] != Py_None ? Py_NewRef(args[12]) : THPVariable_Wrap(out);
    });
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", FAST(bind), "the addresses of the library's functions"},
    {"norm_rotate", FAST(norm_rotate), "idf_norm_rotate on tensors"},
    {"window_attend", FAST(window_attend), "idf_window_attend on tensors"},
    {"decay_attend", FAST(decay_attend), "idf_decay_attend on tensors"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tokens", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tokens() { return PyModule_Create(&module); }
