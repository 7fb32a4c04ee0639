// The way of the operators that mix tokens from Python into the library: tensors' addresses and sizes are read, outputs and workspaces
// taken from torch, and the library called, without a step through the interpreter.  By ctypes a call cost the host 19 to 24 us, more than
// the kernels of a single token's step take.
#include <Python.h>

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <exception>
#include <initializer_list>
#include <optional>
#include <stdexcept>

#include "idf.h"

namespace {

// The library's functions, in the order in which bind takes them.
struct Functions {
    int (*norm_rotate)(const idf_norm_rotate_args *, void *);
    int (*window_workspace)(const idf_window_args *, size_t *);
    int (*window)(const idf_window_args *, void *);
    int (*decay_workspace)(const idf_decay_args *, size_t *);
    int (*decay)(const idf_decay_args *, void *);
    int (*quantize)(const idf_quantize_args *, void *);
    int (*project_workspace)(const idf_project_args *, size_t *);
    int (*project)(const idf_project_args *, void *);
    int (*nibble_append)(const idf_nibble_append_args *, void *);
    int (*nibble_workspace)(const idf_nibble_attend_args *, size_t *);
    int (*nibble_attend)(const idf_nibble_attend_args *, void *);
    int (*nibble_values)(const idf_nibble_values_args *, void *);
    int (*gate_workspace)(const idf_gate_scan_args *, size_t *);
    int (*gate)(const idf_gate_scan_args *, void *);
    int (*gate_back_workspace)(const idf_gate_scan_backward_args *, size_t *);
    int (*gate_back)(const idf_gate_scan_backward_args *, void *);
    int (*gate_marks)(const idf_gate_scan_args *, size_t *);
    int (*is_capturing)(void *, int *);            // the runtime's own
} fn;
constexpr int kFunctions = sizeof(Functions) / sizeof(void *);
bool bound;

PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != kFunctions) { PyErr_Format(PyExc_TypeError, "%d addresses", kFunctions); return nullptr; }
    void *p[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    std::memcpy(&fn, p, sizeof(fn));
    bound = true;
    Py_RETURN_NONE;
}

// Thrown where arguments are not of the usual kinds, or wrong: the call then goes the long way round, which converts them or raises.  Where there is no long way, in a
// backward pass, torch makes an error of it: its threads catch what is an exception, and end the process with anything else.
struct Unusual : std::exception {
    const char *what() const noexcept override { return "tensors of another kind or size than this call takes"; }
};

void need(bool ok)
{
    if (!ok) throw Unusual();
}

const at::Tensor *recorded_tensor(PyObject *o)
{
    if (o == Py_None) return nullptr;
    need(THPVariable_CheckExact(o));
    return &THPVariable_Unpack(o);
}
const at::Tensor *tensor(PyObject *o)
{
    const at::Tensor *t = recorded_tensor(o);
    // (refused there: there is no backward pass, and no tangent of a result)
    need(!t || ((!t->requires_grad() || !c10::GradMode::is_enabled()) && !t->_fw_grad(0).defined()));
    return t;
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

template <class A> int call(int (*f)(const A *, void *), const A &a, void *stream)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(&a, stream);
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

// What a call has written into tensors of the caller's counts as a change in place: torch refuses gradients that would start from what they held before.
void written(std::initializer_list<const at::Tensor *> tensors)
{
    for (const at::Tensor *t : tensors)
        if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// Every entry: what the library returned if that is an error, None where the arguments go the long way round, else the outputs.
template <class F> PyObject *entry(F f)
{
    try {
        return f();
    } catch (const Unusual &) {
        Py_RETURN_NONE;
    } catch (python_error &e) {                    // (Python's own, raised within the call: a hook of the program's, or torch's checkpoints, which end a run by one)
        e.restore();
        return nullptr;
    } catch (...) {                                // (tensors without memory of their own, no memory left: the long way says so)
        if (PyErr_Occurred()) PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// norm_rotate(stream, q, k, positions, frequencies, interleaved, amplitude, q_weight, k_weight, eps, q_out, k_out)
PyObject *norm_rotate(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 12 || !bound) { PyErr_SetString(PyExc_TypeError, "norm_rotate takes 12 arguments"); return nullptr; }
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
        const at::Tensor *given[2] = {tensor(args[10]), tensor(args[11])};
        const at::Tensor q_out = output(given[0], q->sizes(), *q), k_out = output(given[1], k->sizes(), *q);
        a.q_out = rows(q_out, *q, false);
        a.k_out = rows(k_out, *q, false);
        const int rc = call(fn.norm_rotate, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given[0], given[1]});
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
    if (n != 14 || !bound) { PyErr_SetString(PyExc_TypeError, "window_attend takes 14 arguments"); return nullptr; }
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
        const at::Tensor *given = tensor(args[13]);
        const at::Tensor out = output(given, q->sizes(), *q);
        a.out = rows(out, *q, true);
        int rc = fn.window_workspace(&a, &a.workspace_bytes);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        at::Tensor ws;                             // (held until the work is enqueued)
        if (a.workspace_bytes) {
            ws = at::empty({(int64_t)a.workspace_bytes}, q->options().dtype(at::kByte));
            a.workspace = ws.data_ptr();
        }
        rc = call(fn.window, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given, k_ring, v_ring});
        return args[13] != Py_None ? Py_NewRef(args[13]) : THPVariable_Wrap(out);
    });
}

// decay_attend(stream, q, k, v, log_decay, state, state_out, scale, offsets, max_tokens, n_segments, stream_ids, out)
PyObject *decay_attend(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 13 || !bound) { PyErr_SetString(PyExc_TypeError, "decay_attend takes 13 arguments"); return nullptr; }
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
        const at::Tensor *given = tensor(args[12]);
        const at::Tensor out = output(given, {a.n_tokens, a.heads_q, a.dim_v}, *q);
        a.out = rows(out, *q, true);
        int rc = fn.decay_workspace(&a, &a.workspace_bytes);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        at::Tensor ws;
        if (a.workspace_bytes) {
            ws = at::empty({(int64_t)a.workspace_bytes}, q->options().dtype(at::kByte));
            a.workspace = ws.data_ptr();
        }
        rc = call(fn.decay, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given, to});
        return args[12] != Py_None ? Py_NewRef(args[12]) : THPVariable_Wrap(out);
    });
}

// What a call needs beside its arguments, held until the work is enqueued; what the library returned if that is an error.
template <class A> int with_workspace(int (*size)(const A *, size_t *), A &a, const at::Tensor &like, at::Tensor &ws)
{
    const int rc = size(&a, &a.workspace_bytes);
    if (rc == IDF_OK && a.workspace_bytes) {
        ws = at::empty({(int64_t)a.workspace_bytes}, like.options().dtype(at::kByte));
        a.workspace = ws.data_ptr();
    }
    return rc;
}

// A matrix whose values lie next to each other in a row.
idf_rows matrix(const at::Tensor &t, const at::Tensor &like)
{
    need(t.is_cuda() && t.layout() == at::kStrided && t.dim() == 2 && t.device() == like.device() && (t.stride(1) == 1 || t.size(1) <= 1));
    need(t.size(0) <= 1 || t.stride(0) <= 1 << 25);
    return idf_rows{t.data_ptr(), t.size(0) > 1 ? t.stride(0) : t.size(1)};
}

// From the first byte of a matrix to behind its last one; a result that reaches into what is read is looked at more closely the long way round.
struct Reach { uintptr_t from, to; };
Reach reach(const idf_rows &m, int64_t rows, int64_t cols, int64_t bytes)
{
    return {(uintptr_t)m.base, rows && cols ? (uintptr_t)m.base + ((rows - 1) * m.row_stride + cols) * bytes : (uintptr_t)m.base};
}
Reach reach(const at::Tensor &t) { return {(uintptr_t)t.data_ptr(), (uintptr_t)t.data_ptr() + t.numel() * t.element_size()}; }          // (without gaps)
void need_apart(const Reach &a, const Reach &b) { need(a.to <= b.from || b.to <= a.from); }

// quantize_rows(stream, x, codes, scales)
PyObject *quantize_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4 || !bound) { PyErr_SetString(PyExc_TypeError, "quantize_rows takes 4 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *x = tensor(args[1]);
        need(x);
        idf_quantize_args a{};
        a.precision = precision(*x);
        a.x = matrix(*x, *x);
        need(x->size(1) <= INT_MAX - 16);
        a.n_rows = x->size(0);
        a.cols = (int)x->size(1);
        const c10::DeviceGuard guard(x->device());
        const at::Tensor *given[2] = {tensor(args[2]), tensor(args[3])};
        const int64_t padded = (a.cols + 15) / 16 * 16;
        at::Tensor codes = given[0] ? *given[0] : at::empty({a.n_rows, padded}, x->options().dtype(at::kChar));
        at::Tensor scales = given[1] ? *given[1] : at::empty({a.n_rows}, x->options().dtype(at::kFloat));
        need(codes.scalar_type() == at::kChar && codes.device() == x->device() && codes.is_contiguous() && codes.dim() == 2 && codes.size(0) == a.n_rows && codes.size(1) == padded);
        a.codes = static_cast<int8_t *>(codes.data_ptr());
        a.scales = plain<float>(&scales, at::kFloat, a.n_rows, *x);
        const int rc = call(fn.quantize, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given[0], given[1]});
        PyObject *both = PyTuple_New(2);
        if (!both) throw Unusual();
        PyTuple_SET_ITEM(both, 0, given[0] ? Py_NewRef(args[2]) : THPVariable_Wrap(codes));
        PyTuple_SET_ITEM(both, 1, given[1] ? Py_NewRef(args[3]) : THPVariable_Wrap(scales));
        return both;
    });
}

// project_rows(stream, x, weight, weight_scales, bias, x_scales, to_f32, out); to_f32: the type of a new out, 0 or 1, or -1 for x's
PyObject *project_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 8 || !bound) { PyErr_SetString(PyExc_TypeError, "project_rows takes 8 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *x = tensor(args[1]), *w = tensor(args[2]), *ws_ = tensor(args[3]), *bias = tensor(args[4]), *xs = tensor(args[5]), *given = tensor(args[7]);
        need(x && w && ws_);
        idf_project_args a{};
        const bool codes = x->scalar_type() == at::kChar;
        a.precision = codes ? IDF_PREC_I8 : precision(*x);
        need(codes == (xs != nullptr));
        a.x = matrix(*x, *x);
        need(!codes || ((uintptr_t)a.x.base % 16 == 0 && a.x.row_stride % 16 == 0));
        need((uintptr_t)w->data_ptr() % 16 == 0);
        need(x->size(1) <= INT_MAX - 16 && w->dim() == 2 && w->scalar_type() == at::kChar && w->device() == x->device() && w->is_contiguous() && w->size(0) <= INT_MAX);
        a.n_rows = x->size(0);
        a.cols = (int)x->size(1);
        a.n_out = (int)w->size(0);
        need(w->size(1) == (a.cols + 15) / 16 * 16);
        a.weights = static_cast<const int8_t *>(w->data_ptr());
        a.weight_scales = plain<float>(ws_, at::kFloat, a.n_out, *x);
        a.bias = plain<float>(bias, at::kFloat, a.n_out, *x);
        a.x_scales = plain<float>(xs, at::kFloat, a.n_rows, *x);
        const int64_t to_f32 = whole(args[6]);
        need(given ? to_f32 < 0 || given->scalar_type() == (to_f32 ? at::kFloat : at::kBFloat16) : !codes || to_f32 >= 0);
        const at::ScalarType type = given ? given->scalar_type() : to_f32 < 0 ? x->scalar_type() : to_f32 ? at::kFloat : at::kBFloat16;
        const c10::DeviceGuard guard(x->device());
        const at::Tensor out = given ? *given : at::empty({a.n_rows, a.n_out}, x->options().dtype(type));
        need(out.dim() == 2 && out.size(0) == a.n_rows && out.size(1) == a.n_out);
        a.out_precision = precision(out);
        a.out = matrix(out, *x);
        if (given) {
            const Reach to = reach(a.out, a.n_rows, a.n_out, out.element_size());
            need_apart(to, reach(a.x, a.n_rows, a.cols, x->element_size()));
            for (const at::Tensor *t : {w, ws_, bias, xs})
                if (t) need_apart(to, reach(*t));
        }
        at::Tensor ws;
        int rc = with_workspace(fn.project_workspace, a, *x, ws);
        if (rc == IDF_OK) rc = call(fn.project, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given});
        return given ? Py_NewRef(args[7]) : THPVariable_Wrap(out);
    });
}

// The four tensors of a ring; fills in sizes that the first one has.
template <class A> void nibble_ring(A &a, PyObject *const *args, const at::Tensor *like)
{
    const at::Tensor *t[4];
    for (int i = 0; i < 4; ++i) {
        t[i] = tensor(args[i]);
        need(t[i] && t[i]->scalar_type() == at::kByte && t[i]->is_cuda() && t[i]->is_contiguous() && t[i]->dim() == 4 && (!like || t[i]->device() == like->device()));
        need(t[i]->device() == t[0]->device());
        for (int d = 0; d < 3; ++d) need(t[i]->size(d) == t[0]->size(d));
        need(t[i]->size(3) <= 1024 && t[i]->size(3) * (i % 2 ? 16 : 1) == t[0]->size(3));
    }
    need(t[0]->size(0) <= INT_MAX && t[0]->size(1) <= INT_MAX);
    a.n_streams = (int)t[0]->size(0);
    a.heads_kv = (int)t[0]->size(1);
    a.slots = t[0]->size(2);
    a.head_dim = 2 * (int)t[0]->size(3);
    a.ring = idf_nibble_ring{static_cast<uint8_t *>(t[0]->data_ptr()), static_cast<uint8_t *>(t[1]->data_ptr()), static_cast<uint8_t *>(t[2]->data_ptr()), static_cast<uint8_t *>(t[3]->data_ptr())};
}

// Where segments of a ring's streams begin, and which streams they are of.
template <class A> void places(A &a, const at::Tensor &like, PyObject *starts_, PyObject *offsets_, PyObject *max_tokens, PyObject *ids_)
{
    const at::Tensor *starts = tensor(starts_), *offsets = tensor(offsets_), *ids = tensor(ids_);
    const int64_t count = ids ? ids->numel() : starts ? starts->numel() : a.n_streams;
    segments(a, like, offsets, max_tokens, count);
    need(!(ids || starts) || a.n_segments == count);
    a.starts = plain<int64_t>(starts, at::kLong, a.n_segments, like);
    a.stream_ids = plain<int32_t>(ids, at::kInt, a.n_segments, like);
}

// nibble_append(stream, k, v, four of the ring, starts, sinks, frequencies, interleaved, amplitude, k_weight, eps, offsets, max_tokens, stream_ids)
PyObject *nibble_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 17 || !bound) { PyErr_SetString(PyExc_TypeError, "nibble_append takes 17 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *k = tensor(args[1]), *v = tensor(args[2]), *freq = tensor(args[9]);
        need(k && v);
        idf_nibble_append_args a{};
        a.precision = precision(*k);
        a.k = rows(*k, *k, false);
        a.v = rows(*v, *k, false);
        nibble_ring(a, args + 3, k);
        need(k->sizes() == v->sizes() && k->size(1) == a.heads_kv && k->size(2) == a.head_dim && (!freq || freq->numel() <= 1024));
        a.n_tokens = k->size(0);
        places(a, *k, args[7], args[14], args[15], args[16]);
        a.sinks = small(args[8]);
        a.frequencies = plain<double>(freq, at::kDouble, -1, *k);
        a.rotary_dim = freq ? 2 * (int)freq->numel() : 0;
        a.interleaved = small(args[10]);
        a.amplitude = real(args[11]);
        a.k_weight = plain<float>(tensor(args[12]), at::kFloat, a.head_dim, *k);
        a.eps = real(args[13]);
        const c10::DeviceGuard guard(k->device());
        const int rc = call(fn.nibble_append, a, stream);
        if (rc == IDF_OK) written({tensor(args[3]), tensor(args[4]), tensor(args[5]), tensor(args[6])});
        return PyLong_FromLong(rc);
    });
}

// nibble_attend(stream, q, four of the ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out)
PyObject *nibble_attend(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 14 || !bound) { PyErr_SetString(PyExc_TypeError, "nibble_attend takes 14 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *q = tensor(args[1]);
        need(q);
        idf_nibble_attend_args a{};
        a.precision = precision(*q);
        a.q = rows(*q, *q, true);
        nibble_ring(a, args + 2, q);
        need(q->size(1) <= INT_MAX && q->size(2) == a.head_dim);
        a.heads_q = (int)q->size(1);
        a.n_tokens = q->size(0);
        places(a, *q, args[6], args[10], args[11], args[12]);
        a.window = small(args[7]);
        a.sinks = small(args[8]);
        a.scale = args[9] == Py_None ? (float)(1.0 / std::sqrt((double)a.head_dim)) : (float)real(args[9]);
        const c10::DeviceGuard guard(q->device());
        const at::Tensor *given = tensor(args[13]);
        const at::Tensor out = output(given, q->sizes(), *q);
        a.out = rows(out, *q, true);
        at::Tensor ws;
        int rc = with_workspace(fn.nibble_workspace, a, *q, ws);
        if (rc == IDF_OK) rc = call(fn.nibble_attend, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given});
        return args[13] != Py_None ? Py_NewRef(args[13]) : THPVariable_Wrap(out);
    });
}

// nibble_values(stream, four of the ring, to_f32)
PyObject *nibble_values(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6 || !bound) { PyErr_SetString(PyExc_TypeError, "nibble_values takes 6 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        idf_nibble_values_args a{};
        nibble_ring(a, args + 1, nullptr);
        const at::Tensor &like = *tensor(args[1]);
        a.precision = whole(args[5]) ? IDF_PREC_F32 : IDF_PREC_BF16;
        const c10::DeviceGuard guard(like.device());
        at::Tensor out[2];
        for (at::Tensor &t : out) t = at::empty({a.n_streams, a.slots, a.heads_kv, a.head_dim}, like.options().dtype(a.precision == IDF_PREC_F32 ? at::kFloat : at::kBFloat16));
        a.k = out[0].data_ptr();
        a.v = out[1].data_ptr();
        const int rc = call(fn.nibble_values, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        PyObject *both = PyTuple_New(2);
        if (!both) throw Unusual();
        for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(both, i, THPVariable_Wrap(out[i]));
        return both;
    });
}

// States [stream][channel] that a call of the recurrence goes from and to.
int64_t states(const at::Tensor *in, const at::Tensor *to, int64_t channels, const at::Tensor &like)
{
    int64_t streams = -1;
    for (const at::Tensor *s : {in, to}) {
        if (!s) continue;
        need(s->dim() == 2 && s->scalar_type() == at::kFloat && s->device() == like.device() && s->is_contiguous() && s->size(1) == channels && s->size(0) <= INT_MAX);
        need(streams < 0 || streams == s->size(0));
        streams = s->size(0);
    }
    return streams;
}

// Tokens, segments and streams of a call of the recurrence.
template <class A> void gate_segments(A &a, const at::Tensor &x, int64_t streams, PyObject *offsets, PyObject *max_tokens, PyObject *n_segments, PyObject *ids_)
{
    const at::Tensor *ids = tensor(ids_);
    const bool told = ids || n_segments != Py_None;
    const int64_t count = ids ? ids->numel() : n_segments != Py_None ? whole(n_segments) : streams >= 0 ? streams : 1;
    segments(a, x, tensor(offsets), max_tokens, count);
    need(!told || a.n_segments == count);
    a.n_streams = streams >= 0 ? (int)streams : a.n_segments;
    a.stream_ids = plain<int32_t>(ids, at::kInt, a.n_segments, x);
}

// gate_scan(stream, x, gates, state, state_out, offsets, max_tokens, n_segments, stream_ids, out, marks): out; marks True: new ones, (out, marks)
PyObject *gate_scan(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 11 || !bound) { PyErr_SetString(PyExc_TypeError, "gate_scan takes 11 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *x = tensor(args[1]), *g = tensor(args[2]), *in = tensor(args[3]), *to = tensor(args[4]), *given = tensor(args[9]);
        const at::Tensor *marks = args[10] == Py_True ? nullptr : tensor(args[10]);
        need(x && g && x->sizes() == g->sizes() && g->scalar_type() == x->scalar_type());
        idf_gate_scan_args a{};
        a.precision = precision(*x);
        a.x = matrix(*x, *x);
        a.gates = matrix(*g, *x);
        need(x->size(1) <= INT_MAX);
        a.channels = (int)x->size(1);
        a.n_tokens = x->size(0);
        gate_segments(a, *x, states(in, to, a.channels, *x), args[5], args[6], args[7], args[8]);
        a.state_in = in ? static_cast<const float *>(in->data_ptr()) : nullptr;
        a.state_out = to ? static_cast<float *>(to->data_ptr()) : nullptr;
        const c10::DeviceGuard guard(x->device());
        const at::Tensor out = output(given, x->sizes(), *x);
        need(out.scalar_type() == x->scalar_type());
        a.out = matrix(out, *x);
        a.clear_rows = !given && a.offsets;        // (a new result holds nothing yet)
        if (given)
            for (const idf_rows *r : {&a.x, &a.gates})
                need_apart(reach(a.out, a.n_tokens, a.channels, x->element_size()), reach(*r, a.n_tokens, a.channels, x->element_size()));
        at::Tensor fresh, ws;
        int rc = IDF_OK;
        if (marks || args[10] == Py_True) {
            size_t bytes = 0;
            rc = fn.gate_marks(&a, &bytes);
            if (rc != IDF_OK) return PyLong_FromLong(rc);
            if (!marks) { fresh = at::empty({(int64_t)bytes / 4}, x->options().dtype(at::kFloat)); marks = &fresh; }
            a.marks = plain<float>(marks, at::kFloat, (int64_t)bytes / 4, *x);
        }
        rc = with_workspace(fn.gate_workspace, a, *x, ws);
        if (rc == IDF_OK) rc = call(fn.gate, a, stream);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        written({given, to, marks == &fresh ? nullptr : marks});
        PyObject *got = given ? Py_NewRef(args[9]) : THPVariable_Wrap(out);
        if (args[10] != Py_True || !got) return got;
        PyObject *both = PyTuple_New(2);
        if (!both) { Py_DECREF(got); throw Unusual(); }
        PyTuple_SET_ITEM(both, 0, got);
        PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(fresh));
        return both;
    });
}

// Gradients of the recurrence; segments are those of a.
struct GateGradients { at::Tensor x, gates, state; };
int gate_gradients(idf_gate_scan_backward_args &a, const at::Tensor &x, const at::Tensor &g, const at::Tensor &marks, const at::Tensor *grad, const at::Tensor *end, void *stream, GateGradients &to)
{
    a.precision = precision(x);
    a.x = matrix(x, x);
    need(g.sizes() == x.sizes() && g.scalar_type() == x.scalar_type());
    a.gates = matrix(g, x);
    a.channels = (int)x.size(1);
    a.n_tokens = x.size(0);
    if (grad) {
        need(grad->sizes() == x.sizes() && grad->scalar_type() == x.scalar_type());
        a.grad_out = matrix(*grad, x);
    }
    idf_gate_scan_args f{};
    f.precision = a.precision; f.channels = a.channels; f.n_tokens = a.n_tokens; f.max_tokens = a.max_tokens; f.n_segments = a.n_segments; f.n_streams = a.n_streams;
    f.offsets = a.offsets; f.stream_ids = a.stream_ids;
    size_t bytes = 0;
    int rc = fn.gate_marks(&f, &bytes);
    if (rc != IDF_OK) return rc;
    a.marks = plain<float>(&marks, at::kFloat, (int64_t)bytes / 4, x);
    a.grad_end = end ? static_cast<const float *>(end->data_ptr()) : nullptr;
    // (streams that no segment is of have no gradient)
    const auto state = x.options().dtype(at::kFloat);
    to = {at::empty(x.sizes(), x.options()), at::empty(x.sizes(), x.options()), !a.stream_ids && a.n_streams == a.n_segments ? at::empty({a.n_streams, a.channels}, state) : at::zeros({a.n_streams, a.channels}, state)};
    a.grad_x = matrix(to.x, x);
    a.grad_gates = matrix(to.gates, x);
    a.grad_state = static_cast<float *>(to.state.data_ptr());
    at::Tensor ws;
    rc = with_workspace(fn.gate_back_workspace, a, x, ws);
    return rc == IDF_OK ? fn.gate_back(&a, stream) : rc;
}

// gate_scan_backward(stream, x, gates, marks, grad_out, grad_end, offsets, max_tokens, n_segments, stream_ids, n_streams): gradients of x, gates and states
PyObject *gate_scan_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 11 || !bound) { PyErr_SetString(PyExc_TypeError, "gate_scan_backward takes 11 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        void *stream = reinterpret_cast<void *>((uintptr_t)whole(args[0]));
        const at::Tensor *x = tensor(args[1]), *g = tensor(args[2]), *marks = tensor(args[3]), *grad = tensor(args[4]), *end = tensor(args[5]);
        need(x && g && marks && x->dim() == 2 && x->size(1) <= INT_MAX && x->sizes() == g->sizes() && g->scalar_type() == x->scalar_type());
        idf_gate_scan_backward_args a{};
        a.n_tokens = x->size(0);
        const int64_t told = args[10] == Py_None ? -1 : whole(args[10]), have = states(end, nullptr, x->size(1), *x);
        need(told < 0 || have < 0 || told == have);
        gate_segments(a, *x, have >= 0 ? have : told, args[6], args[7], args[8], args[9]);
        const c10::DeviceGuard guard(x->device());
        GateGradients to;
        const int rc = gate_gradients(a, *x, *g, *marks, grad, end, stream, to);
        if (rc != IDF_OK) return PyLong_FromLong(rc);
        PyObject *all = PyTuple_New(3);
        if (!all) throw Unusual();
        PyTuple_SET_ITEM(all, 0, THPVariable_Wrap(to.x));
        PyTuple_SET_ITEM(all, 1, THPVariable_Wrap(to.gates));
        PyTuple_SET_ITEM(all, 2, THPVariable_Wrap(to.state));
        return all;
    });
}

bool captured(void *stream)
{
    int capturing = 0;
    return fn.is_capturing(stream, &capturing) != 0 || capturing;
}

// The recurrence as torch's gradients go through it.  The backward pass runs on the stream of the forward one, as torch has it.
struct GateScan : torch::autograd::Function<GateScan> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext *ctx, const at::Tensor &x, const at::Tensor &gates, const std::optional<at::Tensor> &state,
                                                  const std::optional<at::Tensor> &offsets, int64_t max_tokens, int64_t segments, int64_t stream)
    {
        idf_gate_scan_args a{};
        a.precision = precision(x);
        a.channels = (int)x.size(1);
        a.n_tokens = x.size(0);
        a.max_tokens = max_tokens;
        a.n_segments = a.n_streams = (int)segments;
        a.offsets = offsets ? plain<int64_t>(&*offsets, at::kLong, segments + 1, x) : nullptr;
        a.x = matrix(x, x);
        a.gates = matrix(gates, x);
        a.state_in = state ? static_cast<const float *>(state->data_ptr()) : nullptr;
        const at::Tensor out = at::empty(x.sizes(), x.options()), end = at::empty({segments, x.size(1)}, x.options().dtype(at::kFloat));
        a.out = matrix(out, x);
        a.state_out = static_cast<float *>(end.data_ptr());
        a.clear_rows = a.offsets != nullptr;
        size_t bytes = 0;
        need(fn.gate_marks(&a, &bytes) == IDF_OK);
        const at::Tensor marks = at::empty({(int64_t)bytes / 4}, x.options().dtype(at::kFloat));
        a.marks = static_cast<float *>(marks.data_ptr());
        at::Tensor ws;
        need(with_workspace(fn.gate_workspace, a, x, ws) == IDF_OK && fn.gate(&a, reinterpret_cast<void *>((uintptr_t)stream)) == IDF_OK);
        ctx->save_for_backward({x, gates, marks, offsets ? *offsets : at::Tensor()});
        ctx->saved_data["max_tokens"] = max_tokens;
        ctx->saved_data["segments"] = segments;
        ctx->saved_data["tokens"] = x.size(0);
        ctx->saved_data["channels"] = x.size(1);
        ctx->saved_data["stream"] = stream;
        ctx->saved_data["has_state"] = state.has_value();
        ctx->set_materialize_grads(false);
        return {out, end};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext *ctx, torch::autograd::variable_list grads)
    {
        torch::autograd::variable_list answer(7);
        if (!grads[0].defined() && !grads[1].defined()) return answer;
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &x = saved[0], &offsets = saved[3];
        void *stream = reinterpret_cast<void *>((uintptr_t)ctx->saved_data["stream"].toInt());
        if (captured(stream))
            throw std::runtime_error("gate_scan_recorded's backward pass while a stream is captured: gate_scan_backward can be captured");
        const bool twice = c10::GradMode::is_enabled();
        GateGradients to;
        {
            const c10::AutoGradMode off(false);
            const c10::DeviceGuard guard(x.device());
            const at::Tensor grad = grads[0].defined() ? grads[0].contiguous() : at::Tensor(), end = grads[1].defined() ? grads[1].contiguous() : at::Tensor();
            idf_gate_scan_backward_args a{};
            a.max_tokens = ctx->saved_data["max_tokens"].toInt();
            a.n_segments = a.n_streams = (int)ctx->saved_data["segments"].toInt();
            // (what was saved may come back by way of a hook of the program's)
            need(x.dim() == 2 && x.size(0) == ctx->saved_data["tokens"].toInt() && x.size(1) == ctx->saved_data["channels"].toInt());
            a.offsets = offsets.defined() ? plain<int64_t>(&offsets, at::kLong, a.n_segments + 1, x) : nullptr;
            // (rows that lie too far apart, which the forward call did not take either, are no case here)
            if (gate_gradients(a, x, saved[1], saved[2], grad.defined() ? &grad : nullptr, end.defined() ? &end : nullptr, stream, to) != IDF_OK)
                throw std::runtime_error("gate_scan_backward was refused");
        }
        answer[0] = to.x; answer[1] = to.gates; answer[2] = to.state;
        if (twice) {                               // (gradients of these are refused, when somebody asks for them)
            torch::autograd::variable_list of(answer.begin(), answer.begin() + 3);
            for (at::Tensor &t : of) t.set_requires_grad(true);
            auto refusal = std::make_shared<torch::autograd::DelayedError>("gate_scan_recorded has no gradients of gradients", 3);
            of = (*refusal)(std::move(of));
            std::copy(of.begin(), of.end(), answer.begin());
        }
        // (tensors alone are counted: a state that was not given is none)
        const size_t given = ctx->saved_data["has_state"].toBool() ? 3 : 2;
        for (size_t i = 0; i < 3; ++i)
            if (i >= given || !ctx->needs_input_grad(i)) answer[i] = at::Tensor();
        return answer;
    }
};

// gate_scan_recorded(stream, x, gates, state, offsets, max_tokens, n_segments): (out, states behind the segments)
PyObject *gate_scan_recorded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 7 || !bound) { PyErr_SetString(PyExc_TypeError, "gate_scan_recorded takes 7 arguments"); return nullptr; }
    return entry([&]() -> PyObject * {
        const int64_t stream = whole(args[0]);
        need(!captured(reinterpret_cast<void *>((uintptr_t)stream)));           // (refused there)
        const at::Tensor *x = recorded_tensor(args[1]), *g = recorded_tensor(args[2]), *state = recorded_tensor(args[3]), *offsets = tensor(args[4]);
        need(x && g && x->dim() == 2 && x->size(1) <= INT_MAX && x->sizes() == g->sizes() && g->scalar_type() == x->scalar_type());
        (void)precision(*x);
        (void)matrix(*x, *x);
        (void)matrix(*g, *x);
        idf_gate_scan_args a{};
        a.n_tokens = x->size(0);
        gate_segments(a, *x, states(state, nullptr, x->size(1), *x), args[4], args[5], args[6], Py_None);
        need(!state || state->size(0) == a.n_segments);
        const c10::DeviceGuard guard(x->device());
        const auto got = GateScan::apply(*x, *g, state ? std::optional<at::Tensor>(*state) : std::nullopt, offsets ? std::optional<at::Tensor>(*offsets) : std::nullopt, a.max_tokens,
                                         (int64_t)a.n_segments, stream);
        PyObject *both = PyTuple_New(2);
        if (!both) throw Unusual();
        for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(both, i, THPVariable_Wrap(got[i]));
        return both;
    });
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", FAST(bind), "the addresses of the library's functions"},
    {"norm_rotate", FAST(norm_rotate), "idf_norm_rotate on tensors"},
    {"window_attend", FAST(window_attend), "idf_window_attend on tensors"},
    {"decay_attend", FAST(decay_attend), "idf_decay_attend on tensors"},
    {"quantize_rows", FAST(quantize_rows), "idf_quantize_rows on tensors"},
    {"project_rows", FAST(project_rows), "idf_project_rows on tensors"},
    {"nibble_append", FAST(nibble_append), "idf_nibble_append on tensors"},
    {"nibble_attend", FAST(nibble_attend), "idf_nibble_attend on tensors"},
    {"nibble_values", FAST(nibble_values), "idf_nibble_values on tensors"},
    {"gate_scan", FAST(gate_scan), "idf_gate_scan on tensors"},
    {"gate_scan_backward", FAST(gate_scan_backward), "idf_gate_scan_backward on tensors"},
    {"gate_scan_recorded", FAST(gate_scan_recorded), "both of them as torch's gradients go through them"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tokens", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tokens() { return PyModule_Create(&module); }
