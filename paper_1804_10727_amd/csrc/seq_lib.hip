// Entry points of the operators that mix the tokens of streams: checks of arguments; what is launched is decided in the k_*.hip files.
#include <algorithm>
#include <climits>
#include <cmath>

#include "idf.h"
#include "idf_kernels.h"

using namespace idf;

namespace {

constexpr int kMostSegments = 65535;               // a launch's second or third axis
constexpr int kMostHeads = 1024;
constexpr int64_t kMostPairs = 1 << 23;            // segments times key/value heads (times columns by 64): a launch's first axis, 2^32 threads
constexpr int64_t kMostRows = 65535 * 128;         // query rows of a segment and key/value head: its second
constexpr int64_t kMostTokens = 1 << 30;           // of a segment: places behind its last chunk are counted in 32 bits
constexpr int64_t kMostByToken = 1 << 23;          // the same where tokens follow each other one by one: more would hold the machine for a minute
constexpr int64_t kMostSlots = 1 << 30;            // lists of keys are counted in 32 bits
constexpr int64_t kMostNibbleSlots = 1 << 24;           // places in a ring of 4-bit blocks: bytes of a head in 32 bits
constexpr int kMostCols = 65536;                   // sums of so many products of 8-bit codes stay below 2^31
constexpr int kMostOuts = 1 << 24;
constexpr int64_t kMostMatrixRows = (1 << 24) - 1; // a workgroup each: 2^32 threads
constexpr int64_t kMostOutputs = (int64_t)1 << 37;  // of a product: 2^21 tiles of 256 x 256, which products that large go in
constexpr int64_t kMostAppended = 1 << 26;        // tokens of a segment that go to a ring of 4-bit blocks, eight to a workgroup: a launch's first axis again
constexpr int64_t kMostRowStride = 1 << 25;        // sixteen rows lie within 32 bits of bytes
constexpr int kMostChannels = 1 << 20;

bool precision_ok(int p) { return p == IDF_PREC_F32 || p == IDF_PREC_BF16; }

// Whether two rows of dim values, at token * token_stride + head * head_stride, share a place: for each distance between heads the two distances
// between tokens that come nearest to it.  (Signs do not matter: tokens may be as far apart in either direction.)
bool rows_overlap(const idf_tokens &t, int64_t n_tokens, int heads, int dim)
{
    using Wide = __int128;
    const Wide token = t.token_stride < 0 ? -(Wide)t.token_stride : (Wide)t.token_stride, head = t.head_stride < 0 ? -(Wide)t.head_stride : (Wide)t.head_stride;
    if ((n_tokens > 1 && token < dim) || (heads > 1 && head < dim)) return true;
    if (n_tokens <= 1 || heads <= 1 || token >= (heads - 1) * head + dim || head >= (n_tokens - 1) * token + dim) return false;
    for (int h = 1; h < heads; ++h) {
        const Wide at = h * head, before = std::min<Wide>(at / token, n_tokens - 1);
        if (at - before * token < dim) return true;
        if (before + 1 < n_tokens && (before + 1) * token - at < dim) return true;
    }
    return false;
}

// A matrix of tokens that 16-byte pieces are read from or written to.
int check_tokens(const char *what, const idf_tokens &t, int precision, bool out, int64_t n_tokens, int heads, int dim)
{
    const int eb = precision == IDF_PREC_F32 ? 4 : 2, vl = 16 / eb;
    if (!t.base) return fail(IDF_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)t.base % 16 || t.token_stride % vl || t.head_stride % vl)
        return fail(IDF_EUNSUPPORTED, "%s: base and strides have to be multiples of 16 bytes", what);
    if (out && rows_overlap(t, n_tokens, heads, dim)) return fail(IDF_EINVAL, "%s: rows overlap", what);
    return IDF_OK;
}

// Tokens, segments and streams of a call.
template <class Args>
int check_packing(const Args &a)
{
    if (!precision_ok(a.precision)) return fail(IDF_EUNSUPPORTED, "precision %d: float32 and bfloat16 only", a.precision);
    if (a.n_tokens < 0 || a.n_tokens > INT_MAX || a.max_tokens < 0 || a.max_tokens > INT_MAX || a.n_segments < 0 || a.n_streams < 0)
        return fail(IDF_EINVAL, "%lld tokens, %lld in a segment, %d segments, %d streams", (long long)a.n_tokens, (long long)a.max_tokens, a.n_segments, a.n_streams);
    if (a.n_segments > kMostSegments) return fail(IDF_EUNSUPPORTED, "%d segments: at most %d in a call", a.n_segments, kMostSegments);
    if (!a.offsets && (int64_t)a.n_segments * a.max_tokens != a.n_tokens)
        return fail(IDF_EINVAL, "%lld tokens are not %d segments of %lld", (long long)a.n_tokens, a.n_segments, (long long)a.max_tokens);
    if (!a.stream_ids && a.n_segments > a.n_streams) return fail(IDF_EINVAL, "%d segments of %d streams", a.n_segments, a.n_streams);
    return IDF_OK;
}

template <class Args>
int check_segments(const Args &a)
{
    if (!precision_ok(a.precision)) return fail(IDF_EUNSUPPORTED, "precision %d: float32 and bfloat16 only", a.precision);
    if (a.heads_q < 1 || a.heads_kv < 1 || a.heads_q > kMostHeads || a.heads_q % a.heads_kv)
        return fail(IDF_EINVAL, "%d query heads on %d key/value heads", a.heads_q, a.heads_kv);
    if (int rc = check_packing(a)) return rc;
    if ((int64_t)a.n_segments * a.heads_kv > kMostPairs)
        return fail(IDF_EUNSUPPORTED, "%d segments with %d heads: more than a launch takes", a.n_segments, a.heads_kv);
    if (!(a.scale > 0.f) || std::isinf(a.scale)) return fail(IDF_EINVAL, "scale %g", (double)a.scale);
    return IDF_OK;
}

int check_window(const idf_window_args *a)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_segments(*a)) return rc;
    if (longest(*a) * (a->heads_q / a->heads_kv) > kMostRows)
        return fail(IDF_EUNSUPPORTED, "segments of up to %lld tokens with %d heads on %d: more than a launch takes", (long long)longest(*a), a->heads_q, a->heads_kv);
    const int vl = a->precision == IDF_PREC_F32 ? 4 : 8;
    if (a->head_dim < vl || a->head_dim > 256 || a->head_dim % vl) return fail(IDF_EUNSUPPORTED, "heads of %d values", a->head_dim);
    if (a->window < 1 || a->sinks < 0) return fail(IDF_EINVAL, "a window of %d tokens and %d first ones", a->window, a->sinks);
    if (!a->k_ring != !a->v_ring) return fail(IDF_EINVAL, "a ring of keys or values alone");
    if (a->k_ring) {
        if (a->slots > kMostSlots || a->slots - a->sinks < a->window)
            return fail(IDF_EINVAL, "%lld slots for a window of %d tokens and %d first ones", (long long)a->slots, a->window, a->sinks);
        if (((uintptr_t)a->k_ring | (uintptr_t)a->v_ring) % 16) return fail(IDF_EUNSUPPORTED, "rings have to be 16-byte aligned");
    }
    return IDF_OK;
}

int check_decay(const idf_decay_args *a)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_segments(*a)) return rc;
    const int vl = a->precision == IDF_PREC_F32 ? 4 : 8;
    if (a->dim_k < vl || a->dim_k > 256 || a->dim_k % vl || a->dim_v < vl || a->dim_v % vl || a->dim_v > 4096)
        return fail(IDF_EUNSUPPORTED, "heads of %d and %d values", a->dim_k, a->dim_v);
    if (longest(*a) > (a->dim_k > 128 ? kMostByToken : kMostTokens))
        return fail(IDF_EUNSUPPORTED, "segments of up to %lld tokens with keys of %d values", (long long)longest(*a), a->dim_k);
    if ((int64_t)a->n_segments * a->heads_kv * ((a->dim_v + 63) / 64) > kMostPairs)
        return fail(IDF_EUNSUPPORTED, "%d segments with %d heads of %d values: more than a launch takes", a->n_segments, a->heads_kv, a->dim_v);
    if (((uintptr_t)a->state_in | (uintptr_t)a->state_out) % 16) return fail(IDF_EUNSUPPORTED, "states have to be 16-byte aligned");
    return IDF_OK;
}

// ---- in few bits ----

// A matrix that is read or written value by value, or in larger pieces where it lies that way.
int check_rows(const char *what, const idf_rows &r, int value_bytes, bool out, int64_t n_rows, int cols)
{
    if (!r.base) return fail(IDF_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)r.base % value_bytes) return fail(IDF_EINVAL, "%s: not aligned to its values", what);
    if (r.row_stride < 0 || r.row_stride > kMostRowStride) return fail(IDF_EUNSUPPORTED, "%s: rows %lld values apart", what, (long long)r.row_stride);
    if (out && n_rows > 1 && r.row_stride < cols) return fail(IDF_EINVAL, "%s: rows overlap", what);
    return IDF_OK;
}

int bytes_of(int precision) { return precision == IDF_PREC_F32 ? 4 : precision == IDF_PREC_BF16 ? 2 : 1; }

int check_quantize(const idf_quantize_args *a)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (!precision_ok(a->precision)) return fail(IDF_EUNSUPPORTED, "precision %d: float32 and bfloat16 only", a->precision);
    if (a->cols < 1 || a->cols > kMostCols) return fail(IDF_EUNSUPPORTED, "rows of %d values", a->cols);
    if (a->n_rows < 0 || a->n_rows > kMostMatrixRows) return fail(IDF_EINVAL, "%lld rows", (long long)a->n_rows);
    if (a->n_rows == 0) return IDF_OK;
    if (int rc = check_rows("x", a->x, bytes_of(a->precision), false, a->n_rows, a->cols)) return rc;
    if (!a->codes || !a->scales) return fail(IDF_EINVAL, "codes or scales: null pointer");
    if ((uintptr_t)a->codes % 16) return fail(IDF_EUNSUPPORTED, "codes have to be 16-byte aligned");
    return IDF_OK;
}

int check_project(const idf_project_args *a)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (!precision_ok(a->precision) && a->precision != IDF_PREC_I8) return fail(IDF_EUNSUPPORTED, "precision %d", a->precision);
    if (!precision_ok(a->out_precision)) return fail(IDF_EUNSUPPORTED, "outputs of precision %d: float32 and bfloat16 only", a->out_precision);
    if (a->cols < 1 || a->cols > kMostCols || (a->precision == IDF_PREC_I8 && a->cols % 16)) return fail(IDF_EUNSUPPORTED, "rows of %d values", a->cols);
    if (a->n_out < 1 || a->n_out > kMostOuts) return fail(IDF_EUNSUPPORTED, "%d outputs", a->n_out);
    if (a->n_rows < 0 || a->n_rows > kMostMatrixRows) return fail(IDF_EINVAL, "%lld rows", (long long)a->n_rows);
    if (a->n_rows * a->n_out > kMostOutputs) return fail(IDF_EUNSUPPORTED, "%lld rows of %d outputs: more than a launch takes", (long long)a->n_rows, a->n_out);
    return IDF_OK;
}

int check_nibble(const idf_nibble_ring &r, int head_dim, int64_t slots, int sinks)
{
    if (head_dim < 32 || head_dim > 256 || head_dim % 32) return fail(IDF_EUNSUPPORTED, "heads of %d values", head_dim);
    if (!r.k_codes || !r.k_scales || !r.v_codes || !r.v_scales) return fail(IDF_EINVAL, "ring: null pointer");
    if (((uintptr_t)r.k_codes | (uintptr_t)r.v_codes) % 16) return fail(IDF_EUNSUPPORTED, "rings have to be 16-byte aligned");
    if (sinks < 0 || slots <= sinks) return fail(IDF_EINVAL, "%lld slots with %d first tokens", (long long)slots, sinks);
    if (slots > kMostNibbleSlots) return fail(IDF_EUNSUPPORTED, "%lld slots", (long long)slots);
    return IDF_OK;
}

int check_nibble_attend(const idf_nibble_attend_args *a)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_segments(*a)) return rc;
    if (longest(*a) * (a->heads_q / a->heads_kv) > kMostRows)
        return fail(IDF_EUNSUPPORTED, "segments of up to %lld tokens with %d heads on %d: more than a launch takes", (long long)longest(*a), a->heads_q, a->heads_kv);
    if (a->window < 1) return fail(IDF_EINVAL, "a window of %d tokens", a->window);
    if (int rc = check_nibble(a->ring, a->head_dim, a->slots, a->sinks)) return rc;
    if (a->slots - a->sinks < a->window + std::max<int64_t>(longest(*a), 1) - 1)
        return fail(IDF_EINVAL, "%lld slots for a window of %d tokens, %d first ones and segments of up to %lld", (long long)a->slots, a->window, a->sinks, (long long)longest(*a));
    return IDF_OK;
}

template <class Args>
int check_gate(const Args *a)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_packing(*a)) return rc;
    if (a->channels < 1 || a->channels > kMostChannels) return fail(IDF_EUNSUPPORTED, "%d channels", a->channels);
    if (longest(*a) > kMostTokens) return fail(IDF_EUNSUPPORTED, "segments of up to %lld tokens", (long long)longest(*a));
    if (gate_scan_tiles(*a) >= kMostPairs)
        return fail(IDF_EUNSUPPORTED, "%lld tokens in %d segments of %d channels: more than a launch takes", (long long)a->n_tokens, a->n_segments, a->channels);
    return IDF_OK;
}

// Rows that are none's where a call has no segments: as those behind one segment without tokens, which has no state.
idf_gate_scan_args without_segments(idf_gate_scan_args a)
{
    a.n_segments = 1;
    a.max_tokens = 0;
    a.offsets = nullptr;
    a.stream_ids = nullptr;
    a.state_out = nullptr;
    return a;
}
idf_gate_scan_backward_args without_segments(idf_gate_scan_backward_args a)
{
    a.n_segments = 1;
    a.max_tokens = 0;
    a.offsets = nullptr;
    a.stream_ids = nullptr;
    a.grad_state = nullptr;
    return a;
}

int check_workspace(void *p, size_t have, size_t need)
{
    if (need == 0) return IDF_OK;
    if (!p || have < need) return fail(IDF_ENOMEM, "a workspace of %zu bytes, %zu are needed", p ? have : (size_t)0, need);
    if ((uintptr_t)p % 256) return fail(IDF_EINVAL, "the workspace has to be 256-byte aligned");
    return IDF_OK;
}

}  // namespace

extern "C" {

int idf_rotary_frequencies(int rotary_dim, double base, int scaling, double factor, double trained, double fast, double slow,
                           double *frequencies, double *amplitude)
{
    if (!frequencies || !amplitude) return fail(IDF_EINVAL, "null argument");
    if (rotary_dim < 2 || rotary_dim > 256 || rotary_dim % 2) return fail(IDF_EINVAL, "rotation of %d values", rotary_dim);
    if (!(base > 1.0) || !std::isfinite(base)) return fail(IDF_EINVAL, "base %g", base);
    if (scaling < IDF_ROTARY_PLAIN || scaling > IDF_ROTARY_PARTS) return fail(IDF_EINVAL, "unknown scaling %d", scaling);
    if (scaling != IDF_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(IDF_EINVAL, "factor %g", factor);
    if (scaling == IDF_ROTARY_BASE && rotary_dim < 4) return fail(IDF_EINVAL, "a scaled base needs two pairs");
    if (scaling == IDF_ROTARY_PARTS && (!(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast) || !(trained > 0.0) || !std::isfinite(trained)))
        return fail(IDF_EINVAL, "from %g to %g turns in %g positions", slow, fast, trained);
    if (scaling == IDF_ROTARY_BASE) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
    *amplitude = scaling == IDF_ROTARY_PARTS ? 0.1 * std::log(factor) + 1.0 : 1.0;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rotary_dim);
        if (scaling == IDF_ROTARY_LINEAR) f /= factor;
        if (scaling == IDF_ROTARY_PARTS) {
            const double turns = f * trained / (2.0 * M_PI), keep = std::fmin(std::fmax((turns - slow) / (fast - slow), 0.0), 1.0);
            f = f * keep + f / factor * (1.0 - keep);
        }
        frequencies[i] = f;
    }
    return IDF_OK;
}

int idf_norm_rotate(const idf_norm_rotate_args *a, void *hip_stream)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (!precision_ok(a->precision)) return fail(IDF_EUNSUPPORTED, "precision %d: float32 and bfloat16 only", a->precision);
    if (a->heads_q < 0 || a->heads_k < 0 || a->heads_q > kMostHeads || a->heads_k > kMostHeads || a->heads_q + a->heads_k < 1)
        return fail(IDF_EINVAL, "%d query heads and %d key heads", a->heads_q, a->heads_k);
    if (a->head_dim < 1 || a->head_dim > 256) return fail(IDF_EUNSUPPORTED, "heads of %d values", a->head_dim);
    if (a->rotary_dim < 0 || a->rotary_dim > a->head_dim || a->rotary_dim % 2) return fail(IDF_EINVAL, "rotation of %d of %d values", a->rotary_dim, a->head_dim);
    if (a->n_tokens < 0 || a->n_tokens > INT_MAX) return fail(IDF_EINVAL, "%lld tokens", (long long)a->n_tokens);
    if (!(a->eps >= 0.f) || !std::isfinite(a->amplitude)) return fail(IDF_EINVAL, "eps %g, amplitude %g", (double)a->eps, a->amplitude);
    if (a->n_tokens == 0) return IDF_OK;
    const int eb = a->precision == IDF_PREC_F32 ? 4 : 2;
    const idf_tokens *each[] = {&a->q, &a->k, &a->q_out, &a->k_out};
    for (int i = 0; i < 4; ++i) {
        const int heads = i % 2 ? a->heads_k : a->heads_q;
        if (heads == 0) continue;
        const char *names[] = {"q", "k", "q_out", "k_out"};
        if (!each[i]->base) return fail(IDF_EINVAL, "%s: null pointer", names[i]);
        if ((uintptr_t)each[i]->base % eb) return fail(IDF_EINVAL, "%s: not aligned to its values", names[i]);
        if (i >= 2 && rows_overlap(*each[i], a->n_tokens, heads, a->head_dim)) return fail(IDF_EINVAL, "%s: rows overlap", names[i]);
    }
    if (a->rotary_dim && (!a->positions || !a->frequencies)) return fail(IDF_EINVAL, "a rotation without positions or frequencies");
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_norm_rotate(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "norm_rotate");
}

int idf_window_workspace(const idf_window_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_window(a)) return rc;
    *bytes = a->n_segments && a->n_tokens && a->max_tokens ? window_workspace(*a) : 0;
    return IDF_OK;
}

int idf_window_attend(const idf_window_args *a, void *hip_stream)
{
    if (int rc = check_window(a)) return rc;
    if (a->n_segments == 0 || a->n_tokens == 0 || a->max_tokens == 0) return IDF_OK;
    int rc = check_tokens("q", a->q, a->precision, false, a->n_tokens, a->heads_q, a->head_dim);
    if (!rc) rc = check_tokens("k", a->k, a->precision, false, a->n_tokens, a->heads_kv, a->head_dim);
    if (!rc) rc = check_tokens("v", a->v, a->precision, false, a->n_tokens, a->heads_kv, a->head_dim);
    if (!rc) rc = check_tokens("out", a->out, a->precision, true, a->n_tokens, a->heads_q, a->head_dim);
    if (!rc) rc = check_workspace(a->workspace, a->workspace_bytes, window_workspace(*a));
    if (rc) return rc;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_window(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "window_attend");
}

int idf_decay_workspace(const idf_decay_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_decay(a)) return rc;
    *bytes = decay_workspace(*a);
    return IDF_OK;
}

int idf_decay_attend(const idf_decay_args *a, void *hip_stream)
{
    if (int rc = check_decay(a)) return rc;
    const bool any = a->n_tokens && a->max_tokens;
    if (a->n_segments == 0 || (!any && !a->state_out)) return IDF_OK;
    if (!a->log_decay) return fail(IDF_EINVAL, "log_decay: null pointer");
    if (any) {
        int rc = check_tokens("q", a->q, a->precision, false, a->n_tokens, a->heads_q, a->dim_k);
        if (!rc) rc = check_tokens("k", a->k, a->precision, false, a->n_tokens, a->heads_kv, a->dim_k);
        if (!rc) rc = check_tokens("v", a->v, a->precision, false, a->n_tokens, a->heads_kv, a->dim_v);
        if (!rc) rc = check_tokens("out", a->out, a->precision, true, a->n_tokens, a->heads_q, a->dim_v);
        if (rc) return rc;
    }
    if (int rc = check_workspace(a->workspace, a->workspace_bytes, decay_workspace(*a))) return rc;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_decay(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "decay_attend");
}

int idf_quantize_rows(const idf_quantize_args *a, void *hip_stream)
{
    if (int rc = check_quantize(a)) return rc;
    if (a->n_rows == 0) return IDF_OK;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_quantize_rows(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "quantize_rows");
}

int idf_project_workspace(const idf_project_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_project(a)) return rc;
    *bytes = a->n_rows ? project_workspace(*a) : 0;
    return IDF_OK;
}

int idf_project_rows(const idf_project_args *a, void *hip_stream)
{
    if (int rc = check_project(a)) return rc;
    if (a->n_rows == 0) return IDF_OK;
    int rc = check_rows("x", a->x, bytes_of(a->precision), false, a->n_rows, a->cols);
    if (!rc) rc = check_rows("out", a->out, bytes_of(a->out_precision), true, a->n_rows, a->n_out);
    if (rc) return rc;
    if (!a->weights || !a->weight_scales) return fail(IDF_EINVAL, "weights or their scales: null pointer");
    if ((uintptr_t)a->weights % 16) return fail(IDF_EUNSUPPORTED, "weights have to be 16-byte aligned");
    if (a->precision == IDF_PREC_I8) {
        if (!a->x_scales) return fail(IDF_EINVAL, "x_scales: null pointer");
        if ((uintptr_t)a->x.base % 16 || a->x.row_stride % 16) return fail(IDF_EUNSUPPORTED, "x: base and rows have to be multiples of 16 bytes");
    }
    if (int rc = check_workspace(a->workspace, a->workspace_bytes, project_workspace(*a))) return rc;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_project_rows(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "project_rows");
}

int idf_nibble_append(const idf_nibble_append_args *a, void *hip_stream)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_packing(*a)) return rc;
    if (a->heads_kv < 1 || a->heads_kv > kMostHeads) return fail(IDF_EINVAL, "%d key/value heads", a->heads_kv);
    if (int rc = check_nibble(a->ring, a->head_dim, a->slots, a->sinks)) return rc;
    if (a->rotary_dim < 0 || a->rotary_dim > a->head_dim || a->rotary_dim % 2) return fail(IDF_EINVAL, "rotation of %d of %d values", a->rotary_dim, a->head_dim);
    if (!(a->eps >= 0.0) || !std::isfinite(a->amplitude)) return fail(IDF_EINVAL, "eps %g, amplitude %g", a->eps, a->amplitude);
    if (longest(*a) > kMostAppended) return fail(IDF_EUNSUPPORTED, "segments of up to %lld tokens", (long long)longest(*a));
    if (a->n_segments == 0 || longest(*a) == 0) return IDF_OK;
    const int eb = bytes_of(a->precision);
    for (const idf_tokens *t : {&a->k, &a->v}) {
        if (!t->base) return fail(IDF_EINVAL, "%s: null pointer", t == &a->k ? "k" : "v");
        if ((uintptr_t)t->base % eb) return fail(IDF_EINVAL, "%s: not aligned to its values", t == &a->k ? "k" : "v");
    }
    if (a->rotary_dim && !a->frequencies) return fail(IDF_EINVAL, "a rotation without frequencies");
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_nibble_append(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "nibble_append");
}

int idf_nibble_values(const idf_nibble_values_args *a, void *hip_stream)
{
    if (!a) return fail(IDF_EINVAL, "null argument");
    if (!precision_ok(a->precision)) return fail(IDF_EUNSUPPORTED, "precision %d: float32 and bfloat16 only", a->precision);
    if (a->heads_kv < 1 || a->heads_kv > kMostHeads || a->n_streams < 0) return fail(IDF_EINVAL, "%d key/value heads of %d streams", a->heads_kv, a->n_streams);
    if (int rc = check_nibble(a->ring, a->head_dim, a->slots, 0)) return rc;
    if (a->n_streams == 0) return IDF_OK;
    if (!a->k || !a->v) return fail(IDF_EINVAL, "k or v: null pointer");
    if (((uintptr_t)a->k | (uintptr_t)a->v) % 16) return fail(IDF_EUNSUPPORTED, "k and v have to be 16-byte aligned");
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_nibble_values(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "nibble_values");
}

int idf_nibble_attend_workspace(const idf_nibble_attend_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_nibble_attend(a)) return rc;
    *bytes = a->n_segments && longest(*a) ? nibble_attend_workspace(*a) : 0;
    return IDF_OK;
}

int idf_nibble_attend(const idf_nibble_attend_args *a, void *hip_stream)
{
    if (int rc = check_nibble_attend(a)) return rc;
    if (a->n_segments == 0 || longest(*a) == 0) return IDF_OK;
    int rc = check_tokens("q", a->q, a->precision, false, a->n_tokens, a->heads_q, a->head_dim);
    if (!rc) rc = check_tokens("out", a->out, a->precision, true, a->n_tokens, a->heads_q, a->head_dim);
    if (!rc) rc = check_workspace(a->workspace, a->workspace_bytes, nibble_attend_workspace(*a));
    if (rc) return rc;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_nibble_attend(*a, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "nibble_attend");
}

int idf_gate_scan_marks(const idf_gate_scan_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_gate(a)) return rc;
    *bytes = gate_scan_marks(a->n_tokens, a->n_segments, a->channels);
    return IDF_OK;
}

int idf_gate_scan_workspace(const idf_gate_scan_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_gate(a)) return rc;
    *bytes = a->n_segments ? gate_scan_workspace(*a) : 0;
    return IDF_OK;
}

int idf_gate_scan(const idf_gate_scan_args *a, void *hip_stream)
{
    if (int rc = check_gate(a)) return rc;
    const bool clear = a->clear_rows && a->n_tokens;
    if (!clear && (a->n_segments == 0 || (longest(*a) == 0 && !a->state_out))) return IDF_OK;
    const int eb = bytes_of(a->precision);
    if (a->n_segments && longest(*a)) {
        int rc = check_rows("x", a->x, eb, false, a->n_tokens, a->channels);
        if (!rc) rc = check_rows("gates", a->gates, eb, false, a->n_tokens, a->channels);
        if (rc) return rc;
    }
    if (clear || longest(*a))
        if (int rc = check_rows("out", a->out, eb, true, a->n_tokens, a->channels)) return rc;
    if ((uintptr_t)a->marks % 256) return fail(IDF_EINVAL, "marks have to be 256-byte aligned");
    if (((uintptr_t)a->state_in | (uintptr_t)a->state_out) % 4) return fail(IDF_EINVAL, "states: not aligned to their values");
    const idf_gate_scan_args b = a->n_segments ? *a : without_segments(*a);
    if (int rc = check_workspace(b.workspace, b.workspace_bytes, gate_scan_workspace(b))) return rc;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_gate_scan(b, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "gate_scan");
}

int idf_gate_scan_backward_workspace(const idf_gate_scan_backward_args *a, size_t *bytes)
{
    if (!bytes) return fail(IDF_EINVAL, "null argument");
    if (int rc = check_gate(a)) return rc;
    *bytes = a->n_segments ? gate_scan_workspace(*a) : 0;
    return IDF_OK;
}

int idf_gate_scan_backward(const idf_gate_scan_backward_args *a, void *hip_stream)
{
    if (int rc = check_gate(a)) return rc;
    if (a->n_tokens == 0 && (a->n_segments == 0 || !a->grad_state)) return IDF_OK;
    const int eb = bytes_of(a->precision);
    if (a->n_tokens) {
        int rc = IDF_OK;
        if (a->n_segments) {
            rc = check_rows("x", a->x, eb, false, a->n_tokens, a->channels);
            if (!rc) rc = check_rows("gates", a->gates, eb, false, a->n_tokens, a->channels);
            if (!rc && a->grad_out.base) rc = check_rows("grad_out", a->grad_out, eb, false, a->n_tokens, a->channels);
        }
        if (!rc) rc = check_rows("grad_x", a->grad_x, eb, true, a->n_tokens, a->channels);
        if (!rc) rc = check_rows("grad_gates", a->grad_gates, eb, true, a->n_tokens, a->channels);
        if (rc) return rc;
        if (a->n_segments && !a->marks) return fail(IDF_EINVAL, "marks: null pointer");
    }
    if ((uintptr_t)a->marks % 256) return fail(IDF_EINVAL, "marks have to be 256-byte aligned");
    if (((uintptr_t)a->grad_end | (uintptr_t)a->grad_state) % 4) return fail(IDF_EINVAL, "gradients of states: not aligned to their values");
    const idf_gate_scan_backward_args b = a->n_segments ? *a : without_segments(*a);
    if (int rc = check_workspace(b.workspace, b.workspace_bytes, gate_scan_workspace(b))) return rc;
    LaunchCtx lc;
    lc.st = (hipStream_t)hip_stream;
    const hipError_t e = launch_gate_scan_backward(b, lc);
    return e == hipSuccess ? IDF_OK : dev_fail(e, "gate_scan_backward");
}

}  // extern "C"
