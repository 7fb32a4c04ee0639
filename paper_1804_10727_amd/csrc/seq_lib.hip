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

template <class Args>
int check_segments(const Args &a)
{
    if (!precision_ok(a.precision)) return fail(IDF_EUNSUPPORTED, "precision %d: float32 and bfloat16 only", a.precision);
    if (a.heads_q < 1 || a.heads_kv < 1 || a.heads_q > kMostHeads || a.heads_q % a.heads_kv)
        return fail(IDF_EINVAL, "%d query heads on %d key/value heads", a.heads_q, a.heads_kv);
    if (a.n_tokens < 0 || a.n_tokens > INT_MAX || a.max_tokens < 0 || a.max_tokens > INT_MAX || a.n_segments < 0 || a.n_streams < 0)
        return fail(IDF_EINVAL, "%lld tokens, %lld in a segment, %d segments, %d streams", (long long)a.n_tokens, (long long)a.max_tokens, a.n_segments, a.n_streams);
    if (a.n_segments > kMostSegments) return fail(IDF_EUNSUPPORTED, "%d segments: at most %d in a call", a.n_segments, kMostSegments);
    if (!a.offsets && (int64_t)a.n_segments * a.max_tokens != a.n_tokens)
        return fail(IDF_EINVAL, "%lld tokens are not %d segments of %lld", (long long)a.n_tokens, a.n_segments, (long long)a.max_tokens);
    if ((int64_t)a.n_segments * a.heads_kv > kMostPairs)
        return fail(IDF_EUNSUPPORTED, "%d segments with %d heads: more than a launch takes", a.n_segments, a.heads_kv);
    if (!a.stream_ids && a.n_segments > a.n_streams) return fail(IDF_EINVAL, "%d segments of %d streams", a.n_segments, a.n_streams);
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

}  // extern "C"
