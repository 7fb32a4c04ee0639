// A gated recurrence per channel and its gradients (idf_gate_scan, idf_gate_scan_backward).
//
//   h_t = a_t h_{t-1} + b_t x_t,  a = sigmoid(g), b = 1 - a.  Of a and b the smaller one, e / (1 + e) with e = exp(-|g|), is formed, and a step taken as
// h + b (x - h) or x + a (h - x): the larger one, rounded to a number near one, would be off in the same direction again and again where gates stay the
// same.  A part of a segment takes a state h to k h + n, with n what the part gives from nothing and k the product of its a, formed in the same way.
//   A lane has V neighbouring channels, a wave 64 V of them, and goes along the tokens 16 at a time with the next 16 on their way.  Segments are cut
// into parts along time where channels and segments are too few for the machine: their summaries first, then every part from the state that
// those before it give (x and gates are read twice then).  States within a segment before every 16th token are what the backward pass
// starts from: it forms the 16 states of a block anew, in registers, and goes back through them.
//   What infinite values, gates that are no numbers and gates beyond +-87 ask for is done where a block has any: once more for that block.
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

constexpr int kBlock = 16;                         // tokens that a wave has in registers
constexpr int kMostGroups = 64;                    // groups of parts of a segment: every part goes through the summaries of those before it
constexpr float kGateMost = 87.f;

// The smaller one of what a gate keeps and takes in, with the gate's sign: above zero it is what is taken in.
struct Gate {
    float s;
    __device__ __forceinline__ bool open() const { return __builtin_bit_cast(int, s) >= 0; }
    __device__ __forceinline__ float big() const { return 1.f - __builtin_fabsf(s); }
    __device__ __forceinline__ float take() const { return open() ? s : big(); }
};
template <int PREC> __device__ __forceinline__ Gate gate_of(float g)
{
    constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.9259629911e-8f, kLn2 = 0.6931471805599453f;
    const float size = __builtin_fabsf(g), p = size * -kLog2e;
    float t = __builtin_amdgcn_exp2f(p);
    // the rounding of the product counts by its size: 5e-6 of t where |g| is 87
    if (PREC == IDF_PREC_F32) t = __builtin_fmaf(t, kLn2 * (__builtin_fmaf(size, -kLog2e, -p) - size * kLog2eLow), t);
    const float r = __builtin_amdgcn_rcpf(1.f + t);
    return {__builtin_copysignf(t * r, g)};
}
__device__ __forceinline__ bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }

// The next state, and what flows to the token before it (l: what comes to this one).
__device__ __forceinline__ float step_of(const Gate &w, float x, float h) { return __builtin_fmaf(w.s, x - h, w.open() ? h : x); }
__device__ __forceinline__ float kept_of(const Gate &w, float l) { return __builtin_fmaf(-w.s, l, w.open() ? l : 0.f); }

// The same from the definition, for what the above would make no number: differences of infinite values, gates held to +-87.
template <int PREC> struct Slow {
    float keep, take;
    Gate w;
    __device__ __forceinline__ Slow(float g)
    {
        g = g > kGateMost ? kGateMost : g;         // (comparisons, so that what is not a number stays)
        g = g < -kGateMost ? -kGateMost : g;
        w = gate_of<PREC>(g);
        keep = w.open() ? w.big() : __builtin_fabsf(w.s);
        take = w.take();
    }
    __device__ __forceinline__ float step(float x, float h) const
    {
        const float next = step_of(w, x, h);
        return finite(next) ? next : keep * h + take * x;
    }
    __device__ __forceinline__ float kept(float l) const
    {
        const float next = kept_of(w, l);
        return finite(next) ? next : keep * l;
    }
};

// What a part makes of the state before it: keep * h + made.
struct Summary { float keep, made; };
__device__ __forceinline__ float through(const Summary &s, float h)
{
    return (s.keep == 0.f && !finite(h) ? h : s.keep * h) + s.made;            // (no product of gates is nothing, but 32 bits may say so)
}
__device__ __forceinline__ Summary join(const Summary &first, const Summary &then) { return {first.keep * then.keep, through(then, first.made)}; }

// How a call is cut: waves of a workgroup take parts of `part` tokens (a multiple of a block) behind each other, groups of them lie along y.
struct Cut {
    int part, waves, groups;
    int64_t rows;                                  // of summaries
    __device__ __host__ __forceinline__ int64_t span() const { return (int64_t)part * waves; }
};

// Summaries in the workspace, [row][1 + waves][2][channels], a row for each group that has tokens: of the group, then of its parts.  As with the marks a segment's
// first one goes by the tokens before it, so that there are as many as the tokens need and not as many as all segments would if they were as long as the longest.
__device__ __forceinline__ float *summary_at(void *workspace, const Cut &cut, int64_t row, int part, int channels)
{
    return (float *)workspace + ((row * (1 + cut.waves) + part) * 2) * channels;
}
__device__ __forceinline__ int64_t first_row(const Cut &cut, int64_t begin, int segment) { return (uint32_t)begin / (uint32_t)cut.span() + segment; }
// Behind them the states (or gradients) that segments begin with, [segment][channels]: the last part may write to where they came from before others have read.
__device__ __forceinline__ float *begin_at(void *workspace, const Cut &cut, int segment, int channels)
{
    return summary_at(workspace, cut, cut.rows, 0, channels) + (int64_t)segment * channels;
}
template <int V> __device__ __forceinline__ void put(float *to, int channels, int c, const Summary (&s)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) { to[c + v] = s[v].keep; to[channels + c + v] = s[v].made; }
}

// The state (or gradient) h goes through n summaries that lie `apart` floats from each other; several are asked for at once.
template <int V> __device__ __forceinline__ void go_through(const float *from, int64_t apart, int n, int channels, int c, float (&h)[V])
{
    constexpr int kAhead = 8;
    for (int i = 0; i < n; i += kAhead) {
        Summary s[kAhead][V];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const float *at = from + (int64_t)min(i + j, n - 1) * apart + c;
#pragma unroll
            for (int v = 0; v < V; ++v) s[j][v] = {at[v], at[channels + v]};
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (i + j < n)
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = through(s[j][v], h[v]);
    }
}

// A matrix from a segment's first row on: an address that is the wave's own per block, and offsets of 32 bits in it (rows lie at most 2^25 values apart).
template <int PREC, int V> struct Rows {
    using T = typename Elem<PREC>::type;
    using P = Pack<T, V>;
    const char *base;
    uint32_t stride, lane;                         // in bytes
    __device__ __forceinline__ Rows(const idf_rows &r, int64_t row, int c)
        : base((const char *)r.base + row * r.row_stride * (int64_t)sizeof(T)), stride((uint32_t)r.row_stride * (uint32_t)sizeof(T)), lane((uint32_t)c * (uint32_t)sizeof(T)) {}
    // rows t .. t + kBlock - 1, of which there are those below n (the last one again in place of the others)
    __device__ __forceinline__ void load(P (&to)[kBlock], int t, int n) const
    {
        const char *at = base + (int64_t)t * stride;
        if (t + kBlock <= n) {
#pragma unroll
            for (int u = 0; u < kBlock; ++u) to[u] = *(const P *)(at + (lane + u * stride));
        } else {
#pragma unroll
            for (int u = 0; u < kBlock; ++u) to[u] = *(const P *)(at + (lane + (uint32_t)min(u, n - 1 - t) * stride));
        }
    }
    __device__ __forceinline__ void store(int t, int u, const float (&v)[V]) const
    {
        P p;
#pragma unroll
        for (int i = 0; i < V; ++i) p.v[i] = Elem<PREC>::from_f32(v[i]);
        *(P *)(const_cast<char *>(base) + (int64_t)t * stride + (lane + u * stride)) = p;
    }
};

// What a wave works on: V channels from c on in each lane, tokens t0 <= t < t1 of the segment.
struct Work {
    Segment g;
    int segment, group, wave, c, t0, t1;
    bool on;
};
template <int V, class Args> __device__ __forceinline__ Work work_of(const Args &a, const Cut &cut, int group)
{
    Work w;
    w.segment = blockIdx.z;
    w.group = group;
    w.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    w.g = segment_of(a, w.segment, nullptr);
    w.c = (blockIdx.x * 64 + (threadIdx.x & 63)) * V;
    w.on = w.c < a.channels;
    if (!w.on) w.c = a.channels - V;               // (reads what is there, stores nothing)
    w.t0 = (int)min((int64_t)w.g.len, group * cut.span() + (int64_t)w.wave * cut.part);
    w.t1 = min(w.g.len, w.t0 + cut.part);
    return w;
}
// the first token of a segment has a row of marks of its own, whatever the others' lengths are
__device__ __forceinline__ float *marks_at(float *marks, const Work &w, int t, int channels)
{
    return marks + (w.g.begin / kBlock + w.segment + t / kBlock) * channels + w.c;
}

template <int V> __device__ __forceinline__ void join_group(float *lds, const Work &w, const Cut &cut, void *workspace, int channels, const float *begin, const Summary (&s)[V], bool backwards)
{
    if (w.on && w.group == 0 && w.wave == 0) {
        float *to = begin_at(workspace, cut, w.segment, channels) + w.c;
#pragma unroll
        for (int v = 0; v < V; ++v) to[v] = begin ? begin[(int64_t)w.g.ring * channels + w.c + v] : 0.f;
    }
    const int64_t row = first_row(cut, w.g.begin, w.segment) + w.group;
    if (w.on) put<V>(summary_at(workspace, cut, row, 1 + w.wave, channels), channels, w.c, s);
    float *mine = lds + (w.wave * 64 + (threadIdx.x & 63)) * 2 * V;
#pragma unroll
    for (int v = 0; v < V; ++v) { mine[2 * v] = s[v].keep; mine[2 * v + 1] = s[v].made; }
    lds_barrier();
    if (w.wave != 0 || !w.on) return;
    Summary all[V];
#pragma unroll
    for (int v = 0; v < V; ++v) all[v] = {1.f, 0.f};
    for (int i = 0; i < cut.waves; ++i) {
        const float *its = lds + ((backwards ? cut.waves - 1 - i : i) * 64 + (threadIdx.x & 63)) * 2 * V;
#pragma unroll
        for (int v = 0; v < V; ++v) all[v] = join(all[v], Summary{its[2 * v], its[2 * v + 1]});
    }
    put<V>(summary_at(workspace, cut, row, 0, channels), channels, w.c, all);
}

// ---- forward ----

// f(0), f(1), .. of the n first rows of a block, or in the other order; whole blocks without a look at n.
template <class F> __device__ __forceinline__ void rows_up(int n, F f)
{
    if (n >= kBlock) {
#pragma unroll
        for (int u = 0; u < kBlock; ++u) f(u);
    } else {
#pragma unroll
        for (int u = 0; u < kBlock; ++u)
            if (u < n) f(u);
    }
}
template <class F> __device__ __forceinline__ void rows_down(int n, F f)
{
    if (n >= kBlock) {
#pragma unroll
        for (int u = kBlock - 1; u >= 0; --u) f(u);
    } else {
#pragma unroll
        for (int u = kBlock - 1; u >= 0; --u)
            if (u < n) f(u);
    }
}

// The states after each of the n first rows of a block: each(u, h, gates).  Where one comes out infinite or not a number, or a gate is out of bounds,
// the block is taken once more by the definition.
template <int PREC, int V, class P, class F>
__device__ __forceinline__ void states(const P (&x)[kBlock], const P (&g)[kBlock], int n, float (&h)[V], F each)
{
    float was[V], far = 0.f;
    bool fine = true;
#pragma unroll
    for (int v = 0; v < V; ++v) was[v] = h[v];
    rows_up(n, [&](int u) IDF_INLINE {
        Gate w[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float gate = Elem<PREC>::to_f32(g[u].v[v]);
            far = fmaxf(far, __builtin_fabsf(gate));
            w[v] = gate_of<PREC>(gate);
            h[v] = step_of(w[v], Elem<PREC>::to_f32(x[u].v[v]), h[v]);
        }
        each(u, h, w);
    });
#pragma unroll
    for (int v = 0; v < V; ++v) fine = fine && finite(h[v]);
    if (fine && far <= kGateMost) return;
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = was[v];
#pragma unroll
    for (int u = 0; u < kBlock; ++u)
        if (u < n) {
            Gate w[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Slow<PREC> slow(Elem<PREC>::to_f32(g[u].v[v]));
                w[v] = slow.w;
                h[v] = slow.step(Elem<PREC>::to_f32(x[u].v[v]), h[v]);
            }
            each(u, h, w);
        }
}

template <int PREC, int V>
__global__ void __launch_bounds__(512) k_gate_parts(idf_gate_scan_args a, Cut cut)
{
    extern __shared__ float lds[];
    const Work w = work_of<V>(a, cut, blockIdx.y);
    if (w.group * cut.span() >= w.g.len) return;
    const Rows<PREC, V> x(a.x, w.g.begin, w.c), g(a.gates, w.g.begin, w.c);
    typename Rows<PREC, V>::P xs[kBlock], gs[kBlock];
    Summary s[V];
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { s[v] = {1.f, 0.f}; h[v] = 0.f; }
    if (w.t0 < w.t1) { x.load(xs, w.t0, w.t1); g.load(gs, w.t0, w.t1); }
    for (int t = w.t0; t < w.t1; t += kBlock) {
        typename Rows<PREC, V>::P xn[kBlock], gn[kBlock];
        if (t + kBlock < w.t1) { x.load(xn, t + kBlock, w.t1); g.load(gn, t + kBlock, w.t1); }
        Summary was[V];
#pragma unroll
        for (int v = 0; v < V; ++v) was[v] = s[v];
        states<PREC, V>(xs, gs, min(kBlock, w.t1 - t), h, [&](int u, float (&)[V], Gate (&w)[V]) IDF_INLINE {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (u == 0) s[v] = was[v];
                s[v].keep = kept_of(w[v], s[v].keep);
            }
        });
#pragma unroll
        for (int u = 0; u < kBlock; ++u) { xs[u] = xn[u]; gs[u] = gn[u]; }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) s[v].made = h[v];
    join_group<V>(lds, w, cut, a.workspace, a.channels, a.state_in, s, false);
}

template <int PREC, int V>
__global__ void __launch_bounds__(512) k_gate_out(idf_gate_scan_args a, Cut cut)
{
    // parts that were read last come first: they are still in the caches
    const Work w = work_of<V>(a, cut, gridDim.y - 1 - blockIdx.y);
    if (!w.g.valid) return;
    const bool last = w.t1 == w.g.len && (w.t0 < w.t1 || (w.g.len == 0 && w.group == 0 && w.wave == 0));
    if (w.t0 >= w.t1 && !last) return;
    const Rows<PREC, V> x(a.x, w.g.begin, w.c), g(a.gates, w.g.begin, w.c), out(a.out, w.g.begin, w.c);
    typename Rows<PREC, V>::P xs[kBlock], gs[kBlock];
    if (w.t0 < w.t1) { x.load(xs, w.t0, w.t1); g.load(gs, w.t0, w.t1); }
    float h[V];
    const bool cuts = cut.groups * cut.waves > 1 && w.g.len > 0;
    const float *begin = cuts ? begin_at(a.workspace, cut, w.segment, a.channels) : a.state_in ? a.state_in + (int64_t)w.g.ring * a.channels : nullptr;
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = begin ? begin[w.c + v] : 0.f;
    if (w.t0 > 0) {
        const int64_t apart = 2 * (int64_t)a.channels, row = first_row(cut, w.g.begin, w.segment);
        go_through<V>(summary_at(a.workspace, cut, row, 0, a.channels), (1 + cut.waves) * apart, w.group, a.channels, w.c, h);
        go_through<V>(summary_at(a.workspace, cut, row + w.group, 1, a.channels), apart, w.wave, a.channels, w.c, h);
    }
    for (int t = w.t0; t < w.t1; t += kBlock) {
        typename Rows<PREC, V>::P xn[kBlock], gn[kBlock];
        if (t + kBlock < w.t1) { x.load(xn, t + kBlock, w.t1); g.load(gn, t + kBlock, w.t1); }
        if (a.marks && w.on) {
            float *to = marks_at(a.marks, w, t, a.channels);
#pragma unroll
            for (int v = 0; v < V; ++v) to[v] = h[v];
        }
        states<PREC, V>(xs, gs, min(kBlock, w.t1 - t), h, [&](int u, float (&h)[V], Gate (&)[V]) IDF_INLINE { if (w.on) out.store(t, u, h); });
#pragma unroll
        for (int u = 0; u < kBlock; ++u) { xs[u] = xn[u]; gs[u] = gn[u]; }
    }
    if (last && a.state_out && w.on)
#pragma unroll
        for (int v = 0; v < V; ++v) a.state_out[(int64_t)w.g.ring * a.channels + w.c + v] = h[v];
}

// ---- backward ----

// What flows from a token to the one before it, m = a l with l = grad_out + m of the token behind it, over the n first rows of a block, the last
// first: each(u, l, gates).  As above, once more where it comes out infinite or a gate is out of bounds (far).
template <int PREC, int V, class P, class F, class G>
__device__ __forceinline__ void flow(const P (&g)[kBlock], const P (&d)[kBlock], int n, float (&m)[V], float far, F gates, G each)
{
    float was[V];
    bool fine = true;
#pragma unroll
    for (int v = 0; v < V; ++v) was[v] = m[v];
    rows_down(n, [&](int u) IDF_INLINE {
        float l[V];
        Gate w[V];
        gates(u, w);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = Elem<PREC>::to_f32(d[u].v[v]) + m[v];
            m[v] = kept_of(w[v], l[v]);
        }
        each(u, l, w);
    });
#pragma unroll
    for (int v = 0; v < V; ++v) fine = fine && finite(m[v]);
    if (fine && far <= kGateMost) return;
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = was[v];
#pragma unroll
    for (int u = kBlock - 1; u >= 0; --u)
        if (u < n) {
            float l[V];
            Gate w[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Slow<PREC> slow(Elem<PREC>::to_f32(g[u].v[v]));
                w[v] = slow.w;
                l[v] = Elem<PREC>::to_f32(d[u].v[v]) + m[v];
                m[v] = slow.kept(l[v]);
            }
            each(u, l, w);
        }
}
template <int PREC, int V, class P> __device__ __forceinline__ float farthest(const P (&g)[kBlock])
{
    float far = 0.f;
#pragma unroll
    for (int u = 0; u < kBlock; ++u)
#pragma unroll
        for (int v = 0; v < V; ++v) far = fmaxf(far, __builtin_fabsf(Elem<PREC>::to_f32(g[u].v[v])));
    return far;
}

template <int PREC, int V>
__global__ void __launch_bounds__(256) k_gate_back_parts(idf_gate_scan_backward_args a, Cut cut)
{
    extern __shared__ float lds[];
    const Work w = work_of<V>(a, cut, blockIdx.y);
    if (w.group * cut.span() >= w.g.len) return;
    using R = Rows<PREC, V>;
    const R g(a.gates, w.g.begin, w.c), d(a.grad_out, w.g.begin, w.c);
    typename R::P gs[kBlock], ds[kBlock] = {};
    Summary s[V];
    float m[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { s[v] = {1.f, 0.f}; m[v] = 0.f; }
    const int from = w.t0 < w.t1 ? w.t0 + (w.t1 - 1 - w.t0) / kBlock * kBlock : w.t0 - kBlock;
    const bool any = a.grad_out.base;
    if (w.t0 < w.t1) { g.load(gs, from, w.t1); if (any) d.load(ds, from, w.t1); }
    for (int t = from; t >= w.t0; t -= kBlock) {
        typename R::P gn[kBlock], dn[kBlock] = {};
        if (t > w.t0) { g.load(gn, t - kBlock, w.t1); if (any) d.load(dn, t - kBlock, w.t1); }
        const int n = min(kBlock, w.t1 - t);
        float was[V];
#pragma unroll
        for (int v = 0; v < V; ++v) was[v] = s[v].keep;
        flow<PREC, V>(gs, ds, n, m, farthest<PREC, V>(gs), [&](int u, Gate (&w)[V]) IDF_INLINE {
#pragma unroll
            for (int v = 0; v < V; ++v) w[v] = gate_of<PREC>(Elem<PREC>::to_f32(gs[u].v[v]));
        }, [&](int u, float (&)[V], Gate (&w)[V]) IDF_INLINE {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (u == n - 1) s[v].keep = was[v];
                s[v].keep = kept_of(w[v], s[v].keep);
            }
        });
#pragma unroll
        for (int u = 0; u < kBlock; ++u) { gs[u] = gn[u]; ds[u] = dn[u]; }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) s[v].made = m[v];
    join_group<V>(lds, w, cut, a.workspace, a.channels, a.grad_end, s, true);
}

template <int PREC, int V>
__global__ void __launch_bounds__(256, 2) k_gate_back(idf_gate_scan_backward_args a, Cut cut)
{
    const Work w = work_of<V>(a, cut, blockIdx.y);
    const bool first = w.group == 0 && w.wave == 0;
    if (w.t0 >= w.t1 && !first) return;
    using R = Rows<PREC, V>;
    if (first) {                                   // rows that no segment has have no gradient: those in front of the first one, and from a segment's last token to the next one
        auto clear = [&](int64_t from, int64_t to) {
            const float zero[V] = {};
            for (int64_t t = from; t < to; ++t)
                if (w.on) {
                    R(a.grad_x, t, w.c).store(0, 0, zero);
                    R(a.grad_gates, t, w.c).store(0, 0, zero);
                }
        };
        const bool last = w.segment + 1 == a.n_segments;
        if (a.offsets && w.segment == 0) clear(0, w.g.begin);
        clear(w.g.begin + w.g.len, last ? a.n_tokens : a.offsets ? min(max(a.offsets[w.segment + 1], (int64_t)0), a.n_tokens) : w.g.begin + a.max_tokens);
    }
    if (!w.g.valid) return;
    const R x(a.x, w.g.begin, w.c), g(a.gates, w.g.begin, w.c), d(a.grad_out, w.g.begin, w.c), gx(a.grad_x, w.g.begin, w.c), gg(a.grad_gates, w.g.begin, w.c);
    typename R::P xs[kBlock], gs[kBlock], ds[kBlock] = {};
    float mark[V];
    const bool any = a.grad_out.base;
    const int from = w.t0 < w.t1 ? w.t0 + (w.t1 - 1 - w.t0) / kBlock * kBlock : w.t0 - kBlock;
    auto load = [&](int t, typename R::P (&xs)[kBlock], typename R::P (&gs)[kBlock], typename R::P (&ds)[kBlock], float (&mark)[V]) IDF_INLINE {
        x.load(xs, t, w.t1);
        g.load(gs, t, w.t1);
        if (any) d.load(ds, t, w.t1);
        const float *at = marks_at(const_cast<float *>(a.marks), w, t, a.channels);
#pragma unroll
        for (int v = 0; v < V; ++v) mark[v] = at[v];
    };
    const bool on = w.on;
    if (w.t0 < w.t1) load(from, xs, gs, ds, mark);
    float m[V];
    const bool cuts = cut.groups * cut.waves > 1 && w.g.len > 0;
    const float *end = cuts ? begin_at(a.workspace, cut, w.segment, a.channels) : a.grad_end ? a.grad_end + (int64_t)w.g.ring * a.channels : nullptr;
#pragma unroll
    for (int v = 0; v < V; ++v) m[v] = end ? end[w.c + v] : 0.f;
    if (w.t1 < w.g.len) {
        const int64_t apart = 2 * (int64_t)a.channels, row = first_row(cut, w.g.begin, w.segment);
        // groups and parts that have tokens, the last first
        const int groups = (int)((w.g.len + cut.span() - 1) / cut.span());
        const int parts = (int)((min((int64_t)w.g.len, (w.group + 1) * cut.span()) - w.group * cut.span() + cut.part - 1) / cut.part);
        go_through<V>(summary_at(a.workspace, cut, row + groups - 1, 0, a.channels), -(1 + cut.waves) * apart, groups - 1 - w.group, a.channels, w.c, m);
        go_through<V>(summary_at(a.workspace, cut, row + w.group, parts, a.channels), -apart, parts - 1 - w.wave, a.channels, w.c, m);
    }
    for (int t = from; t >= w.t0; t -= kBlock) {
        typename R::P xn[kBlock], gn[kBlock], dn[kBlock] = {};
        float mark_n[V];
        if (t > w.t0) load(t - kBlock, xn, gn, dn, mark_n);
        const int n = min(kBlock, w.t1 - t);
        // of every token the state before it less x, and its gate
        float apart[kBlock][V], h[V], before[V];
        Gate gate[kBlock][V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = before[v] = mark[v];
        states<PREC, V>(xs, gs, n, h, [&](int u, float (&h)[V], Gate (&w)[V]) IDF_INLINE {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (u == 0) before[v] = mark[v];
                apart[u][v] = before[v] - Elem<PREC>::to_f32(xs[u].v[v]);
                gate[u][v] = w[v];
                before[v] = h[v];
            }
        });
        flow<PREC, V>(gs, ds, n, m, farthest<PREC, V>(gs), [&](int u, Gate (&w)[V]) IDF_INLINE {
#pragma unroll
            for (int v = 0; v < V; ++v) w[v] = gate[u][v];
        }, [&](int u, float (&l)[V], Gate (&w)[V]) IDF_INLINE {
            float dx[V], dg[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                dx[v] = l[v] * w[v].take();
                dg[v] = l[v] * apart[u][v] * (__builtin_fabsf(w[v].s) * w[v].big());
            }
            if (on) { gx.store(t, u, dx); gg.store(t, u, dg); }
        });
#pragma unroll
        for (int u = 0; u < kBlock; ++u) { xs[u] = xn[u]; gs[u] = gn[u]; ds[u] = dn[u]; }
#pragma unroll
        for (int v = 0; v < V; ++v) mark[v] = mark_n[v];
    }
    if (first && a.grad_state && w.on)
#pragma unroll
        for (int v = 0; v < V; ++v) a.grad_state[(int64_t)w.g.ring * a.channels + w.c + v] = m[v];
}

// ---- host ----

template <class Args> bool pairs(const Args &a, std::initializer_list<const idf_rows *> rows)
{
    if (a.precision == IDF_PREC_F32 || a.channels % 2) return false;
    for (const idf_rows *r : rows)
        if ((uintptr_t)r->base % 4 || r->row_stride % 2) return false;
    return true;
}
bool pairs(const idf_gate_scan_args &a) { return pairs(a, {&a.x, &a.gates, &a.out}); }
bool pairs(const idf_gate_scan_backward_args &a) { return pairs(a, {&a.x, &a.gates, &a.grad_out, &a.grad_x, &a.grad_gates}); }

// Waves that a call is cut into, by the tokens that there are (us, forward and backward, with 2048 : 4096 : 8192; 16 uneven segments of up to 2048 tokens of 1536 channels
// 74, 130 : 62, 109 : 60, 109; 65536 tokens of 2048 channels 296, 449 : 311, 470 : 304, 468; 8 segments of 4096 tokens of 1024 channels 76, 125 : 78, 128 : 80, 137).
constexpr int64_t kWaves = 4096;
template <class Args> Cut cut_of(const Args &a, int most_waves)
{
    const int64_t blocks = (longest(a) + kBlock - 1) / kBlock, wide = 64 * (pairs(a) ? 2 : 1);
    const int64_t lanes = (a.channels + wide - 1) / wide;                      // waves of a token
    Cut c = {(int)std::max<int64_t>(blocks, 1) * kBlock, 1, 1, 0};
    // blocks of a part so that all tokens that there are make kWaves waves, and more where the longest segment has no room for so many parts
    const int64_t all = std::min<int64_t>(a.n_tokens / kBlock + a.n_segments, a.n_segments * blocks);
    const int64_t part = std::max<int64_t>({(all * lanes + kWaves - 1) / kWaves, 1, (blocks + kMostGroups * most_waves - 1) / (kMostGroups * most_waves)});
    const int64_t parts = (blocks + part - 1) / part;
    if (parts < 2) return c;
    c.waves = (int)std::min<int64_t>(parts <= kMostGroups * 4 ? 4 : most_waves, parts);
    c.part = (int)part * kBlock;
    c.groups = (int)((blocks * kBlock + c.span() - 1) / c.span());
    c.rows = a.n_tokens / c.span() + a.n_segments;
    return c;
}
constexpr int kForwardWaves = 8, kBackwardWaves = 4;

template <class Args> size_t summaries(const Args &a, const Cut &c)
{
    return c.groups * c.waves > 1 ? ((size_t)c.rows * (1 + c.waves) * 2 + a.n_segments) * a.channels * sizeof(float) : 0;
}

template <int PREC, int V>
hipError_t forward(const idf_gate_scan_args &a, const LaunchCtx &lc)
{
    const Cut c = cut_of(a, kForwardWaves);
    const dim3 grid((a.channels + 64 * V - 1) / (64 * V), c.groups, a.n_segments), block(64 * c.waves);
    if (c.groups * c.waves > 1)
        if (const hipError_t e = launch(k_gate_parts<PREC, V>, grid, block, (size_t)c.waves * 64 * 2 * V * sizeof(float), lc, a, c)) return e;
    return launch(k_gate_out<PREC, V>, grid, block, 0, lc, a, c);
}
template <int PREC, int V>
hipError_t backward(const idf_gate_scan_backward_args &a, const LaunchCtx &lc)
{
    const Cut c = cut_of(a, kBackwardWaves);
    const dim3 grid((a.channels + 64 * V - 1) / (64 * V), c.groups, a.n_segments), block(64 * c.waves);
    if (c.groups * c.waves > 1)
        if (const hipError_t e = launch(k_gate_back_parts<PREC, V>, grid, block, (size_t)c.waves * 64 * 2 * V * sizeof(float), lc, a, c)) return e;
    return launch(k_gate_back<PREC, V>, grid, block, 0, lc, a, c);
}

}  // namespace

size_t gate_scan_marks(int64_t n_tokens, int n_segments, int channels) { return (size_t)(n_tokens / kBlock + n_segments + 1) * channels * sizeof(float); }
size_t gate_scan_workspace(const idf_gate_scan_args &a) { return summaries(a, cut_of(a, kForwardWaves)); }
size_t gate_scan_workspace(const idf_gate_scan_backward_args &a) { return summaries(a, cut_of(a, kBackwardWaves)); }

hipError_t launch_gate_scan(const idf_gate_scan_args &a, const LaunchCtx &lc)
{
    if (a.precision == IDF_PREC_F32) return forward<IDF_PREC_F32, 1>(a, lc);
    return pairs(a) ? forward<IDF_PREC_BF16, 2>(a, lc) : forward<IDF_PREC_BF16, 1>(a, lc);
}
hipError_t launch_gate_scan_backward(const idf_gate_scan_backward_args &a, const LaunchCtx &lc)
{
    if (a.precision == IDF_PREC_F32) return backward<IDF_PREC_F32, 1>(a, lc);
    return pairs(a) ? backward<IDF_PREC_BF16, 2>(a, lc) : backward<IDF_PREC_BF16, 1>(a, lc);
}

}  // namespace idf
