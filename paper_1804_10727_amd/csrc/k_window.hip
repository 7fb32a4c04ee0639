// Attention over a sliding window and first tokens, with the ring that caches keys and values (idf_window_attend).
//
// Scores are formed transposed, S^T = K Q^T: a lane then holds the scores of one query row, so that the softmax's maximum and sum are kept
// per lane, and what comes out of the matrix cores is the operand that O^T = V^T P^T takes, without a way through LDS.  Query heads that share
// a key/value head are rows next to each other: row = token * group + head of the group.
//   Sums, maxima and outputs are float32; in bfloat16 the weights exp(s - max) are rounded to bfloat16 for the product with V (their sum
// is not): half a step of 2^-8 on each, independent from key to key, about as much as the rounding of the output (error against 64 bits 0.0020 to
// 0.0023 of the output, that of its own rounding alone 0.0015 to 0.0017).  Weights in two parts would take half as many matrix instructions more.
#include <algorithm>

#include "idf.h"
#include "seq_mfma.h"

namespace idf {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStepRows = 16;                      // query rows of a segment and key/value head that the step kernel takes
constexpr int kMostSplits = 128;                   // parts of a list of keys: a wave joins them, a lane has two
constexpr int kTileRows = 128;                     // query rows of a workgroup of the tile kernel

// The keys that query positions first .. last see, as a list in order of position: first tokens of the stream, then from the beginning of
// the oldest window on.  Entry i is entry of the ring or of the segment's own tokens; position p sees entry i if
// i <= p - shift and (i > p - window - shift or i < n_first).
struct Keys {
    int n, n_first;            // entries, and how many of them are first tokens ahead of the window
    int skip;                  // position of entry 0 where it is a first token
    int own;                   // entries n_first + own .. are the segment's own, own token 0 being entry n_first + own (may be negative)
    int first_own;             // the same for entries that are first tokens: entry i is own token i - first_own where not negative
    uint32_t slot0, period;    // ring slot, counted behind the first tokens, of entry n_first
    int64_t shift;             // position of entry i >= n_first is i + shift
};

__device__ __forceinline__ Keys keys_of(const idf_window_args &a, const Segment &g, int64_t p0, int64_t p1)
{
    Keys k;
    const int64_t held = a.k_ring ? 0 : g.start;                 // (without a ring nothing from before the segment)
    const int64_t first = min((int64_t)a.sinks, p1 + 1), skip = min(first, held), low = max(max(first, p0 - a.window + 1), held);
    k.skip = (int)skip;
    k.n_first = (int)(first - skip);
    k.shift = low - k.n_first;
    k.n = (int)(p1 - k.shift + 1);
    k.own = (int)max(min(g.start - low, (int64_t)0x7fffffff), -(int64_t)0x7fffffff);
    k.first_own = (int)min(g.start - skip, (int64_t)0x7fffffff);
    k.period = a.k_ring ? (uint32_t)(a.slots - a.sinks) : 1u;
    k.slot0 = low >= a.sinks ? (uint32_t)((low - a.sinks) % k.period) : 0u;
    return k;
}

// Where a matrix of keys or values lies: own tokens and the ring of the segment's stream, from the head's first value on.
template <class T> struct Held {
    const T *own, *ring;
    int64_t own_stride, ring_stride;
    __device__ __forceinline__ Held(const idf_window_args &a, const Segment &g, const idf_tokens &t, const void *ring_base, int kv)
    {
        own = (const T *)t.base + g.begin * t.token_stride + kv * t.head_stride;
        own_stride = t.token_stride;
        ring_stride = (int64_t)a.heads_kv * a.head_dim;
        ring = (const T *)ring_base + g.ring * a.slots * ring_stride + (int64_t)kv * a.head_dim;
    }
};

// Entry i of the list (0 <= i < n): its place, for keys and values alike.
struct Place { bool own; int64_t row; };
__device__ __forceinline__ Place place_of(const idf_window_args &a, const Keys &k, int i)
{
    const int rel = i - k.n_first, t = rel < 0 ? i - k.first_own : rel - k.own;
    Place p;
    p.own = t >= 0;
    uint32_t s = k.slot0 + (uint32_t)rel;
    if (s >= k.period) s -= k.period;
    p.row = p.own ? (int64_t)t : rel < 0 ? (int64_t)(k.skip + i) : (int64_t)a.sinks + s;
    return p;
}
template <class T> __device__ __forceinline__ const T *at(const Held<T> &h, const Place &p)
{
    return p.own ? h.own + p.row * h.own_stride : h.ring + p.row * h.ring_stride;
}

// Rounds whose entries lie behind each other, all own tokens or all in the ring without its end between them, are read from one address on;
// the others (first tokens, the ring's end, the list's) look for the place of each entry.
struct Flat {
    bool own, ring;            // rows near enough to each other for offsets of 32 bits
    template <class T> struct Round {
        const T *k, *v;        // nullptr: no such round
        int k_step, v_step;
    };
    template <class T> __device__ __forceinline__ Flat(const Held<T> &kh, const Held<T> &vh, int entries, int row)
    {
        const int64_t far = ((int64_t)1 << 31) / entries / (int)sizeof(T) - row;
        own = kh.own_stride >= 0 && vh.own_stride >= 0 && kh.own_stride < far && vh.own_stride < far;
        ring = kh.ring_stride < far;
    }
    template <class T> __device__ __forceinline__ Round<T> round(const idf_window_args &a, const Keys &keys, const Held<T> &kh, const Held<T> &vh, int i0, int entries) const
    {
        Round<T> f = {nullptr, nullptr, 0, 0};
        const int rel = i0 - keys.n_first;
        if (i0 + entries > keys.n || rel < 0) return f;
        if (own && rel >= keys.own) {
            f.k = kh.own + (int64_t)(rel - keys.own) * kh.own_stride; f.v = vh.own + (int64_t)(rel - keys.own) * vh.own_stride;
            f.k_step = (int)kh.own_stride; f.v_step = (int)vh.own_stride;
        } else if (ring && rel + entries <= keys.own) {
            uint32_t s = keys.slot0 + (uint32_t)rel;
            if (s >= keys.period) s -= keys.period;
            if (s + entries <= keys.period) {
                f.k = kh.ring + (a.sinks + (int64_t)s) * kh.ring_stride; f.v = vh.ring + (a.sinks + (int64_t)s) * vh.ring_stride;
                f.k_step = f.v_step = (int)kh.ring_stride;
            }
        }
        return f;
    }
};

// Partial results of rows whose keys are split over workgroups: [split][token][head][head_dim] sums, then [split][token][head] maximum (of
// scores in units of log 2) and sum of weights.
struct Partial {
    float *o, *ml;
    int splits;
};
__device__ __host__ __forceinline__ Partial partial_of(const idf_window_args &a, int splits)
{
    Partial p;
    p.splits = splits;
    p.o = (float *)a.workspace;
    p.ml = p.o + (int64_t)splits * a.n_tokens * a.heads_q * a.head_dim;
    return p;
}

// A row whose sums came out infinite or not a number: once more, by one wave, reading only the values that the row sees -- on the
// matrix cores a weight of zero times an infinite value that another row of the tile sees would be no zero.
template <int PREC>
__device__ __forceinline__ void exact_row(const idf_window_args &a, const Segment &g, const Keys &keys, int kv, int h, int t, int i0, int i1, const Partial &part, int split)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    const int lane = threadIdx.x & 63;
    const int64_t p = g.start + t, token = g.begin + t;
    const int hi = (int)(p - keys.shift);
    const int64_t lo = p - a.window - keys.shift;
    const T *q = (const T *)a.q.base + token * a.q.token_stride + h * a.q.head_stride;
    const Held<T> kh(a, g, a.k, a.k_ring, kv), vh(a, g, a.v, a.v_ring, kv);
    float m = -__FLT_MAX__, l = 0.f, o[4] = {};
    for (int b = i0; b < i1; b += 64) {
        const int i = b + lane;
        const bool seen = i < i1 && i <= hi && (i > lo || i < keys.n_first);
        float s = -__builtin_inff();
        if (seen) {
            const T *k = at(kh, place_of(a, keys, i));
            s = 0.f;
            for (int d = 0; d < a.head_dim; ++d) s += E::to_f32(q[d]) * E::to_f32(k[d]);
            s *= a.scale * kLog2e;
        }
        const unsigned long long all = __ballot(seen);
        if (!all) continue;
        // a NaN among the scores has to stay: the maximum alone would drop it, its weight does not
        const float m2 = fmaxf(m, wave_max(s)), w = seen ? exp2f(s - m2) : 0.f, fade = exp2f(m - m2);
        m = m2;
        l = l * fade + wave_sum(w);
        for (int c = 0; c < 4; ++c) o[c] *= fade;
        for (int j = 0; j < 64; ++j) {
            if (!(all >> j & 1)) continue;
            const T *v = at(vh, place_of(a, keys, b + j));
            const float wj = __shfl(w, j);
            for (int c = 0; c < 4; ++c)
                if (lane + 64 * c < a.head_dim) o[c] += wj * E::to_f32(v[lane + 64 * c]);
        }
    }
    if (part.splits > 1) {
        const int64_t row = ((int64_t)split * a.n_tokens + token) * a.heads_q + h;
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < a.head_dim) part.o[row * a.head_dim + lane + 64 * c] = o[c];
        if (lane == 0) { part.ml[2 * row] = m; part.ml[2 * row + 1] = l; }
        return;
    }
    T *out = (T *)a.out.base + token * a.out.token_stride + h * a.out.head_stride;
    for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < a.head_dim) out[lane + 64 * c] = E::from_f32(o[c] / l);
}

// Tokens t0 <= t < t1 of a segment into the ring, by the workgroup that attended over them.  Only where the ring has room for the segment beside
// a window (Plan): the slots that they take then hold tokens that no query of the segment sees any more, while other workgroups still
// read the ring.
template <class T>
__device__ __forceinline__ void append_tokens(const idf_window_args &a, const Segment &g, const Keys &keys, const Held<T> &kh, const Held<T> &vh, int t0, int t1)
{
    constexpr int VL = 16 / (int)sizeof(T);
    const int pieces = a.head_dim / VL;
    for (int x = threadIdx.x; x < (t1 - t0) * pieces; x += 256) {
        const int t = t0 + x / pieces, c = (x - (x / pieces) * pieces) * VL;
        const int64_t p = g.start + t, slot = p < a.sinks ? p : a.sinks + (p - a.sinks) % (int64_t)keys.period;
        *(i32x4 *)(const_cast<T *>(kh.ring) + slot * kh.ring_stride + c) = *(const i32x4 *)(kh.own + t * kh.own_stride + c);
        *(i32x4 *)(const_cast<T *>(vh.ring) + slot * vh.ring_stride + c) = *(const i32x4 *)(vh.own + t * vh.own_stride + c);
    }
}

// ---- few rows on a long axis: single tokens, short segments ----

// A workgroup takes the at most 16 query rows of one segment and key/value head and a part of the keys; its four waves take 16 NT of them at a
// time, in turn, each with a softmax of its own, and are joined at the end.  Keys go from memory straight into the layout of the matrix
// instruction, values through a piece of LDS that is the wave's own, to be read along the keys; both are asked for one round ahead.  No
// barrier but the last.  Bound by memory: every row of the ring is read once (64 streams on 4096 keys of 8 x 128 in bfloat16: 192 us, 5.6 TB/s, in
// float32 361, where two registers are spilled; 64 streams of 16 tokens on 1000 keys of 8 x 64 in float32: 54 to 56 us, 5 TB/s; one stream on 16384
// keys, split: 21 us with the join, 3.2 TB/s).
template <int PREC, int DP> struct StepShape {
    static constexpr int NT = PREC == IDF_PREC_BF16 ? 2 : 1;                  // tiles of 16 keys
    static constexpr int KEYS = 16 * NT;
    static constexpr int STRIDE = DP + (PREC == IDF_PREC_BF16 ? 16 : 4);      // of a row of values in LDS: rows that are read together begin in banks of their own
    static constexpr int ROW16 = DP / Elem<PREC>::VL;                         // pieces of 16 bytes in a row
    static constexpr int LOADS = KEYS * ROW16 / 64;
    static constexpr int WAVE_FLOATS = 16 * DP > KEYS * STRIDE / (4 / (int)sizeof(typename Elem<PREC>::type)) ? 16 * DP : KEYS * STRIDE / (4 / (int)sizeof(typename Elem<PREC>::type));
};

template <int PREC, int DP>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1) k_window_step(idf_window_args a, int splits, bool append)
{
    using M = Mfma<PREC>;
    using T = typename M::T;
    using S = StepShape<PREC, DP>;
    constexpr int NT = S::NT, KS = DP / 32, DT = DP / 16;
    __shared__ __align__(16) float lds[4 * S::WAVE_FLOATS];
    __shared__ float stats[2][4][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    const int split = blockIdx.x, kv = blockIdx.y, group = a.heads_q / a.heads_kv;
    const Segment g = segment_of(a, blockIdx.z, a.starts);
    if (g.len == 0) return;
    const int rows = min(g.len * group, kStepRows);
    const Keys keys = keys_of(a, g, g.start, g.start + g.len - 1);
    const Held<T> kh(a, g, a.k, a.k_ring, kv), vh(a, g, a.v, a.v_ring, kv);
    const Partial part = partial_of(a, splits);

    // this split's entries, whole tiles of them; the waves take them in turn
    const int tiles = (keys.n + S::KEYS - 1) / S::KEYS, per = (tiles + splits - 1) / splits;
    const int t0 = split * per, t1 = min(tiles, t0 + per);
    const int my_t = col / group;                                             // the query row of this lane
    const int my_h = kv * group + col - my_t * group;
    const int64_t p = g.start + min(my_t, g.len - 1);
    const int hi = (int)(p - keys.shift);
    const int lo = (int)max(p - a.window - keys.shift, (int64_t)-1);
    const float scale = a.scale * kLog2e;

    typename M::frag q[KS];
    {
        const T *src = (const T *)a.q.base + (g.begin + my_t) * a.q.token_stride + my_h * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = col < rows ? M::load(src + 32 * s + 8 * grp, a.head_dim - 32 * s - 8 * grp) : M::zero();
    }

    T *v_lds = (T *)(lds + wave * S::WAVE_FLOATS);
    typename M::frag kf[NT][KS];
    i32x4 vf[S::LOADS];
    const int r0 = lane / S::ROW16, c0 = (lane - r0 * S::ROW16) * M::VL;
    const Flat flat(kh, vh, S::KEYS, DP);
    auto load = [&](int tile) IDF_INLINE {
        const int i0 = tile * S::KEYS;
        if (const auto f = flat.round(a, keys, kh, vh, i0, S::KEYS); f.k) {
            const uint32_t ko = (uint32_t)(col * f.k_step + 8 * grp) * sizeof(T), vo = (uint32_t)(r0 * f.v_step + c0) * sizeof(T);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const T *src = (const T *)((const char *)(f.k + (int64_t)(16 * t) * f.k_step) + ko);
#pragma unroll
                for (int s = 0; s < KS; ++s) kf[t][s] = M::load(src + 32 * s, a.head_dim - 32 * s - 8 * grp);
            }
#pragma unroll
            for (int j = 0; j < S::LOADS; ++j) {
                if constexpr (64 % S::ROW16 == 0) {
                    constexpr int rows = 64 / S::ROW16;
                    vf[j] = c0 < a.head_dim ? *(const i32x4 *)((const char *)(f.v + (int64_t)(j * rows) * f.v_step) + vo) : i32x4{0, 0, 0, 0};
                } else {
                    const int piece = j * 64 + lane, r = piece / S::ROW16, c = (piece - r * S::ROW16) * M::VL;
                    vf[j] = c < a.head_dim ? *(const i32x4 *)(f.v + r * f.v_step + c) : i32x4{0, 0, 0, 0};
                }
            }
            return;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const T *src = at(kh, place_of(a, keys, min(i0 + 16 * t + col, keys.n - 1)));
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[t][s] = M::load(src + 32 * s + 8 * grp, a.head_dim - 32 * s - 8 * grp);
        }
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int piece = j * 64 + lane, r = piece / S::ROW16, c = (piece - r * S::ROW16) * M::VL, i = i0 + r;
            vf[j] = i < keys.n && c < a.head_dim ? *(const i32x4 *)(at(vh, place_of(a, keys, i)) + c) : i32x4{0, 0, 0, 0};
        }
    };

    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -__FLT_MAX__, l = 0.f;
    if (t0 + wave < t1) load(t0 + wave);
    for (int tile = t0 + wave; tile < t1; tile += 4) {
        f32x4 st[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            st[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) st[t] = M::mma16(kf[t][s], q[s], st[t]);
        }
        __builtin_amdgcn_wave_barrier();                                      // (LDS serves a wave in order: only the compiler has to keep it)
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int piece = j * 64 + lane, r = piece / S::ROW16, c = (piece - r * S::ROW16) * M::VL;
            *(i32x4 *)(v_lds + r * S::STRIDE + c) = vf[j];
        }
        __builtin_amdgcn_wave_barrier();
        if (tile + 4 < t1) load(tile + 4);

        float w[NT * 4], top = m;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = tile * S::KEYS + 16 * t + 4 * grp + e;
                const bool seen = i <= hi && (i > lo || i < keys.n_first);
                w[4 * t + e] = seen ? st[t][e] * scale : -__builtin_inff();
                top = fmaxf(top, w[4 * t + e]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__ballot(top > m)) {
            const float fade = __builtin_amdgcn_exp2f(m - top);
            l *= fade;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= fade;
            m = top;
        }
#pragma unroll
        for (int e = 0; e < NT * 4; ++e) { w[e] = __builtin_amdgcn_exp2f(w[e] - m); l += w[e]; }
        if constexpr (PREC == IDF_PREC_BF16) {
            const bf16x8 pf = M::pack(w);
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = M::mma16(read_column(v_lds, S::STRIDE, 16 * d, 4 * grp, 16 + 4 * grp), pf, o[d]);
        } else {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v_lds[(4 * grp + e) * S::STRIDE + 16 * d + col], w[e], o[d], 0, 0, 0);
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // the waves' rows joined: [wave][row][value]
    __builtin_amdgcn_wave_barrier();
    float *mine = lds + wave * S::WAVE_FLOATS;
#pragma unroll
    for (int d = 0; d < DT; ++d) *(f32x4 *)(mine + col * DP + 16 * d + 4 * grp) = o[d];
    if (grp == 0) { stats[0][wave][col] = m; stats[1][wave][col] = l; }
    __syncthreads();
    bool bad = false;
    constexpr int V4 = DP / 4;
    for (int x = threadIdx.x; x < rows * V4; x += 256) {
        const int r = x / V4, c = (x - r * V4) * 4;
        float top = -__FLT_MAX__, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, stats[0][w][r]);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float fade = __builtin_amdgcn_exp2f(stats[0][w][r] - top);
            sum += fade * stats[1][w][r];
            v += fade * *(const f32x4 *)(lds + w * S::WAVE_FLOATS + r * DP + c);
        }
        if (c >= a.head_dim) continue;
        const int t = r / group, h = kv * group + r - t * group;
        const int64_t token = g.begin + t;
        const f32x4 none = v * 0.f;
        bad |= !(none[0] + none[1] + none[2] + none[3] == 0.f);
        if (splits > 1) {
            const int64_t row = ((int64_t)split * a.n_tokens + token) * a.heads_q + h;
            *(f32x4 *)(part.o + row * a.head_dim + c) = v;
            if (c == 0) { part.ml[2 * row] = top; part.ml[2 * row + 1] = sum; }
        } else {
            Pack<T, 4> out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out.v[e] = Elem<PREC>::from_f32(v[e] / sum);
            *(Pack<T, 4> *)((T *)a.out.base + token * a.out.token_stride + h * a.out.head_stride + c) = out;
        }
    }
    if (g.len > 1 && __syncthreads_or(bad))                                   // (a single token sees every key of its list)
        for (int r = wave; r < rows; r += 4) {
            const int t = r / group;
            exact_row<PREC>(a, g, keys, kv, kv * group + r - t * group, t, t0 * S::KEYS, min(t1 * S::KEYS, keys.n), part, split);
        }
    if (append && split == 0) append_tokens(a, g, keys, kh, vh, 0, g.len);
}

// ---- many rows ----

// A workgroup takes 128 query rows of one segment and key/value head and walks over their keys; a wave has 32 of the rows.  Keys and values of a round
// go through registers into LDS, the next round's being asked for while this one's are worked on.  Two prompts of 16384 tokens, 32 heads of 128 on a
// window of 4096: 1990 to 2150 us by the machine, 890 to 965 TFLOP/s.  No unit is busy all the time: matrix cores 44 %, vector units in all 46 % (of
// 128 values a head, a round costs a wave 32 matrix instructions of 32 cycles and some 200 others, 32 of them exponentials of 16), LDS 34 % without
// bank conflicts; a wave waits for a quarter of its time for memory or the others, and 31 % to issue.  Of 64 values, half the matrix instructions and as many others,
// which is why these run four waves to a SIMD, held to 128 registers with eight spilled ones, one of them read in the loop (three: 273 us, four: 263, uneven
// segments; there compute units have work for 53 % of the time only, with matrix cores busy 18 % and vector units 36 % of the whole).  Two
// halves of LDS with one barrier a round instead of two took longer (2182 : 2158 us), reads from LDS held ahead of the products as long (2076 : 2065).
// Heads of more than 128 values are not loaded ahead: two prompts of 4096 tokens, 16 heads of 256 on 4, 483 us, 570 TFLOP/s (float32 2480 us, 111).
template <int PREC, int DP> struct TileShape {
    static constexpr int KEYS = PREC == IDF_PREC_BF16 ? 64 : 32;
    static constexpr int VL = Elem<PREC>::VL, ROW16 = DP / VL;
    static constexpr int K_STRIDE = DP + VL;                                  // neighbouring rows begin 16 bytes apart in the banks
    static constexpr int V_STRIDE = DP + (PREC != IDF_PREC_BF16 ? 4 : DP % 64 ? 0 : 32);      // four rows by 64 bytes are read together: rows begin 16 banks apart
    static constexpr int LOADS = KEYS * ROW16 / 256;
    static_assert(KEYS * ROW16 % 256 == 0, "a round is loaded whole");
    static constexpr bool AHEAD = DP <= 128;                                  // (longer rows leave no registers for a round on its way)
    static constexpr int LDS_BYTES = KEYS * (K_STRIDE + V_STRIDE) * (int)sizeof(typename Elem<PREC>::type);
};

template <int PREC, int DP>
__global__ void __launch_bounds__(256, PREC != IDF_PREC_BF16 || DP > 128 ? 1 : DP > 64 ? 2 : 4) k_window_tile(idf_window_args a, int splits, bool append)
{
    using M = Mfma<PREC>;
    using T = typename M::T;
    using S = TileShape<PREC, DP>;
    constexpr int KT = S::KEYS / 32, KS = DP / 16, DT = DP / 32;
    extern __shared__ __align__(16) unsigned char raw[];
    T *k_lds = (T *)raw, *v_lds = k_lds + S::KEYS * S::K_STRIDE;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int group = a.heads_q / a.heads_kv;
    const int kv = blockIdx.x % a.heads_kv, seg = blockIdx.x / a.heads_kv;
    const int split = blockIdx.z, tile = gridDim.y - 1 - blockIdx.y;          // long lists first
    const Segment g = segment_of(a, seg, a.starts);
    const int64_t rows = (int64_t)g.len * group, row0 = (int64_t)tile * kTileRows;
    if (row0 >= rows) return;
    const int64_t row_last = min(row0 + kTileRows, rows) - 1;
    const Keys keys = keys_of(a, g, g.start + row0 / group, g.start + row_last / group);
    const Held<T> kh(a, g, a.k, a.k_ring, kv), vh(a, g, a.v, a.v_ring, kv);
    const Partial part = partial_of(a, splits);
    const int rounds = (keys.n + S::KEYS - 1) / S::KEYS, per = (rounds + splits - 1) / splits;
    const int t0 = split * per, t1 = min(rounds, t0 + per);

    const int64_t my_row = row0 + wave * 32 + col;
    const bool on = my_row < rows;
    const int my_t = (int)(min(my_row, rows - 1) / group), my_h = kv * group + (int)(min(my_row, rows - 1) - (int64_t)my_t * group);
    const int64_t p = g.start + my_t, token = g.begin + my_t;
    const int hi = (int)(p - keys.shift);
    const int lo = (int)max(p - a.window - keys.shift, (int64_t)-1);
    const float scale = a.scale * kLog2e;
    // what all rows of the wave see without a look at the mask
    const int hi_all = (int)(g.start + min(row0 + wave * 32, rows - 1) / group - keys.shift);
    const int lo_all = (int)max(g.start + min(row0 + wave * 32 + 31, rows - 1) / group - a.window - keys.shift, (int64_t)-1);

    typename M::frag q[KS];
    {
        const T *src = (const T *)a.q.base + token * a.q.token_stride + my_h * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = M::load(src + 16 * s + 8 * half, a.head_dim - 16 * s - 8 * half);
    }
    const int r0 = threadIdx.x / S::ROW16, c0 = (threadIdx.x - r0 * S::ROW16) * M::VL;
    const bool in_row = c0 < a.head_dim;
    const Flat flat(kh, vh, S::KEYS, DP);
    i32x4 kr[S::LOADS], vr[S::LOADS];
    auto load = [&](int t) IDF_INLINE {
        const int i0 = t * S::KEYS;
        if (const auto f = flat.round(a, keys, kh, vh, i0, S::KEYS); f.k) {
            const T *kb = f.k, *vb = f.v;
            const int ks = f.k_step, vs = f.v_step;
            const uint32_t ko = (uint32_t)(r0 * ks + c0) * sizeof(T), vo = (uint32_t)(r0 * vs + c0) * sizeof(T);
#pragma unroll
            for (int j = 0; j < S::LOADS; ++j) {
                constexpr int rows = 256 / S::ROW16;
                if constexpr (256 % S::ROW16 == 0) {
                    kr[j] = in_row ? *(const i32x4 *)((const char *)(kb + (int64_t)(j * rows) * ks) + ko) : i32x4{0, 0, 0, 0};
                    vr[j] = in_row ? *(const i32x4 *)((const char *)(vb + (int64_t)(j * rows) * vs) + vo) : i32x4{0, 0, 0, 0};
                } else {
                    const int piece = j * 256 + threadIdx.x, r = piece / S::ROW16, c = (piece - r * S::ROW16) * M::VL;
                    kr[j] = c < a.head_dim ? *(const i32x4 *)(kb + r * ks + c) : i32x4{0, 0, 0, 0};
                    vr[j] = c < a.head_dim ? *(const i32x4 *)(vb + r * vs + c) : i32x4{0, 0, 0, 0};
                }
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int piece = j * 256 + threadIdx.x, r = piece / S::ROW16, c = (piece - r * S::ROW16) * M::VL, i = i0 + r;
            const bool there = i < keys.n && c < a.head_dim;
            const Place pl = place_of(a, keys, min(i, keys.n - 1));
            kr[j] = there ? *(const i32x4 *)(at(kh, pl) + c) : i32x4{0, 0, 0, 0};
            vr[j] = there ? *(const i32x4 *)(at(vh, pl) + c) : i32x4{0, 0, 0, 0};
        }
    };
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = -__FLT_MAX__, l = 0.f;
    if (S::AHEAD && t0 < t1) load(t0);
    for (int t = t0; t < t1; ++t) {
        if (!S::AHEAD) load(t);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int piece = j * 256 + threadIdx.x, r = piece / S::ROW16, c = (piece - r * S::ROW16) * M::VL;
            *(i32x4 *)(k_lds + r * S::K_STRIDE + c) = kr[j];
            *(i32x4 *)(v_lds + r * S::V_STRIDE + c) = vr[j];
        }
        __syncthreads();
        if (S::AHEAD && t + 1 < t1) load(t + 1);

        // a wave in its products goes first: those of another on the same SIMD, in its softmax, fill what it leaves (two long prompts 2158 -> 2065 us)
        __builtin_amdgcn_s_setprio(1);
        f32x16 st[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
            for (int e = 0; e < 16; ++e) st[kt][e] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) st[kt] = M::mma32(M::load(k_lds + (32 * kt + col) * S::K_STRIDE + 16 * s + 8 * half), q[s], st[kt]);
        }
        __builtin_amdgcn_s_setprio(0);
        const int i0 = t * S::KEYS;
        if (!(i0 + S::KEYS - 1 <= hi_all && (i0 > lo_all || i0 + S::KEYS <= keys.n_first))) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int i = i0 + 32 * kt + 8 * (e / 4) + 4 * half + e % 4;
                    if (!(i <= hi && (i > lo || i < keys.n_first))) st[kt][e] = -__builtin_inff();
                }
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, st[kt][e]);
        top = fmaxf(top, __shfl_xor(top, 32));
        // the maximum that weights are taken against may lag behind by a factor of 2^8, far from any overflow: outputs are scaled anew only
        // where it falls back further
        top *= scale;
        if (__ballot(top > m + 8.f)) {
            top = fmaxf(m, top);
            const float fade = __builtin_amdgcn_exp2f(m - top);
            l *= fade;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= fade;
            m = top;
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                st[kt][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kt][e], scale, -m));
                l += st[kt][e];
            }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < 2 * KT; ++s) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = st[s / 2][8 * (s % 2) + e];
            const typename M::frag pf = M::pack(w);
#pragma unroll
            for (int d = 0; d < DT; ++d)
                o[d] = M::mma32(read_column(v_lds, S::V_STRIDE, 32 * d + (lane & 16), 16 * s + 4 * half, 16 * s + 8 + 4 * half), pf, o[d]);
        }
        __builtin_amdgcn_s_setprio(0);
    }
    l += __shfl_xor(l, 32);

    float none = 0.f;
    T *out = (T *)a.out.base + token * a.out.token_stride + my_h * a.out.head_stride;
    const int64_t prow = ((int64_t)split * a.n_tokens + token) * a.heads_q + my_h;
    const float r = 1.f / l;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int c = 32 * d + 2 * e + 4 * half;
#pragma unroll
            for (int x = 0; x < 4; ++x) none += o[d][e + x] * 0.f;
            if (!on || c >= a.head_dim) continue;
            if (splits > 1) {
                *(f32x4 *)(part.o + prow * a.head_dim + c) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
            } else {
                Pack<T, 4> w;
#pragma unroll
                for (int x = 0; x < 4; ++x) w.v[x] = Elem<PREC>::from_f32(o[d][e + x] * r);
                *(Pack<T, 4> *)(out + c) = w;
            }
        }
    if (splits > 1 && on && half == 0) { part.ml[2 * prow] = m; part.ml[2 * prow + 1] = l; }
    if (__ballot(!(none == 0.f)))
        for (int x = 0; x < 32 && row0 + wave * 32 + x < rows; ++x) {
            const int64_t row = row0 + wave * 32 + x;
            const int t = (int)(row / group);
            exact_row<PREC>(a, g, keys, kv, kv * group + (int)(row - (int64_t)t * group), t, t0 * S::KEYS, min(t1 * S::KEYS, keys.n), part, split);
        }
    // the tokens whose first row lies in this tile
    if (append && split == 0) append_tokens(a, g, keys, kh, vh, (int)((row0 + group - 1) / group), (int)(row_last / group) + 1);
}

// Splits joined.  A workgroup takes a row, each of its waves every fourth split: its lanes first the maximum and sum of a split each, whose
// shares then go from lane to lane while a lane adds up four values of the row, with splits side by side where the row leaves lanes.  All of
// a wave's reads are on their way together: one after the other, each would wait for memory.
template <int PREC>
__global__ void __launch_bounds__(256) k_window_join(idf_window_args a, int splits, int lanes_log2)
{
    using T = typename Elem<PREC>::type;
    constexpr int kAhead = 8;
    __shared__ __align__(16) float sums[4][256];
    const Segment g = segment_of(a, blockIdx.y, a.starts);
    const Partial part = partial_of(a, splits);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = (lane & ((1 << lanes_log2) - 1)) * 4, first = wave + 4 * (lane >> lanes_log2), step = 4 * (64 >> lanes_log2);
    const int64_t n = (int64_t)g.len * a.heads_q, apart = a.n_tokens * a.heads_q;
    for (int64_t x = blockIdx.x; x < n; x += gridDim.x) {
        const int64_t t = x / a.heads_q, token = g.begin + t, row = token * a.heads_q + (x - t * a.heads_q);
        float m[2], l[2], share[2] = {}, sum = 0.f;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int s = lane + 64 * y;
            m[y] = s < splits ? part.ml[2 * (row + s * apart)] : -__FLT_MAX__;
            l[y] = s < splits ? part.ml[2 * (row + s * apart) + 1] : 0.f;
        }
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < splits; s0 += kAhead * step) {
            f32x4 in[kAhead];
#pragma unroll
            for (int y = 0; y < kAhead; ++y) {
                const int s = s0 + first + y * step;
                in[y] = s < splits && c < a.head_dim ? *(const f32x4 *)(part.o + (row + s * apart) * a.head_dim + c) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
            if (s0 == 0) {
                const float top = wave_max(fmaxf(m[0], m[1]));
#pragma unroll
                for (int y = 0; y < 2; ++y) share[y] = __builtin_amdgcn_exp2f(m[y] - top);
                sum = wave_sum((lane < splits ? l[0] * share[0] : 0.f) + (lane + 64 < splits ? l[1] * share[1] : 0.f));
            }
#pragma unroll
            for (int y = 0; y < kAhead; ++y) {
                const int s = s0 + first + y * step;
                const float low = __shfl(share[0], s & 63), high = __shfl(share[1], s & 63);
                v += (s & 64 ? high : low) * in[y];
            }
        }
        for (int mask = 1 << lanes_log2; mask < 64; mask <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], mask);
        __syncthreads();                           // (the row before has been read)
        if (first < 4 && c < a.head_dim) *(f32x4 *)(sums[wave] + c) = v;
        __syncthreads();
        if (threadIdx.x * 4 >= a.head_dim) continue;
        const int at = threadIdx.x * 4;
        v = *(const f32x4 *)(sums[0] + at) + *(const f32x4 *)(sums[1] + at) + *(const f32x4 *)(sums[2] + at) + *(const f32x4 *)(sums[3] + at);
        Pack<T, 4> w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.v[e] = Elem<PREC>::from_f32(v[e] / sum);
        *(Pack<T, 4> *)((T *)a.out.base + token * a.out.token_stride + (x - t * a.heads_q) * a.out.head_stride + at) = w;
    }
}

// The segments' tokens into their rings, behind the attention that still reads what they take the place of.  Of a segment longer than
// the ring the newest tokens are written, so that no slot is written twice.
__global__ void __launch_bounds__(256) k_window_append(idf_window_args a, int row16, int elem16)
{
    const Segment g = segment_of(a, blockIdx.y, a.starts);
    const int64_t period = a.slots - a.sinks;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < (int64_t)g.len * row16; c += (int64_t)gridDim.x * 256) {
        const int t = (int)(c / row16), piece = (int)(c - (int64_t)t * row16);       // pieces of 16 bytes: head, then place in it
        const int64_t p = g.start + t;
        if (p >= a.sinks && t < g.len - period) continue;
        const int64_t slot = p < a.sinks ? p : a.sinks + (p - a.sinks) % period;
        const int per_head = row16 / a.heads_kv, h = piece / per_head, at = (piece - h * per_head) * elem16, eb = 16 / elem16;
        const int64_t to = (((g.ring * a.slots + slot) * a.heads_kv + h) * a.head_dim + at) * eb;
        const int64_t kf = ((g.begin + t) * a.k.token_stride + h * a.k.head_stride + at) * eb, vf = ((g.begin + t) * a.v.token_stride + h * a.v.head_stride + at) * eb;
        *(i32x4 *)((char *)a.k_ring + to) = *(const i32x4 *)((const char *)a.k.base + kf);
        *(i32x4 *)((char *)a.v_ring + to) = *(const i32x4 *)((const char *)a.v.base + vf);
    }
}

// How a call is cut: which kernel, and into how many parts the keys go.
struct Plan {
    bool step;
    int tiles, splits;
    bool append;               // tokens go to the ring with the attention over them, and not by a launch behind it
};
// Into how many parts a list of keys goes: the number with the least estimated time.  A workgroup's rounds follow each other, at a time each that
// is latency where few of them run (measured, us: four tiles of the step kernel 1.4 in bfloat16, 0.9 + 0.0075 per value of a head in float32; a round
// of the tile kernel 1.0 + 0.006, and 1.3 + 0.0275; by the head's size, not by the one it is padded to); a join is a launch of 4 to
// 5 us and reads every row of every part.  At most 512 workgroups, whichever kernel: compute units hold two of most, but one of float32 tiles of more than 64
// values and bfloat16 ones of more than 128, three of steps of 64 values and four of bfloat16 tiles of 64; whole rounds of the machine are not counted.  256
// where one is held (us per pass, 256 : 512): 8 streams x 300 tokens on 4000 keys, 4 heads of 96 in float32 504 : 391, but 4 streams x 100 tokens on 8000
// keys, 4 heads of 128, 331 : 377, and 200 tokens on 8000 keys, 4 heads of 256 in bfloat16, 75 : 86.  Against parts of 256 keys (step) or 512 (tile) at
// least, us per pass: one stream, four heads of 128 on one, 1500 keys 14.2 -> 11.1, in float32 19.2 -> 11.8; 40 tokens, eight heads on two, 500 keys 27.7 -> 15.9,
// 95.5 -> 21.3; 1200 tokens, 600 keys, where the join costs more than it brings, 45.6 -> 29.4.
int splits_of(const idf_window_args &a, bool step, int64_t pairs, int64_t keys)
{
    const bool bf = a.precision == IDF_PREC_BF16;
    const int64_t round = step ? (bf ? 128 : 64) : bf ? 64 : 32, rounds = (keys + round - 1) / round, held = 512;
    const double each = step ? (bf ? 1.4 : 0.9 + 0.0075 * a.head_dim) : bf ? 1.0 + 0.006 * a.head_dim : 1.3 + 0.0275 * a.head_dim;
    const double rows = (double)std::min<int64_t>(a.n_tokens, a.n_segments * longest(a)) * a.heads_q;
    int best = 1;
    double least = 0.0;
    for (int64_t per = rounds; per >= 1; per = per > 8 ? per * 7 / 8 : per - 1) {
        const int64_t n = (rounds + per - 1) / per;
        if (n > 1 && (n > kMostSplits || pairs * n > held)) break;
        const double us = per * each + (n > 1 ? (step ? 4.2 : 5.0) + rows * (1.6e-3 + 1e-6 * n * a.head_dim) : 0.0);
        if (n == 1 || us < least) { least = us; best = (int)n; }
    }
    return best;
}

Plan plan_of(const idf_window_args &a)
{
    Plan p;
    const int64_t rows = longest(a) * (a.heads_q / a.heads_kv);
    p.step = rows <= kStepRows;
    // the ring has room for a segment beside a window (64 streams of 16 tokens, float32: 60 -> 50 us a pass)
    p.append = a.k_ring && a.slots - a.sinks - a.window >= longest(a) - 1;
    p.tiles = p.step ? 1 : (int)((rows + kTileRows - 1) / kTileRows);
    const int64_t pairs = (int64_t)a.n_segments * a.heads_kv * p.tiles;
    const int64_t own = p.step ? longest(a) : std::min<int64_t>(longest(a), kTileRows / (a.heads_q / a.heads_kv) + 1);
    const int64_t keys = std::min<int64_t>(a.window, a.k_ring ? a.slots : longest(a)) + a.sinks + own;
    p.splits = splits_of(a, p.step, pairs, keys);
    return p;
}

template <int PREC, int DP>
hipError_t attend(const idf_window_args &a, const Plan &p, const LaunchCtx &lc)
{
    if (p.step)
        return launch(k_window_step<PREC, DP>, dim3(p.splits, a.heads_kv, a.n_segments), dim3(256), 0, lc, a, p.splits, p.append);
    constexpr int bytes = TileShape<PREC, DP>::LDS_BYTES;
    if (bytes > 65536)
        if (const hipError_t e = allow_lds<bytes>(Kernel<k_window_tile<PREC, DP>>{})) return e;
    return launch(k_window_tile<PREC, DP>, dim3(a.n_segments * a.heads_kv, p.tiles, p.splits), dim3(256), bytes, lc, a, p.splits, p.append);
}

template <int PREC>
hipError_t by_dim(const idf_window_args &a, const LaunchCtx &lc)
{
    const Plan p = plan_of(a);
    hipError_t e = a.head_dim <= 64 ? attend<PREC, 64>(a, p, lc) : a.head_dim <= 96 ? attend<PREC, 96>(a, p, lc) : a.head_dim <= 128 ? attend<PREC, 128>(a, p, lc) : attend<PREC, 256>(a, p, lc);
    if (e == hipSuccess && p.splits > 1) {
        int lanes_log2 = 0;
        while (4 << lanes_log2 < a.head_dim) ++lanes_log2;
        e = launch(k_window_join<PREC>, dim3((unsigned)std::min<int64_t>(longest(a) * a.heads_q, 8192), a.n_segments), dim3(256), 0, lc, a, p.splits, lanes_log2);
    }
    if (e == hipSuccess && a.k_ring && !p.append) {
        const int elem16 = Elem<PREC>::VL, row16 = a.heads_kv * a.head_dim / elem16;
        e = launch(k_window_append, dim3((unsigned)std::min<int64_t>((longest(a) * row16 + 255) / 256, 4096), a.n_segments), dim3(256), 0, lc, a, row16, elem16);
    }
    return e;
}

}  // namespace

size_t window_workspace(const idf_window_args &a)
{
    const Plan p = plan_of(a);
    return p.splits > 1 ? (size_t)p.splits * a.n_tokens * a.heads_q * (a.head_dim + 2) * sizeof(float) : 0;
}

hipError_t launch_window(const idf_window_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? by_dim<IDF_PREC_F32>(a, lc) : by_dim<IDF_PREC_BF16>(a, lc);
}

}  // namespace idf
