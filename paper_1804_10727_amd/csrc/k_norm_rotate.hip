// Norms of queries and keys with their rotation by position, in one pass (idf_norm_rotate).
//
// A workgroup takes a few tokens with all their heads, so that cosines and sines are formed once per token: angle = position * f in
// float64, taken to quarter turns and reduced there (a float32 angle is off by a radian at position 2^24), then cosine and sine of the rest in
// float32.  A group of lanes holds a head, each lane two pieces of P neighbouring values chosen so that the two values of a pair are in the
// same lane: no exchange but the sum of squares.  Bound by memory: every value is read and written once (16384 tokens of 32 + 8 heads of 128 in
// bfloat16: 72 us, 4.7 TB/s; 4001 tokens of 12 + 4 heads of 96 in float32: 13.6 us, 3.6 TB/s); one token each of 64 streams 5.4 to 6.1 us, a launch.
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 1024;                      // workgroups that go on from tokens to tokens: four for a compute unit
constexpr int kMostDeep = 4;                       // heads that a group of lanes has in flight

// P: values of a piece; N: pairs of pieces of a lane (2 only where single values make a head longer than 64 lanes can hold)
template <int PREC, int P, int N, int kDeep>
__global__ void __launch_bounds__(kThreads) k_norm_rotate(idf_norm_rotate_args a, int lanes_log2, int tokens_per_group)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    using Piece = Pack<T, P>;
    extern __shared__ float2 lds[];                // weights of queries and keys, then twice [tokens_per_group][rotary_dim / 2]: amplitude * (cos, sin)
    const int half = a.rotary_dim / 2, heads = a.heads_q + a.heads_k, padded = (a.head_dim + 3) / 4 * 4;
    float *weights = (float *)lds;
    float2 *turn = lds + padded;
    const int table = tokens_per_group * half;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), group = threadIdx.x >> lanes_log2, groups = kThreads >> lanes_log2;
    const float per_head = 1.f / (float)heads;

    // where this lane's pieces begin, and the pair whose angle the first value has
    int at0[N], at1[N], pair[N];
    bool turned[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int c = lane + n * 64;
        if (a.interleaved) {
            at0[n] = 2 * P * c; at1[n] = at0[n] + P; pair[n] = P * c; turned[n] = at0[n] < a.rotary_dim;
        } else if (P * c < half) {
            at0[n] = P * c; at1[n] = half + P * c; pair[n] = P * c; turned[n] = true;
        } else {
            at0[n] = a.rotary_dim + 2 * (P * c - half); at1[n] = at0[n] + P; pair[n] = 0; turned[n] = false;
        }
    }

    // A workgroup goes through its tokens as the groups of lanes take their heads, kDeep each at a time; the values of the next time, and
    // the angles where they belong to further tokens, are fetched and formed while this time's are worked on.
    struct Where { int64_t token0; int row0; };
    auto tokens_of = [&](const Where &w) { return (int)min((int64_t)tokens_per_group, a.n_tokens - w.token0); };
    auto next_of = [&](Where w) {
        w.row0 += groups * kDeep;
        if (w.row0 >= tokens_of(w) * heads) { w.row0 = 0; w.token0 += (int64_t)gridDim.x * tokens_per_group; }
        return w;
    };
    struct Head { int t, h; bool on, key; };
    auto head_of = [&](const Where &w, int u) {
        Head r;
        const int row = w.row0 + u * groups + group;
        r.on = row < tokens_of(w) * heads;
        r.t = r.on ? (int)(((float)row + 0.5f) * per_head) : 0;                // (fewer than 2^16 rows: the quotient is exact)
        r.h = r.on ? row - r.t * heads : 0;
        r.key = r.h >= a.heads_q;
        if (r.key) r.h -= a.heads_q;
        return r;
    };
    auto fetch = [&](const Where &w, Piece (&x)[kDeep][N][2]) IDF_INLINE {
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const Head r = head_of(w, u);
            const idf_tokens &from = r.key ? a.k : a.q;
            const T *src = (const T *)from.base + (w.token0 + r.t) * from.token_stride + r.h * from.head_stride;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                x[u][n][0] = Piece{}; x[u][n][1] = Piece{};
                if (r.on && at0[n] < a.head_dim) x[u][n][0] = *(const Piece *)(src + at0[n]);
                if (r.on && at1[n] < a.head_dim) x[u][n][1] = *(const Piece *)(src + at1[n]);
            }
        }
    };
    auto form_angles = [&](const Where &w, float2 *to) IDF_INLINE {
        const int n = tokens_of(w) * half;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int t = i / half;
            // quarter turns, reduced to the nearest whole one while still in 64 bits: what is left is small where a cosine or sine is
            const double quarters = (double)a.positions[w.token0 + t] * a.frequencies[i - t * half] * 0.63661977236758134308;
            const double whole = __builtin_rint(quarters);
            float s, c;
            sincospif(0.5f * (float)(quarters - whole), &s, &c);
            const int quadrant = (int)(whole - 4.0 * __builtin_floor(0.25 * whole));
            if (quadrant & 1) { const float was = c; c = -s; s = was; }
            if (quadrant & 2) { c = -c; s = -s; }
            to[i] = make_float2((float)(a.amplitude * (double)c), (float)(a.amplitude * (double)s));
        }
    };

    Where at = {(int64_t)blockIdx.x * tokens_per_group, 0};
    if (at.token0 >= a.n_tokens) return;
    Piece x[kDeep][N][2];
    fetch(at, x);
    for (int i = threadIdx.x; i < 2 * padded; i += kThreads) {
        const float *w = i < padded ? a.q_weight : a.k_weight;
        const int d = i < padded ? i : i - padded;
        weights[i] = w && d < a.head_dim ? w[d] : 1.f;
    }
    form_angles(at, turn);
    __syncthreads();
    for (int buffer = 0;;) {
        const Where ahead = next_of(at);
        const bool more = ahead.token0 < a.n_tokens, other_tokens = more && ahead.row0 == 0;
        Piece next[kDeep][N][2];
        if (more) fetch(ahead, next);
        if (other_tokens) form_angles(ahead, turn + (buffer ^ 1) * table);
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const Head r = head_of(at, u);
            float y0[N][P], y1[N][P], sum = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    y0[n][e] = E::to_f32(x[u][n][0].v[e]); y1[n][e] = E::to_f32(x[u][n][1].v[e]);
                    sum += y0[n][e] * y0[n][e] + y1[n][e] * y1[n][e];
                }
            for (int m = 1; m < 1 << lanes_log2; m <<= 1) sum += __shfl_xor(sum, m);
            if (!r.on) continue;
            if (r.key ? a.k_weight : a.q_weight) {
                const float norm = 1.f / sqrtf(sum / (float)a.head_dim + a.eps);
                const float *w = weights + (r.key ? padded : 0);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const Pack<float, P> w0 = at0[n] < a.head_dim ? *(const Pack<float, P> *)(w + at0[n]) : Pack<float, P>{}, w1 = at1[n] < a.head_dim ? *(const Pack<float, P> *)(w + at1[n]) : Pack<float, P>{};
#pragma unroll
                    for (int e = 0; e < P; ++e) { y0[n][e] *= norm * w0.v[e]; y1[n][e] *= norm * w1.v[e]; }
                }
            }
            const float2 *cs = turn + buffer * table + r.t * half;
            const idf_tokens &out = r.key ? a.k_out : a.q_out;
            T *to = (T *)out.base + (at.token0 + r.t) * out.token_stride + r.h * out.head_stride;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (turned[n]) {
                    if (P > 1 && a.interleaved) {
#pragma unroll
                        for (int e = 0; e + 1 < P; e += 2) {
                            const float2 r = cs[pair[n] + e / 2];
                            const float p = y0[n][e], q = y0[n][e + 1];
                            y0[n][e] = p * r.x - q * r.y; y0[n][e + 1] = q * r.x + p * r.y;
                            if (at1[n] >= a.rotary_dim) continue;             // (not turned by nothing: zero times infinite is no zero)
                            const float2 s = cs[pair[n] + P / 2 + e / 2];
                            const float v = y1[n][e], w = y1[n][e + 1];
                            y1[n][e] = v * s.x - w * s.y; y1[n][e + 1] = w * s.x + v * s.y;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < P; ++e) {
                            const float2 r = cs[pair[n] + e];
                            const float p = y0[n][e], q = y1[n][e];
                            y0[n][e] = p * r.x - q * r.y; y1[n][e] = q * r.x + p * r.y;
                        }
                    }
                }
                Piece o0, o1;
#pragma unroll
                for (int e = 0; e < P; ++e) { o0.v[e] = E::from_f32(y0[n][e]); o1.v[e] = E::from_f32(y1[n][e]); }
                if (at0[n] < a.head_dim) *(Piece *)(to + at0[n]) = o0;
                if (at1[n] < a.head_dim) *(Piece *)(to + at1[n]) = o1;
            }
        }
        if (!more) break;
        if (other_tokens) { __syncthreads(); buffer ^= 1; }
        at = ahead;
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
#pragma unroll
            for (int n = 0; n < N; ++n) { x[u][n][0] = next[u][n][0]; x[u][n][1] = next[u][n][1]; }
    }
}

// Pieces of p values: the rotated part and the rest have to be made of them, and every row begin at a multiple of them.
bool pieces_fit(const idf_norm_rotate_args &a, int p, int bytes)
{
    if (a.head_dim % p || (a.interleaved ? a.rotary_dim : a.rotary_dim / 2) % p || (a.head_dim - a.rotary_dim) % p) return false;
    for (const idf_tokens *t : {&a.q, &a.k, &a.q_out, &a.k_out}) {
        if ((t == &a.q || t == &a.q_out ? a.heads_q : a.heads_k) == 0) continue;
        if ((uintptr_t)t->base % (p * bytes) || t->token_stride % p || t->head_stride % p) return false;
    }
    return true;
}

template <int PREC, int P, int N>
hipError_t go(const idf_norm_rotate_args &a, const LaunchCtx &lc)
{
    // pairs of pieces of a head: the rotated ones, and what is left two by two
    const int pieces = a.interleaved ? (a.head_dim + 2 * P - 1) / (2 * P) : a.rotary_dim / 2 / P + (a.head_dim - a.rotary_dim + 2 * P - 1) / (2 * P);
    int lanes_log2 = 0;
    while ((1 << lanes_log2) < pieces && lanes_log2 < 6) ++lanes_log2;
    const int heads = a.heads_q + a.heads_k, groups = kThreads >> lanes_log2;
    // as many tokens as the groups take in one go, but workgroups for every compute unit first
    int64_t per = std::max(1, groups * kMostDeep / heads);
    per = std::max<int64_t>(1, std::min<int64_t>({per, a.n_tokens / 1024, 16}));
    const int64_t grid = std::min<int64_t>((a.n_tokens + per - 1) / per, kGroups);
    const size_t bytes = ((size_t)(a.head_dim + 3) / 4 * 4 + 2 * (size_t)per * (a.rotary_dim / 2)) * sizeof(float2);
    // few tokens: every group of lanes has one head and is done
    if (per * heads <= groups && grid * per >= a.n_tokens)
        return launch(k_norm_rotate<PREC, P, N, 1>, dim3((unsigned)grid), dim3(kThreads), bytes, lc, a, lanes_log2, (int)per);
    return launch(k_norm_rotate<PREC, P, N, kMostDeep>, dim3((unsigned)grid), dim3(kThreads), bytes, lc, a, lanes_log2, (int)per);
}

template <int PREC>
hipError_t by_pieces(const idf_norm_rotate_args &a, const LaunchCtx &lc)
{
    constexpr int VL = Elem<PREC>::VL, bytes = 16 / VL;
    if (pieces_fit(a, VL, bytes)) return go<PREC, VL, 1>(a, lc);
    if (pieces_fit(a, 2, bytes)) return go<PREC, 2, 1>(a, lc);
    return go<PREC, 1, 2>(a, lc);
}

}  // namespace

hipError_t launch_norm_rotate(const idf_norm_rotate_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? by_pieces<IDF_PREC_F32>(a, lc) : by_pieces<IDF_PREC_BF16>(a, lc);
}

}  // namespace idf
