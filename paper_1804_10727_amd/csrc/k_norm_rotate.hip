// Norms of queries and keys with their rotation by position, in one pass (idf_norm_rotate).
//
// A workgroup takes a few tokens with all their heads, so that cosines and sines are formed once per token: angle = position * f in
// float64, taken to quarter turns and reduced there (a float32 angle is off by a radian at position 2^24), then cosine and sine of the rest in
// float32.  A group of lanes holds a head, each lane two pieces of P neighbouring values chosen so that the two values of a pair are in the
// same lane: no exchange but the sum of squares.  Bound by memory: every value is read and written once.
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

constexpr int kThreads = 256;
constexpr int kDeep = 4;                           // heads that a group of lanes has in flight

// P: values of a piece; N: pairs of pieces of a lane (2 only where single values make a head longer than 64 lanes can hold)
template <int PREC, int P, int N>
__global__ void __launch_bounds__(kThreads) k_norm_rotate(idf_norm_rotate_args a, int lanes_log2, int tokens_per_group)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    using Piece = Pack<T, P>;
    extern __shared__ float2 turn[];               // [tokens_per_group][rotary_dim / 2]: amplitude * (cos, sin)
    const int half = a.rotary_dim / 2, heads = a.heads_q + a.heads_k;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), group = threadIdx.x >> lanes_log2, groups = kThreads >> lanes_log2;

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

    for (int64_t token0 = (int64_t)blockIdx.x * tokens_per_group; token0 < a.n_tokens; token0 += (int64_t)gridDim.x * tokens_per_group)
    for (int row0 = 0, tokens = (int)min((int64_t)tokens_per_group, a.n_tokens - token0), rows = tokens * heads; row0 < rows; row0 += groups * kDeep) {
        Piece x0[kDeep][N], x1[kDeep][N];
        T *to[kDeep];
        const float *weight[kDeep];
        int token[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int row = row0 + u * groups + group;
            const bool on = row < rows;
            const int t = on ? row / heads : 0, h = on ? row - t * heads : 0;
            const bool is_k = h >= a.heads_q;
            const idf_tokens &from = is_k ? a.k : a.q, &out = is_k ? a.k_out : a.q_out;
            const int hh = is_k ? h - a.heads_q : h;
            const T *src = (const T *)from.base + (token0 + t) * from.token_stride + hh * from.head_stride;
            to[u] = on ? (T *)out.base + (token0 + t) * out.token_stride + hh * out.head_stride : nullptr;
            weight[u] = is_k ? a.k_weight : a.q_weight;
            token[u] = t;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                x0[u][n] = Piece{}; x1[u][n] = Piece{};
                if (on && at0[n] < a.head_dim) x0[u][n] = *(const Piece *)(src + at0[n]);
                if (on && at1[n] < a.head_dim) x1[u][n] = *(const Piece *)(src + at1[n]);
            }
        }
        if (row0 == 0) {
            __syncthreads();                       // (the angles of the tokens before are no longer read)
            for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
                const int t = i / half;
                // quarter turns, reduced to the nearest whole one while still in 64 bits: what is left is small where a cosine or sine is
                const double quarters = (double)a.positions[token0 + t] * a.frequencies[i - t * half] * 0.63661977236758134308;
                const double whole = __builtin_rint(quarters);
                float s, c;
                sincospif(0.5f * (float)(quarters - whole), &s, &c);
                const int quadrant = (int)(whole - 4.0 * __builtin_floor(0.25 * whole));
                if (quadrant & 1) { const float was = c; c = -s; s = was; }
                if (quadrant & 2) { c = -c; s = -s; }
                turn[i] = make_float2((float)(a.amplitude * (double)c), (float)(a.amplitude * (double)s));
            }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            float y0[N][P], y1[N][P], sum = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    y0[n][e] = E::to_f32(x0[u][n].v[e]); y1[n][e] = E::to_f32(x1[u][n].v[e]);
                    sum += y0[n][e] * y0[n][e] + y1[n][e] * y1[n][e];
                }
            for (int m = 1; m < 1 << lanes_log2; m <<= 1) sum += __shfl_xor(sum, m);
            if (!to[u]) continue;
            if (weight[u]) {
                const float norm = 1.f / sqrtf(sum / (float)a.head_dim + a.eps);
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        if (at0[n] < a.head_dim) y0[n][e] *= norm * weight[u][at0[n] + e];
                        if (at1[n] < a.head_dim) y1[n][e] *= norm * weight[u][at1[n] + e];
                    }
            }
            const float2 *cs = turn + token[u] * half;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (turned[n]) {
                    if (P > 1 && a.interleaved) {
#pragma unroll
                        for (int e = 0; e + 1 < P; e += 2) {
                            const float2 r = cs[pair[n] + e / 2], s = at1[n] < a.rotary_dim ? cs[pair[n] + P / 2 + e / 2] : make_float2(1.f, 0.f);
                            const float p = y0[n][e], q = y0[n][e + 1], v = y1[n][e], w = y1[n][e + 1];
                            y0[n][e] = p * r.x - q * r.y; y0[n][e + 1] = q * r.x + p * r.y;
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
                if (at0[n] < a.head_dim) *(Piece *)(to[u] + at0[n]) = o0;
                if (at1[n] < a.head_dim) *(Piece *)(to[u] + at1[n]) = o1;
            }
        }
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
    int64_t per = std::max(1, groups * kDeep / heads);
    per = std::max<int64_t>(1, std::min<int64_t>({per, a.n_tokens / 1024, 32}));
    const int64_t grid = std::min<int64_t>((a.n_tokens + per - 1) / per, 1 << 20);
    return launch(k_norm_rotate<PREC, P, N>, dim3((unsigned)grid), dim3(kThreads), (size_t)per * (a.rotary_dim / 2) * sizeof(float2), lc, a, lanes_log2, (int)per);
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
