// Linear attention with a decay per head (idf_decay_attend).
#include <algorithm>
#include <type_traits>

#include "idf.h"
#include "seq_mfma.h"

namespace idf {

namespace {

// A decay that is applied again and again, as the largest float32 number not above it and the rest: one rounded number would be off in the same
// direction each time (half a step of 2^-25: after 4000 tokens 1e-4, where the roundings of the state cancel to 1e-6).  Both are positive wherever
// the decay is, so that an infinite state stays infinite.
struct Factor {
    float high, low;
    __device__ __forceinline__ float times(float s) const { return __builtin_fmaf(high, s, low * s); }
};
__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }
// high + rest, a rest of half a step of it at most, either sign.
__device__ __forceinline__ Factor factor_of(float high, float rest)
{
    if (rest < 0.f) {                              // (one step down; exact, as the two are of one size)
        const float down = __builtin_bit_cast(float, __builtin_bit_cast(int, high) - 1);
        rest += high - down;
        high = down;
    }
    return {uniform(high), uniform(fmaxf(rest, high * 0x1p-60f))};
}
__device__ __forceinline__ Factor factor_of(double decay) { return factor_of((float)decay, (float)(decay - (double)(float)decay)); }
// exp(log_decay).  Where it is near one, by what it lacks, to 2^-23 of that; where not, what has been multiplied a few times is gone.
__device__ __forceinline__ Factor factor_of(float log_decay)
{
    if (log_decay < -0.5f) return factor_of(expf(log_decay), 0.f);
    const float lacks = expm1f(log_decay), high = 1.f + lacks;
    return factor_of(high, lacks - (high - 1.f));
}

// The recurrence itself, token by token.  A wave owns 32 columns of the state of one key/value head: eight lanes side by side hold four
// columns each, eight lanes below each other ROWS rows each, so that a token costs four multiply-adds per value of the state and a sum
// over eight lanes per query; nothing is shared between waves.  Bound by memory: the state is
// read and written once (64 streams x 16 heads of 128 x 128, a token each: 29.6 us, 4.6 TB/s).
template <int PREC, int ROWS>
__global__ void __launch_bounds__(256, ROWS == 8 ? 3 : 1) k_decay_tokens(idf_decay_args a, int column_groups)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int kv = wave / column_groups, c0 = (wave - kv * column_groups) * 32 + (lane & 7) * 4, r0 = (lane >> 3) * ROWS;
    if (kv >= a.heads_kv) return;
    const Segment g = segment_of(a, blockIdx.y, nullptr);
    if (!g.valid) return;
    const int queries = a.heads_q / a.heads_kv;
    const Factor lambda = factor_of(a.log_decay[kv]);
    const bool on = c0 < a.dim_v;
    const int64_t state = ((int64_t)g.ring * a.heads_kv + kv) * a.dim_k * a.dim_v;
    f32x4 s[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        s[r] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (a.state_in && on && r0 + r < a.dim_k) s[r] = *(const f32x4 *)(a.state_in + state + (int64_t)(r0 + r) * a.dim_v + c0);
    }
    for (int t = 0; t < g.len; ++t) {
        const int64_t row = g.begin + t;
        const T *k = (const T *)a.k.base + row * a.k.token_stride + kv * a.k.head_stride;
        const T *v = (const T *)a.v.base + row * a.v.token_stride + kv * a.v.head_stride;
        f32x4 vv = {0.f, 0.f, 0.f, 0.f};
        if (on)
#pragma unroll
            for (int e = 0; e < 4; ++e) vv[e] = E::to_f32(v[c0 + e]);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float kr = r0 + r < a.dim_k ? E::to_f32(k[r0 + r]) : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[r][e] = __builtin_fmaf(kr, vv[e], lambda.times(s[r][e]));
        }
        for (int h = kv * queries; h < (kv + 1) * queries; ++h) {
            const T *q = (const T *)a.q.base + row * a.q.token_stride + h * a.q.head_stride;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r0 + r >= a.dim_k) continue;
                const float qr = E::to_f32(q[r0 + r]);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(qr, s[r][e], o[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int m = 8; m < 64; m <<= 1) o[e] += __shfl_xor(o[e], m);
            if (lane < 8 && on) {
                T *out = (T *)a.out.base + row * a.out.token_stride + h * a.out.head_stride;
                Pack<T, 4> w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w.v[e] = E::from_f32(a.scale * o[e]);
                *(Pack<T, 4> *)(out + c0) = w;
            }
        }
    }
    if (a.state_out && on)
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (r0 + r < a.dim_k) *(f32x4 *)(a.state_out + state + (int64_t)(r0 + r) * a.dim_v + c0) = s[r];
}

// ---- segments of many tokens, 32 at a time ----

// With S the state before a chunk of L <= 32 tokens, i and j tokens of it:
//   O_i = lambda^(i+1) q_i S + sum_{j<=i} lambda^(i-j) (q_i . k_j) v_j,     S' = lambda^L S + sum_j k_j^T (lambda^(L-1-j) v_j),
// matrix products throughout, no power of the decay above one.  A wave owns 32 columns of the state, in accumulators; scores are formed
// transposed, K Q^T, by every wave for itself, so that what comes out is an operand of the next product; so is the state.  Keys and values
// go through LDS, to be read along the tokens too, the next chunk's asked for while this one's are worked on.
//   Roundings in bfloat16: scores times decay, and the state where it meets the queries, are rounded to bfloat16 (half a step of 2^-8, as the
// output is).  The state itself stays float32: a decayed value, 24 bits, goes into the product as three bfloat16 numbers that add up to it.
//   Bound by memory: q, k, v and out once, k and v twice where a segment is cut into parts (one prompt of 65536 tokens, 16 heads of 128 x 128 in
// bfloat16: 400 to 418 us by the machine, of them 135 to 145 for the states of the parts, 14 for the scan and 240 to 275 for the outputs, 4 TB/s;
// matrix cores and LDS a third of the time, waves waiting for 33 to 40 %; loads of the outputs' pass
// two chunks ahead took longer, 512 us in all: between stores they are waited for all the same).  Short calls by latency: 64 streams of 16 tokens,
// 4 heads of 64 x 64 in float32, 10.2 us.
constexpr int kChunk = 32;

// Segments cut into parts along time, so that there is work for every compute unit: the state that each part leaves if it begins with none,
// then the states that the parts begin with, then the parts themselves.
struct Parts {
    int n, tokens;             // parts of the longest segment, tokens of a part (a multiple of the chunk)
    float *states;             // [segment][head][part][dim_k][dim_v]; nullptr for one part
};

__device__ __forceinline__ float log2_of(float log_decay)
{
    const float x = log_decay * 1.4426950408889634f;
    return x < -1e30f ? -1e30f : x;                // (a decay to nothing: times zero stays zero; a maximum would drop what is not a number)
}

template <int N> __device__ __forceinline__ bool finite(const f32x16 (&s)[N])
{
    float none[4] = {};
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) none[e % 4] += s[t][e] * 0.f;
    return none[0] + none[1] + (none[2] + none[3]) == 0.f;
}

// What a wave does in k_decay_chunks, once more, by the recurrence, where something infinite or not a number came into a state that had begun without:
// three parts of an infinite value are no number, nor is an infinite key times a part that is zero, nor an infinite value times the zeros behind a
// key that is shorter than DK.  Outputs that are finite are as they should be and stay.  Lanes side by side hold a column of the state each, either half
// of the wave half of its rows.  False: the state had begun so, or the decay is not a number and nothing else can come of it.
template <int PREC, int DK, int NW, bool states_only>
__device__ __forceinline__ bool part_by_tokens(const idf_decay_args &a, const Parts &parts, int blocks, int x, int y, int thread, bool good)
{
    using M = Mfma<PREC>;
    using E = Elem<PREC>;
    using T = typename M::T;
    constexpr int ROWS = DK / 16;                  // times eight rows
    const int part = gridDim.y - 1 - y, kv = x / blocks % a.heads_kv, seg = x / blocks / a.heads_kv;
    const int c = x % blocks * 32 * NW + (thread & ~63) / 2 + (thread & 31), half = thread >> 5 & 1;
    const Segment g = segment_of(a, seg, nullptr);
    const int first = part * parts.tokens, len = min(g.len - first, parts.tokens), queries = a.heads_q / a.heads_kv;
    const bool own = c < a.dim_v, last = first + parts.tokens >= g.len;
    const int64_t state = ((int64_t)g.ring * a.heads_kv + kv) * a.dim_k * a.dim_v + c;
    float *mid = parts.states ? parts.states + ((int64_t)(seg * a.heads_kv + kv) * parts.n + part) * a.dim_k * a.dim_v + c : nullptr;
    const float *from = states_only ? nullptr : mid ? mid : a.state_in ? a.state_in + state : nullptr;
    float s[ROWS][8], none = 0.f;
#pragma unroll
    for (int p = 0; p < ROWS; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int r = 16 * p + 8 * half + e;
            s[p][e] = from && own && r < a.dim_k ? from[r * a.dim_v] : 0.f;
            none += s[p][e] * 0.f;
        }
    const float lambda = __builtin_amdgcn_exp2f(log2_of(a.log_decay[kv]));
    if (lambda != lambda || !__ballot(!good && none == 0.f)) return false;
    __threadfence_block();                         // (outputs are written once more)
    const T *k = (const T *)a.k.base + (g.begin + first) * a.k.token_stride + kv * a.k.head_stride;
    const T *v = (const T *)a.v.base + (g.begin + first) * a.v.token_stride + kv * a.v.head_stride + c;
#pragma unroll 1
    for (int t = 0; t < len; ++t, k += a.k.token_stride, v += a.v.token_stride) {
        const float vc = own ? E::to_f32(*v) : 0.f;
#pragma unroll
        for (int p = 0; p < ROWS; ++p) {
            const int r = 16 * p + 8 * half;
            const typename M::frag f = M::load(k + r, a.dim_k - r);
#pragma unroll
            for (int e0 = 0; e0 < 8; e0 += M::VL)                             // (zeros behind the key would meet infinities)
                if (r + e0 < a.dim_k)
#pragma unroll
                    for (int e = e0; e < e0 + M::VL; ++e) s[p][e] = __builtin_fmaf(E::to_f32(f[e]), vc, lambda * s[p][e]);
        }
        if constexpr (!states_only)
#pragma unroll 1
            for (int h = kv * queries; h < (kv + 1) * queries; ++h) {
                const int64_t token = g.begin + first + t;
                const T *q = (const T *)a.q.base + token * a.q.token_stride + h * a.q.head_stride;
                float o = 0.f;
#pragma unroll
                for (int p = 0; p < ROWS; ++p) {
                    const int r = 16 * p + 8 * half;
                    const typename M::frag f = M::load(q + r, a.dim_k - r);
                    if (r < a.dim_k)
#pragma unroll
                        for (int e = 0; e < 8; ++e) o = __builtin_fmaf(E::to_f32(f[e]), s[p][e], o);
                }
                o += __shfl_xor(o, 32);
                if (own && half == 0 && !(o * 0.f == 0.f)) ((T *)a.out.base)[token * a.out.token_stride + h * a.out.head_stride + c] = E::from_f32(a.scale * o);
            }
    }
    float *to = states_only ? mid : last && a.state_out ? a.state_out + state : nullptr;
    if (to && own)
#pragma unroll
        for (int p = 0; p < ROWS; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (16 * p + 8 * half + e < a.dim_k) to[(16 * p + 8 * half + e) * a.dim_v] = s[p][e];
    return true;
}

// (bfloat16, keys of up to 64, four waves: held to the 168 registers of three waves to a SIMD at the price of three spilled ones -- with two waves
// uneven segments took 94 us in place of 80)
template <int PREC, int DK, int NW, bool states_only>
__global__ void __launch_bounds__(64 * NW, PREC != IDF_PREC_BF16 ? 1 : NW == 4 ? (DK <= 64 ? 3 : 2) : DK <= 64 ? 2 : 1) k_decay_chunks(idf_decay_args a, Parts parts, int blocks)
{
    using M = Mfma<PREC>;
    using E = Elem<PREC>;
    using T = typename M::T;
    using frag = typename M::frag;
    constexpr int KS = DK / 16, KT = DK / 32, VL = M::VL, THREADS = 64 * NW;
    constexpr int K_STRIDE = DK + VL, V_STRIDE = 32 * NW + (PREC == IDF_PREC_BF16 ? 16 : 4);
    constexpr int K_LOADS = kChunk * DK / VL / THREADS, V_LOADS = kChunk * 32 / VL / 64;
    constexpr int BF = PREC == IDF_PREC_BF16;
    constexpr int SCORE_STRIDE = kChunk + 4, STAGES = states_only ? 2 : 1;
    __shared__ __align__(16) T k_both[2][kChunk * K_STRIDE], q_both[2][kChunk * K_STRIDE], v_both[2][kChunk * V_STRIDE];
    __shared__ __align__(16) float score[kChunk * SCORE_STRIDE], fresh[2 * kChunk];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int part = gridDim.y - 1 - blockIdx.y;   // (the parts whose keys and values were read last are the first to be read again)
    const int block = blockIdx.x % blocks, kv = blockIdx.x / blocks % a.heads_kv, seg = blockIdx.x / blocks / a.heads_kv;
    const Segment g = segment_of(a, seg, nullptr);
    const int first = part * parts.tokens;
    const int len = min(g.len - first, parts.tokens);
    const bool last = first + parts.tokens >= g.len;                          // the state behind this part is the segment's
    if (!g.valid || (len <= 0 && part > 0) || (states_only && last)) return;
    const int queries = a.heads_q / a.heads_kv;
    const int c0 = block * 32 * NW;                                           // the workgroup's first column
    const float l2 = log2_of(a.log_decay[kv]);
    const int my_c = c0 + 32 * wave + ((col & 0x13) | (col & 4) << 1 | (col & 8) >> 1);
    const bool own = my_c < a.dim_v;

    // row e of a state's tile: 16 (e / 8) + 8 half + e % 8, so that eight registers are eight rows in order; columns 4 .. 7 and 8 .. 11 of
    // each 16 are in each other's place, so that of an output, too, a lane has eight values in order
    f32x16 s[KT];
    const int64_t state = ((int64_t)g.ring * a.heads_kv + kv) * a.dim_k * a.dim_v;
    float *mid = parts.states ? parts.states + ((int64_t)(seg * a.heads_kv + kv) * parts.n + part) * a.dim_k * a.dim_v : nullptr;
    const float *from = states_only ? nullptr : mid ? mid : a.state_in ? a.state_in + state : nullptr;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
    if (from && own)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 32 * t + 16 * (e / 8) + 8 * half + e % 8;
                const float x = from[min(r, a.dim_k - 1) * a.dim_v + my_c];
                s[t][e] = r < a.dim_k ? x : 0.f;
            }

    // powers of the decay, by way of LDS: scale * lambda^(i-j) between tokens of a chunk, and what a token leaves at a whole chunk's end
    for (int x = threadIdx.x; x < kChunk * kChunk; x += THREADS) {
        const int i = x / kChunk, j = x % kChunk;
        score[i * SCORE_STRIDE + j] = i >= j ? __builtin_amdgcn_exp2f((float)(i - j) * l2) * a.scale : 0.f;
        if (i == 0) { fresh[j] = __builtin_amdgcn_exp2f((float)(kChunk - 1 - j) * l2); fresh[kChunk + j] = 0.f; }
    }
    const float faded = __builtin_amdgcn_exp2f((float)(col + 1) * l2) * a.scale;
    // The decay of a whole chunk is applied again and again, and its own rounding would add up: each factor takes back what those before it
    // were off (drift: what has been applied over what should have been), and the last one of the call, which may be of a short chunk, leaves nothing
    // for the next call to add to.
    const double whole = exp2((double)kChunk * (double)l2), inverse = whole > 1e-30 ? 1.0 / whole : 0.0;
    double drift = 1.0;
    const double short_one = exp2((double)((max(len, 1) - 1) % kChunk + 1) * (double)l2);

    // A step is a chunk for one of the heads.  While one is worked on, what the next one needs is written from registers into the other half
    // of LDS, and what the one behind it needs is on its way; where nothing is stored between the loads, what the next but one needs, too.
    const T *kb = (const T *)a.k.base + (g.begin + first) * a.k.token_stride + kv * a.k.head_stride;
    const T *vb = (const T *)a.v.base + (g.begin + first) * a.v.token_stride + kv * a.v.head_stride;
    const T *qb = (const T *)a.q.base + (g.begin + first) * a.q.token_stride + kv * queries * a.q.head_stride;
    const int heads = states_only ? 1 : queries;
    struct Step { int t0, h; };
    auto next_of = [&](Step x) { return x.h + 1 < heads ? Step{x.t0, x.h + 1} : Step{x.t0 + kChunk, 0}; };
    // Loads are issued whether there is something to load or not, from the nearest place that there is, and become zeros on their way into
    // LDS: behind a branch the compiler would have to wait for all of them instead of the oldest.
    i32x4 kr[STAGES][K_LOADS], qr[STAGES][K_LOADS], vr[STAGES][V_LOADS];
    auto load = [&](const Step &x, int stage) IDF_INLINE {
        if (STAGES == 1 && x.t0 >= len) return;
#pragma unroll
        for (int y = 0; y < K_LOADS; ++y) {
            const int piece = y * THREADS + threadIdx.x, r = piece / (DK / VL), c = (piece - r * (DK / VL)) * VL;
            if constexpr (STAGES == 2) {
                kr[stage][y] = *(const i32x4 *)(kb + (int64_t)min(x.t0 + r, len - 1) * a.k.token_stride + min(c, a.dim_k - VL));
            } else {
                const bool there = x.t0 + r < len && c < a.dim_k;
                if (x.h == 0) kr[stage][y] = there ? *(const i32x4 *)(kb + (int64_t)(x.t0 + r) * a.k.token_stride + c) : i32x4{0, 0, 0, 0};
                qr[stage][y] = there ? *(const i32x4 *)(qb + (int64_t)(x.t0 + r) * a.q.token_stride + x.h * a.q.head_stride + c) : i32x4{0, 0, 0, 0};
            }
        }
        if (x.h == 0)
#pragma unroll
            for (int y = 0; y < V_LOADS; ++y) {
                const int piece = y * THREADS + threadIdx.x, r = piece / (32 * NW / VL), c = c0 + (piece - r * (32 * NW / VL)) * VL;
                if constexpr (STAGES == 2) vr[stage][y] = *(const i32x4 *)(vb + (int64_t)min(x.t0 + r, len - 1) * a.v.token_stride + min(c, a.dim_v - VL));
                else vr[stage][y] = x.t0 + r < len && c < a.dim_v ? *(const i32x4 *)(vb + (int64_t)(x.t0 + r) * a.v.token_stride + c) : i32x4{0, 0, 0, 0};
            }
    };
    auto store = [&](const Step &x, int step, int stage) IDF_INLINE {
        if (STAGES == 1 && x.t0 >= len) return;
        T *k_to = k_both[x.t0 / kChunk & 1], *v_to = v_both[x.t0 / kChunk & 1], *q_to = q_both[step & 1];
        const i32x4 none = {0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < K_LOADS; ++y) {
            const int piece = y * THREADS + threadIdx.x, r = piece / (DK / VL), c = (piece - r * (DK / VL)) * VL;
            const bool there = STAGES == 1 || (x.t0 + r < len && c < a.dim_k);
            if (x.h == 0) *(i32x4 *)(k_to + r * K_STRIDE + c) = there ? kr[stage][y] : none;
            if (!states_only) *(i32x4 *)(q_to + r * K_STRIDE + c) = there ? qr[stage][y] : none;
        }
        if (x.h == 0)
#pragma unroll
            for (int y = 0; y < V_LOADS; ++y) {
                const int piece = y * THREADS + threadIdx.x, r = piece / (32 * NW / VL), c = (piece - r * (32 * NW / VL)) * VL;
                *(i32x4 *)(v_to + r * V_STRIDE + c) = STAGES == 1 || (x.t0 + r < len && c0 + c < a.dim_v) ? vr[stage][y] : none;
            }
    };
    // values of this wave's columns along the tokens: register x of piece p is token 16 p + 8 (x / 4) + 4 half + x % 4
    auto read_values = [&](const T *v_lds, frag (&v)[2]) IDF_INLINE {
#pragma unroll
        for (int p = 0; p < 2; ++p) v[p] = read_rows_swapped(v_lds, V_STRIDE, 32 * wave + (lane & 16), 16 * p + 4 * half, 16 * p + 8 + 4 * half);
    };
    // what the n tokens of a chunk add to the state, each weighed by what it leaves at the chunk's end, and that by `left`
    auto gain = [&](const frag (&v)[2], const T *k_lds, int n, float left) IDF_INLINE {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = E::to_f32(v[p][e]) * (fresh[16 * p + 8 * (e / 4) + 4 * half + e % 4 + kChunk - n] * left);
            frag pieces[BF ? 3 : 1];
            if constexpr (BF) {
#pragma unroll
                for (int y = 0; y < 3; ++y) {
                    uint32_t u[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {  // the upper 16 bits, and what is left
                        u[e] = __builtin_bit_cast(uint32_t, x[e]);
                        x[e] -= __builtin_bit_cast(float, u[e] & 0xffff0000u);
                    }
                    i32x4 both;
#pragma unroll
                    for (int e = 0; e < 4; ++e) both[e] = (int)__builtin_amdgcn_perm(u[2 * e + 1], u[2 * e], 0x07060302u);
                    pieces[y] = __builtin_bit_cast(frag, both);
                }
            } else {
                pieces[0] = M::pack(x);
            }
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const frag k = read_rows_swapped(k_lds, K_STRIDE, 32 * t + (lane & 16), 16 * p + 4 * half, 16 * p + 8 + 4 * half);
#pragma unroll
                for (int y = 0; y < (BF ? 3 : 1); ++y) s[t] = M::mma32(k, pieces[y], s[t]);
            }
        }
    };
    Step now = {0, 0}, ahead = next_of(now), beyond = next_of(ahead);
    auto step_of = [&](int step, int stage) IDF_INLINE {
        __syncthreads();
        store(ahead, step + 1, stage);
        const Step then = next_of(beyond);
        load(STAGES == 2 ? then : beyond, stage);
        const int t0 = now.t0, n = min(kChunk, len - t0), h = now.h;
        const T *k_lds = k_both[t0 / kChunk & 1], *v_lds = v_both[t0 / kChunk & 1], *q_lds = q_both[step & 1];
        now = ahead;
        ahead = beyond;
        beyond = then;

        frag v[2];
        read_values(v_lds, v);

        if (!states_only) {
                f32x16 w, o;
#pragma unroll
                for (int e = 0; e < 16; ++e) { w[e] = 0.f; o[e] = 0.f; }
#pragma unroll
                for (int p = 0; p < KS; ++p) {
                    float sv[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) sv[e] = s[p / 2][8 * (p % 2) + e];
                    const frag q = M::load(q_lds + col * K_STRIDE + 16 * p + 8 * half);
                    o = M::mma32(M::pack(sv), q, o);
                    w = M::mma32(M::load(k_lds + col * K_STRIDE + 16 * p + 8 * half), q, w);
                }
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 f = *(const f32x4 *)(score + col * SCORE_STRIDE + 2 * e + 4 * half);
#pragma unroll
                    for (int x = 0; x < 4; ++x) w[e + x] *= f[x];
                }
                o *= faded;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    float wv[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) wv[e] = w[8 * p + e];
                    o = M::mma32(v[p], M::pack(wv), o);
                }
                float none = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) none += o[e] * 0.f;
                if (__ballot(!(none == 0.f))) {
                    // something infinite or not a number: a weight of zero times a later token's value is no zero then.  Once more, with the
                    // tokens up to this one only
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0.f;
#pragma unroll
                    for (int p = 0; p < KS; ++p) {
                        float sv[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) sv[e] = s[p / 2][8 * (p % 2) + e];
                        o = M::mma32(M::pack(sv), M::load(q_lds + col * K_STRIDE + 16 * p + 8 * half), o);
                    }
                    o *= faded;
#pragma unroll 1
                    for (int j = 0; j < n; ++j) {
                        float qk = 0.f;            // (a lane takes every other value, lane ^ 32 the ones between)
#pragma unroll 1
                        for (int d = half; d < a.dim_k; d += 2) qk += E::to_f32(q_lds[col * K_STRIDE + d]) * E::to_f32(k_lds[j * K_STRIDE + d]);
                        qk += __shfl_xor(qk, 32);
                        if (j > col) continue;
                        qk *= __builtin_amdgcn_exp2f((float)(col - j) * l2) * a.scale;
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] += qk * E::to_f32(v_lds[j * V_STRIDE + 32 * wave + 16 * (e / 8) + 8 * half + e % 8]);
                    }
                }
                if (col < n) {
                    const int c = c0 + 32 * wave + 8 * half;
                    T *out = (T *)a.out.base + (g.begin + first + t0 + col) * a.out.token_stride + (kv * queries + h) * a.out.head_stride + c;
#pragma unroll
                    for (int e = 0; e < 16; e += VL) {
                        Pack<T, VL> pk;
#pragma unroll
                        for (int x = 0; x < VL; ++x) pk.v[x] = E::from_f32(o[e + x]);
                        if (c + 16 * (e / 8) + e % 8 < a.dim_v) *(Pack<T, VL> *)(out + 16 * (e / 8) + e % 8) = pk;
                    }
                }
            }

        if (h + 1 < heads) return;
        // what this chunk's last token leaves at the end of the part, where only that is asked for: nothing is faded on the way then
        if constexpr (states_only) {
            gain(v, k_lds, n, __builtin_amdgcn_exp2f((float)(len - t0 - n) * l2));
        } else if (t0 + kChunk < len) {
            const float fade = uniform((float)(whole * (2.0 - drift)));       // (2 - x is 1 / x so near to one)
            if (inverse > 0.0) drift *= (double)fade * inverse;
#pragma unroll
            for (int t = 0; t < KT; ++t) s[t] *= fade;
            gain(v, k_lds, kChunk, 1.f);
        }
    };
    if (len > 0) {
        load(now, 0);
        store(now, 0, 0);
        load(ahead, 0);
        if (STAGES == 2) load(beyond, STAGES - 1);
        for (int step = 0; now.t0 < len; step += STAGES) {
            step_of(step, 0);
            if (STAGES == 1 || now.t0 >= len) continue;
            step_of(step + 1, STAGES - 1);
        }
        if constexpr (!states_only) {              // the last chunk, which is still in LDS (within the loop the state's registers would be copied for it)
            const int t0 = (len - 1) / kChunk * kChunk;
            const Factor fade = factor_of(short_one * (2.0 - drift));
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = fade.times(s[t][e]);
            frag v[2];
            read_values(v_both[t0 / kChunk & 1], v);
            gain(v, k_both[t0 / kChunk & 1], len - t0, 1.f);
        }
    }

    if (const bool good = finite(s); __builtin_expect(__ballot(!good) != 0, 0)) {
        int x = blockIdx.x, y = blockIdx.y, thread = threadIdx.x;
        asm volatile("" : "+s"(x), "+s"(y), "+v"(thread));                    // (everything anew: kept from the beginning it would take the registers of the loop)
        if (part_by_tokens<PREC, DK, NW, states_only>(a, parts, blocks, x, y, thread, good)) return;
    }
    float *to = states_only ? mid : last && a.state_out ? a.state_out + state : nullptr;
    int row = 8 * half;
    asm volatile("" : "+v"(row));                  // (places of the rows anew: kept from the beginning they would take the registers of the loop)
    if (to && own)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = 32 * t + 16 * (e / 8) + row + e % 8;
                if (r < a.dim_k) to[r * a.dim_v + my_c] = s[t][e];
            }
}

// What each part begins with, in place of what it would leave by itself: in the order of the parts, four values by a thread, what eight parts
// leave being read at a time (16 heads x 32 parts of 128 x 128: 17.5 us one after the other, 14.6 so).
__global__ void __launch_bounds__(256) k_decay_scan(idf_decay_args a, Parts parts)
{
    const int kv = blockIdx.y % a.heads_kv, seg = blockIdx.y / a.heads_kv;
    const int x = (blockIdx.x * 256 + threadIdx.x) * 4, size = a.dim_k * a.dim_v;
    const Segment g = segment_of(a, seg, nullptr);
    if (!g.valid || x >= size) return;
    const int n = max(1, (g.len + parts.tokens - 1) / parts.tokens);
    const Factor keep = factor_of(exp2((double)parts.tokens * (double)log2_of(a.log_decay[kv])));
    float *at = parts.states + (int64_t)blockIdx.y * parts.n * size + x;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (a.state_in) s = *(const f32x4 *)(a.state_in + ((int64_t)g.ring * a.heads_kv + kv) * size + x);
    constexpr int kAhead = 8;
    for (int p0 = 0; p0 < n; p0 += kAhead, at += (int64_t)kAhead * size) {
        f32x4 left[kAhead];                        // (what lies in the last part's place is read and not used)
#pragma unroll
        for (int y = 0; y < kAhead; ++y) left[y] = *(const f32x4 *)(at + (int64_t)min(y, n - 1 - p0) * size);
#pragma unroll
        for (int y = 0; y < kAhead; ++y) {
            if (p0 + y >= n) break;
            *(f32x4 *)(at + (int64_t)y * size) = s;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = keep.times(s[e]) + left[y][e];
        }
    }
}

Parts parts_of(const idf_decay_args &a)
{
    Parts p;
    p.states = nullptr;
    const int64_t max_tokens = longest(a);
    // as many workgroups as the machine holds, by the tokens that there are and not by the longest segment's (uneven segments 87 -> 81 us); a part
    // is long next to the state that it reads and writes, and states that mostly empty segments would not use stay few (512 MB of 128 x 128)
    const int64_t pairs = (int64_t)a.n_segments * a.heads_kv, tokens = std::max<int64_t>(1, std::min(a.n_tokens, a.n_segments * max_tokens) * a.heads_kv * ((a.dim_v + 127) / 128));
    // Where few workgroups run, a part's chunks follow each other by latency: up to sixteen parts, of a chunk at least, then of 128 tokens; the two
    // launches more pay from 256 tokens on, 128 in float32 (us per call with parts of 256 tokens and so: 400 tokens, 16 heads of 128 x 128 32 -> 24; 800
    // tokens, a head of 64 x 64 30 -> 15, in float32 68 -> 24).
    const int64_t held = a.precision == IDF_PREC_F32 && a.dim_k > 64 ? 256 : 512;        // workgroups of the machine: by their LDS one or two to a compute unit
    const int64_t part = std::min<int64_t>(std::max<int64_t>(max_tokens / 16, kChunk), 128);
    const int64_t most = max_tokens < (a.precision == IDF_PREC_BF16 ? 256 : 128) ? 1 : max_tokens / part;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>({max_tokens * held / tokens, most, 8192 / std::max<int64_t>(pairs, 1)}));
    p.tokens = (int)(((max_tokens + want - 1) / want + kChunk - 1) / kChunk * kChunk);
    p.n = (int)((max_tokens + p.tokens - 1) / std::max(p.tokens, 1));
    if (p.n <= 1) { p.n = 1; p.tokens = std::max(p.tokens, kChunk); }
    return p;
}

// Token by token or by chunks.  A chunk costs the same whatever it holds, each token by itself about 3 us more (us per call, tokens against
// chunk: 64 streams x 16 heads of 128 x 128 in bfloat16 26.6 : 28.2 for one token, 30 : 28.2 for two; 16 streams x 8 heads x 4 queries of 64 x 64
// 8.0 : 8.7 and 12.0 : 8.7).  In float32 a chunk takes eight instructions for one: 64 streams x 4 heads of 64 x 64 9.5 : 10.2 for four tokens, 10.4 : 10.2
// for five; x 16 heads of 128 x 128, 35 : 61 for four and about level, 63 : 61, at twelve.  There is no chunk form for keys of more than 128 values:
// they go token by token whatever their number, some 4 to 6 us a token (4000 tokens, 8 heads of 256 x 64: 22.9 ms, in float32 16.2 ms).
bool by_token(const idf_decay_args &a)
{
    const int most = a.precision == IDF_PREC_BF16 ? 1 : a.dim_k <= 64 ? 4 : 12;
    return longest(a) <= most || a.dim_k > 128;
}

template <int PREC, int DK>
hipError_t chunks(const idf_decay_args &a, const LaunchCtx &lc)
{
    Parts p = parts_of(a);
    const int waves = a.dim_v <= 64 ? 2 : 4, blocks = (a.dim_v + 32 * waves - 1) / (32 * waves);
    const dim3 grid((unsigned)((int64_t)a.n_segments * a.heads_kv * blocks), p.n);
    auto go = [&](auto states_only) {
        constexpr bool S = decltype(states_only)::value;
        return waves == 2 ? launch(k_decay_chunks<PREC, DK, 2, S>, grid, dim3(128), 0, lc, a, p, blocks) : launch(k_decay_chunks<PREC, DK, 4, S>, grid, dim3(256), 0, lc, a, p, blocks);
    };
    hipError_t e = hipSuccess;
    if (p.n > 1) {
        p.states = (float *)a.workspace;
        e = go(std::true_type{});
        if (e == hipSuccess)
            e = launch(k_decay_scan, dim3((unsigned)((a.dim_k * a.dim_v + 1023) / 1024), a.n_segments * a.heads_kv), dim3(256), 0, lc, a, p);
    }
    return e == hipSuccess ? go(std::false_type{}) : e;
}

template <int PREC>
hipError_t tokens(const idf_decay_args &a, const LaunchCtx &lc)
{
    const int column_groups = (a.dim_v + 31) / 32;
    const dim3 grid((unsigned)(((int64_t)a.heads_kv * column_groups + 3) / 4), a.n_segments);
    if (a.dim_k <= 64) return launch(k_decay_tokens<PREC, 8>, grid, dim3(256), 0, lc, a, column_groups);
    if (a.dim_k <= 128) return launch(k_decay_tokens<PREC, 16>, grid, dim3(256), 0, lc, a, column_groups);
    return launch(k_decay_tokens<PREC, 32>, grid, dim3(256), 0, lc, a, column_groups);
}

template <int PREC>
hipError_t by_shape(const idf_decay_args &a, const LaunchCtx &lc)
{
    if (by_token(a)) return tokens<PREC>(a, lc);
    return a.dim_k <= 64 ? chunks<PREC, 64>(a, lc) : chunks<PREC, 128>(a, lc);
}

}  // namespace

size_t decay_workspace(const idf_decay_args &a)
{
    const Parts p = parts_of(a);
    return !by_token(a) && p.n > 1 ? (size_t)a.n_segments * a.heads_kv * p.n * a.dim_k * a.dim_v * sizeof(float) : 0;
}

hipError_t launch_decay(const idf_decay_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? by_shape<IDF_PREC_F32>(a, lc) : by_shape<IDF_PREC_BF16>(a, lc);
}

}  // namespace idf
