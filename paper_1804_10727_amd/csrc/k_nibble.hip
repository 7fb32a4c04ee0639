// The ring of keys and values in 4 bits: appending to it, attention over it, and what it stands for (idf_nibble_append, idf_nibble_attend,
// idf_nibble_values).
//
// A block is 32 values of a head and a power of two; a code is one of this machine's 4-bit floating-point numbers (one bit of mantissa, two of exponent), so that
// one instruction takes two codes and the power to two bfloat16 values, exactly.  From there attention goes as over a ring of bfloat16: scores S^T = K Q^T,
// the softmax per lane, O^T = V^T P^T; a quarter of the bytes is read.  Queries and weights in float32 enter the bfloat16 instructions as three numbers that add up to
// them (24 bits), which costs three instructions where float32 ones would take eight times as long; in bfloat16 weights are rounded once, as in the window's
// attention.  Sums, maxima and outputs are float32.
#include <algorithm>

#include "idf.h"
#include "seq_split.h"

namespace idf {

namespace {

constexpr int kBits = 32;                          // values of a block
constexpr int kStepRows = 32;                      // query rows of a segment and key/value head that the step kernel takes, in one or two tiles of 16
constexpr int kTileRows = 128;                     // query rows of a workgroup of the tile kernel
constexpr int kMostTokens = 8;                     // of a workgroup that appends

typedef __attribute__((ext_vector_type(2))) float f32x2;

// The power of two of a block as the conversions take it: the exponent of a float32 (255: not a number, and so is what they give).
__device__ __forceinline__ float power_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Eight codes as eight bfloat16 values.
__device__ __forceinline__ bf16x8 values8(uint32_t codes, float power)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float value_of(const uint8_t *codes, const uint8_t *scales, int d)
{
    const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)codes[d >> 1], power_of(scales[d / kBits]), 0);
    return d & 1 ? v[1] : v[0];
}

// Rows of a stream's head: codes of head_dim / 2 bytes, scales of head_dim / 32, from a slot on.
template <class B> struct Held4 {
    B *codes, *scales;
    __device__ __forceinline__ Held4(B *c, B *s, int64_t slots, int heads, int head_dim, int ring, int h)
    {
        const int64_t row = ((int64_t)ring * heads + h) * slots;
        codes = c + row * (head_dim / 2);
        scales = s + row * (head_dim / kBits);
    }
};

// ---- appending ----

// float64 to the float32 that rounds to any shorter number as it does itself: towards zero, with the last bit set where something is cut off.
__device__ __forceinline__ float to_odd(double d)
{
    const float f = (float)d;
    const double back = f;
    uint32_t bits = __builtin_bit_cast(uint32_t, f);
    if (back != d) {
        if (__builtin_fabs(back) > __builtin_fabs(d)) --bits;
        bits |= 1u;
    }
    return __builtin_bit_cast(float, bits);
}

// The smallest power with most <= 7 * 2^power, 7 being 1.75 * 2^2: from the exponent and the mantissa of most, held to what a block can have.
__device__ __forceinline__ int power_for(float most)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, most);
    return min(max((int)(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 2 : 1), -100), 125);
}
__device__ __forceinline__ int power_for(double most)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, most);
    return min(max((int)(bits >> 52) - 1023 - ((bits & 0xfffffffffffffull) <= 0xc000000000000ull ? 2 : 1), -100), 125);
}

// A lane's neighbours within four and within a row of 16, without a way through LDS: v with those of lanes that lie apart by a mask, or mirrored.
template <int CTRL> __device__ __forceinline__ float moved(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 15, 15, false)); }
template <int CTRL> __device__ __forceinline__ double moved(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t low = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)b, CTRL, 15, 15, false), high = (uint32_t)__builtin_amdgcn_mov_dpp((int)(b >> 32), CTRL, 15, 15, false);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
constexpr int kApart1 = 0xb1, kApart2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;           // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
template <class F> __device__ __forceinline__ F block_max(F v)
{
    v = __builtin_elementwise_max(v, moved<kApart1>(v));
    return __builtin_elementwise_max(v, moved<kApart2>(v));
}
// Over 1 << lanes_log2 lanes, four at least.
__device__ __forceinline__ double lanes_sum(double v, int lanes_log2)
{
    v += moved<kApart1>(v);
    v += moved<kApart2>(v);
    if (lanes_log2 > 2) v += moved<kMirror8>(v);
    if (lanes_log2 > 3) v += moved<kMirror16>(v);
    if (lanes_log2 > 4) v += __shfl_xor(v, 16);
    return v;
}

__device__ __forceinline__ uint32_t to_codes(const float (&f)[8], float by)
{
    uint32_t codes = 0u;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], by, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], by, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], by, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], by, 3);
    return codes;
}

// Eight values of a lane, a block being four neighbouring lanes': codes, and the byte of the power.  EXACT: y are the values themselves; else they were rounded from 64
// bits, and close says whether one of them lies on a middle between two codes, or the largest on the border between two powers (a multiple of a quarter of the
// power), where that rounding may have decided.
template <bool EXACT> __device__ __forceinline__ uint32_t encode(const float (&y)[8], uint32_t &byte, bool &close)
{
    float most = 0.f, none = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        none = __builtin_fmaf(y[e], 0.f, none);
        most = fmaxf(most, __builtin_fabsf(y[e]));
    }
    if (!(none == 0.f)) most = __builtin_inff();
    most = block_max(most);
    byte = 255u;
    close = !EXACT;                                // (what is finite in 64 bits may be none of float32)
    if (!(most < __builtin_inff())) return 0u;
    const int power = power_for(most);
    byte = (uint32_t)(power + 127);
    const float four = power_of((uint32_t)(129 - power));                     // 4 / 2^power
    float f[8], off = 1.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = y[e] * four;
        if (!EXACT) off = fminf(off, __builtin_amdgcn_fractf(f[e]));
        f[e] = __builtin_amdgcn_fmed3f(f[e], -24.f, 24.f);                    // (beyond 6: 6)
    }
    close = !EXACT && off == 0.f;
    return to_codes(f, 4.f);
}
// The same of 64 bits.
__device__ __forceinline__ uint32_t encode_exact(const double (&y)[8], uint32_t &byte)
{
    double most = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = __builtin_fabs(y[e]) <= 0x1.fffffffffffffp+1023 ? fmax(most, __builtin_fabs(y[e])) : __builtin_inf();
    most = block_max(most);
    byte = 255u;
    if (!(most < __builtin_inf())) return 0u;
    const int power = power_for(most);
    byte = (uint32_t)(power + 127);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __builtin_amdgcn_fmed3f(to_odd(y[e] * __builtin_bit_cast(double, (uint64_t)(1023 - power) << 52)), -6.f, 6.f);
    return to_codes(f, 1.f);
}

// Eight values as they lie in memory: those of 16 bits stay two to a register until they are asked for.
template <int PREC> struct alignas(16) Eight {
    using T = typename Elem<PREC>::type;
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[e]);
        else return __builtin_bit_cast(float, e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
    __device__ __forceinline__ static uint32_t bits(T v) { if constexpr (sizeof(T) == 4) return __builtin_bit_cast(uint32_t, v); else return __builtin_bit_cast(uint16_t, v); }
    // eight values from there, or the n first of them (with whatever behind them)
    __device__ __forceinline__ void load(const T *from, bool aligned, int n)
    {
        if (aligned && n >= 8) { *this = *(const Eight *)from; return; }
#pragma unroll
        for (int i = 0; i < (int)(2 * sizeof(T)); ++i) w[i] = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) w[e * sizeof(T) / 4] |= bits(from[e]) << (sizeof(T) == 4 ? 0 : 16 * (e % 2));
    }
};

// A lane has eight values of a head, four lanes a block; a workgroup a few tokens with all their heads, so that slots, cosines and sines are formed once per
// token.  Keys that are normalised or turned are formed in 64 bits, whose instructions run as fast as those of 32 here: a value next to the middle between two codes goes to
// the same one however sums and products are ordered.  (So it would by 32 bits with a border of their error about every middle, and 64 for what lies in it; not built.)
//   What is read and written asks for 17 us of 15,104 tokens with 8 heads of 128 in bfloat16; it takes 38.5, by the vector instructions and 5 to 12 registers that go to scratch
// memory (with every code decided in 64 bits 97; with a workgroup per token 52; with keys on the same two of a workgroup's waves, and so on two SIMDs of four, 46).  One token
// of 64 streams: 5.7 us.
template <int PREC, bool ALIGNED>
__global__ void __launch_bounds__(256, 4) k_nibble_append(idf_nibble_append_args a, int lanes_log2, int tokens_per_group)
{
    using T = typename Elem<PREC>::type;
    extern __shared__ double2 turn[];              // [token][rotary_dim / 2]: amplitude * (cos, sin)
    __shared__ int64_t slots[kMostTokens];         // of each token; negative: none
    __shared__ __align__(16) float weight[256];
    const Segment g = segment_of(a, blockIdx.y, a.starts);
    const int t0 = blockIdx.x * tokens_per_group;
    if (t0 >= g.len) return;
    const int n = min(tokens_per_group, g.len - t0), half = a.rotary_dim / 2;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), c = lane * 8, heads = a.heads_kv, d = a.head_dim;
    const bool on = c < d, plain = !a.k_weight && !half;
    const float per_token = 1.f / (float)(2 * heads);
    const double per_value = 1.0 / d;
    // a row of a head, and what lies in a pair with this lane's values in the other half of what is turned; the next one is on its way while this one is worked on
    struct Row { int t, h; bool key; Eight<PREC> x, other; };
    const int total = n * 2 * heads, step = 256 >> lanes_log2;
    const T *const k0 = (const T *)a.k.base + (g.begin + t0) * a.k.token_stride, *const v0 = (const T *)a.v.base + (g.begin + t0) * a.v.token_stride;
    auto fetch = [&](int row, Row &r) IDF_INLINE {
        r.t = (int)(((float)row + 0.5f) * per_token);                          // (fewer than 2^15 rows: exact)
        const int which = row - r.t * 2 * heads;
        r.key = (which < heads) != (bool)((t0 + r.t) & 1);                     // (keys take longer: a wave has those of every other token)
        r.h = which < heads ? which : which - heads;
        if (!on) return;
        const T *src = r.key ? k0 + r.t * a.k.token_stride + r.h * a.k.head_stride : v0 + r.t * a.v.token_stride + r.h * a.v.head_stride;
        r.x.load(src + c, ALIGNED, 8);
        if (r.key && c < a.rotary_dim && !a.interleaved) {
            if (half % 8 == 0) {
                r.other.load(src + (c < half ? c + half : c - half), ALIGNED, 8);
            } else {
                Pack<T, 8> p = {};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < a.rotary_dim) p.v[e] = src[c + e < half ? c + e + half : c + e - half];
                r.other.load(p.v, false, 8);
            }
        }
    };
    const int row0 = threadIdx.x >> lanes_log2;
    Row next = {};                                 // (lanes that have no values keep zeros)
    if (row0 < total) fetch(row0, next);
    if ((int)threadIdx.x < n) {
        const int64_t period = a.slots - a.sinks, p = g.start + t0 + threadIdx.x;
        slots[threadIdx.x] = p < a.sinks ? p : t0 + (int)threadIdx.x < g.len - period ? -1 : a.sinks + (p - a.sinks) % period;
    }
    if (a.k_weight && (int)threadIdx.x < a.head_dim) weight[threadIdx.x] = a.k_weight[threadIdx.x];
    for (int i = threadIdx.x; i < n * half; i += 256) {
        const int t = i / half;
        double s, c;
        sincos((double)(g.start + t0 + t) * a.frequencies[i - t * half], &s, &c);
        turn[i] = make_double2(a.amplitude * c, a.amplitude * s);
    }
    __syncthreads();
    const uint64_t ring = (uint64_t)g.ring * heads * a.slots;
    for (int row = row0; row < total; row += step) {
        const Row now = next;
        if (row + step < total) fetch(row + step, next);
        const int t = now.t, h = now.h;
        const bool key = now.key;
        const int64_t slot = slots[t];
        if (slot < 0) continue;
        uint32_t codes, byte;
        if (!key || plain) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = now.x.get(e);
            bool close;
            codes = encode<true>(x, byte, close);
        } else {
            double y[8], norm = 1.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = now.x.get(e);
            if (a.k_weight) {
                double sum = 0.0;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += y[e] * y[e];
                // 1 / sqrt by the instruction's start (some 26 bits) and two steps
                sum = lanes_sum(sum, lanes_log2) * per_value + a.eps;
                norm = __builtin_amdgcn_rsq(sum);
#pragma unroll
                for (int i = 0; i < 2; ++i) norm = norm * __builtin_fma(-0.5 * sum * norm, norm, 1.5);
                if (sum == __builtin_inf()) norm = 0.0;
                if (on)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= norm * weight[c + e];
            }
            if (on && c < a.rotary_dim) {
                const double2 *cs = turn + t * half;
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        if (c + e >= a.rotary_dim) continue;
                        const double2 r = cs[(c + e) / 2];
                        const double u = y[e], w = y[e + 1];
                        y[e] = u * r.x - w * r.y;
                        y[e + 1] = w * r.x + u * r.y;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int i = c + e, j = i < half ? i + half : i - half;
                        if (i >= a.rotary_dim) continue;
                        const double q = now.other.get(e), o = a.k_weight ? q * (norm * weight[j]) : q;
                        const double2 r = cs[i < half ? i : j];
                        y[e] = y[e] * r.x + (i < half ? -o : o) * r.y;
                    }
                }
            }
            float near[8];
            bool close;
#pragma unroll
            for (int e = 0; e < 8; ++e) near[e] = (float)y[e];
            codes = encode<false>(near, byte, close);
            if (__ballot(close)) codes = encode_exact(y, byte);
        }
        const uint64_t place = ring + (uint64_t)(uint32_t)h * (uint32_t)a.slots + (uint32_t)slot;
        if (on) *(uint32_t *)((key ? a.ring.k_codes : a.ring.v_codes) + (place * (uint32_t)(d / 2) + c / 2)) = codes;
        if (on && lane % 4 == 0) (key ? a.ring.k_scales : a.ring.v_scales)[place * (uint32_t)(d / kBits) + lane / 4] = (uint8_t)byte;
    }
}

// ---- what a ring stands for ----

// A workgroup takes a head of a stream's keys or values and some of its slots, a lane eight values at a time: lanes read and write next to each other.  Bound by memory, most
// of it what is written: 8 streams of 4100 slots with 8 heads of 128 to bfloat16 in 28 us, 170 MB, 6.0 TB/s.
template <int PREC>
__global__ void __launch_bounds__(256) k_nibble_values(idf_nibble_values_args a)
{
    using T = typename Elem<PREC>::type;
    constexpr int kAhead = 4;
    const int lanes = a.head_dim / 8, rows = 256 / lanes, row = threadIdx.x / lanes, at = threadIdx.x - row * lanes;
    if (row >= rows) return;
    const int64_t head = blockIdx.y, stream = head / a.heads_kv, h = head - stream * a.heads_kv;
    const bool key = blockIdx.z == 0;
    const uint8_t *codes = (key ? a.ring.k_codes : a.ring.v_codes) + head * a.slots * (a.head_dim / 2) + at * 4;
    const uint8_t *scales = (key ? a.ring.k_scales : a.ring.v_scales) + head * a.slots * (a.head_dim / kBits) + at / 4;
    T *to = (T *)(key ? a.k : a.v) + (stream * a.slots * a.heads_kv + h) * a.head_dim + at * 8;
    const int64_t step = (int64_t)gridDim.x * rows;
    for (int64_t s = (int64_t)blockIdx.x * rows + row; s < a.slots; s += kAhead * step) {
        uint32_t c[kAhead], p[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t slot = min(s + u * step, a.slots - 1);
            c[u] = *(const uint32_t *)(codes + slot * (a.head_dim / 2));
            p[u] = scales[slot * (a.head_dim / kBits)];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (s + u * step >= a.slots) break;
            const bf16x8 v = values8(c[u], power_of(p[u]));
            Pack<T, 8> out;
#pragma unroll
            for (int e = 0; e < 8; ++e) out.v[e] = Elem<PREC>::from_f32((float)v[e]);
            *(Pack<T, 8> *)(to + (s + u * step) * a.heads_kv * a.head_dim) = out;
        }
    }
}

// ---- attention ----

// The keys that query positions first .. last see, as a list in order of position: first tokens of the stream, then from the beginning of the
// oldest window on.  Position p sees entry i if i <= p - shift and (i > p - window - shift or i < n_first).
struct Keys {
    int n, n_first;            // entries, and how many of them are first tokens ahead of the window
    uint32_t slot0, period;    // ring slot, counted behind the first tokens, of entry n_first
    int64_t shift;             // position of entry i >= n_first is i + shift
    int sinks;
    __device__ __forceinline__ Keys(const idf_nibble_attend_args &a, int64_t p0, int64_t p1)
    {
        const int64_t first = min((int64_t)a.sinks, p1 + 1), low = max(first, p0 - a.window + 1);
        n_first = (int)first;
        shift = low - first;
        n = (int)(p1 - shift + 1);
        period = (uint32_t)(a.slots - a.sinks);
        slot0 = low >= a.sinks ? (uint32_t)((low - a.sinks) % period) : 0u;
        sinks = a.sinks;
    }
    __device__ __forceinline__ uint32_t slot(int i) const
    {
        uint32_t s = slot0 + (uint32_t)(i - n_first);
        if (s >= period) s -= period;
        return i < n_first ? (uint32_t)i : (uint32_t)sinks + s;
    }
};

// Numbers of float32 as PARTS bfloat16 ones that add up to them.
template <int PREC> struct Parts { static constexpr int N = PREC == IDF_PREC_BF16 ? 1 : 3; };
template <int N> __device__ __forceinline__ void in_parts(const float (&v)[8], bf16x8 (&to)[N])
{
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            to[p][e] = (__bf16)rest[e];
            if (p + 1 < N) rest[e] -= (float)to[p][e];
        }
}
// Eight values of a query row that has n from p on (n a multiple of 8; zeros behind them).
template <int PREC> __device__ __forceinline__ void load_query(const typename Elem<PREC>::type *p, int n, bf16x8 (&to)[Parts<PREC>::N])
{
    if constexpr (PREC == IDF_PREC_BF16) {
        to[0] = Mfma<IDF_PREC_BF16>::load(p, n);
    } else {
        const f32x8 v = Mfma<IDF_PREC_F32>::load(p, n);
        const float w[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
        in_parts(w, to);
    }
}

// A row whose sums came out infinite or not a number: once more, by one wave, reading only the values that the row sees -- on the matrix cores a weight of
// zero times what is not a number, and is seen by another row, would be no zero.
template <int PREC>
__device__ __forceinline__ void exact_row(const idf_nibble_attend_args &a, const Segment &g, const Keys &keys, int kv, int h, int t, int i0, int i1, const Partial &part, int split)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    const int lane = threadIdx.x & 63;
    const int64_t p = g.start + t, token = g.begin + t;
    const int hi = (int)(p - keys.shift);
    const int64_t lo = p - a.window - keys.shift;
    const T *q = (const T *)a.q.base + token * a.q.token_stride + h * a.q.head_stride;
    const Held4<const uint8_t> kh(a.ring.k_codes, a.ring.k_scales, a.slots, a.heads_kv, a.head_dim, g.ring, kv), vh(a.ring.v_codes, a.ring.v_scales, a.slots, a.heads_kv, a.head_dim, g.ring, kv);
    const int row_codes = a.head_dim / 2, row_scales = a.head_dim / kBits;
    float m = -__FLT_MAX__, l = 0.f, o[4] = {};
    for (int b = i0; b < i1; b += 64) {
        const int i = b + lane;
        const bool seen = i < i1 && i <= hi && (i > lo || i < keys.n_first);
        float s = -__builtin_inff();
        if (seen) {
            const int64_t slot = keys.slot(i);
            s = 0.f;
            for (int d = 0; d < a.head_dim; ++d) s += E::to_f32(q[d]) * value_of(kh.codes + slot * row_codes, kh.scales + slot * row_scales, d);
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
            const int64_t slot = keys.slot(b + j);
            const float wj = __shfl(w, j);
            for (int c = 0; c < 4; ++c)
                if (lane + 64 * c < a.head_dim) o[c] += wj * value_of(vh.codes + slot * row_codes, vh.scales + slot * row_scales, lane + 64 * c);
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

// -- few rows on a long axis: single tokens, short segments --

// A workgroup takes the at most 16 RT query rows of one segment and key/value head and a part of the keys; its waves take 32 of them at a time, in turn, each
// with a softmax of its own, and are joined at the end.  Eight waves where one workgroup to a compute unit is enough (64 x 16 tokens in float32 on 1000 keys of
// 4 x 64: 20.7 us by four, 17.6 by eight, before what is said of LDS below), else four with two rounds each on their way (64 streams on 4096 keys of 8 x 128: one round 61.6, two 56.5; reading alone, with
// nothing done, takes 52, 5.5 TB/s).  What had cost most were choices on the loaded values next to the loads, which wait for them (72 -> 62).  Codes of keys go from memory into the layout of the matrix instruction, a lane having a quarter of a
// row, whose place along the summed axis is free; those of values through a piece of LDS that is the wave's own, to be read along the keys.
template <int PREC, int DP, int RT, int WAVES> struct StepShape {
    static constexpr int KEYS = 32, NT = 2;
    static constexpr int AHEAD = WAVES == 4 && DP <= 128 && !(PREC == IDF_PREC_F32 && DP == 128 && RT == 2) ? 2 : 1;      // rounds that a wave has on their way
    static constexpr int STRIDE = DP + 16;                                    // of a row of values in LDS: rows that are read together begin in banks of their own
    static constexpr int BLOCKS = DP / kBits;                                 // of a row
    static constexpr int LOADS = (KEYS * BLOCKS + 63) / 64;                   // of 16 bytes of values per lane
    static constexpr int K_WORDS = DP / 32;                                   // words of eight codes of a key per lane
    static constexpr int K_POWERS = DP == 256 ? 2 : 1;
    static constexpr int OUT = DP + 4;                                        // of a row of sums there
    static constexpr int WAVE_FLOATS = 16 * RT * OUT > KEYS * STRIDE / 2 ? 16 * RT * OUT : KEYS * STRIDE / 2;
};
// In LDS a block's four pieces of eight values change places, x to x ^ turn: eight lanes that write a piece each, of blocks that follow each other, then write to banks of
// their own; rows of sums that are joined there begin four banks apart.  (Without either the 16 tokens of 64 streams above took 16.8 us in a call, with them 15.5; a token on
// 65,536 keys 22.5 and 21.2.)  read_turned: the values of read_column that lie so, of columns 16 d on.
template <int DP> __device__ __forceinline__ int step_turn(int row, int block) { return DP == 64 ? row >> 1 & 1 : DP == 128 ? block >> 1 & 1 : block >> 1 & 3; }
template <int DP> __device__ __forceinline__ bf16x8 read_turned(const __bf16 *lds, int stride, int d, int r0, int r1)
{
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const int lane = threadIdx.x & 15, r = lane >> 2, at = r * stride + d / 2 * kBits + (((d & 1) << 1 | (lane >> 1 & 1)) ^ step_turn<DP>(r, d / 2)) * 8 + (lane & 1) * 4;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r0 * stride + at));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r1 * stride + at));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int PREC, int DP, int RT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 8 || DP <= 128 ? 2 : 1) k_nibble_step(idf_nibble_attend_args a, int splits)
{
    using M = Mfma<IDF_PREC_BF16>;
    using T = typename Elem<PREC>::type;
    using S = StepShape<PREC, DP, RT, WAVES>;
    constexpr int NT = S::NT, KS = DP / 32, DT = DP / 16, N = Parts<PREC>::N;
    extern __shared__ __align__(16) float lds[];
    __shared__ float stats[2][WAVES][16 * RT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    const int split = blockIdx.x, kv = blockIdx.y, group = a.heads_q / a.heads_kv;
    const Segment g = segment_of(a, blockIdx.z, a.starts);
    if (g.len == 0) return;
    const int rows = min(g.len * group, 16 * RT);
    const Keys keys(a, g.start, g.start + g.len - 1);
    const Held4<const uint8_t> kh(a.ring.k_codes, a.ring.k_scales, a.slots, a.heads_kv, a.head_dim, g.ring, kv), vh(a.ring.v_codes, a.ring.v_scales, a.slots, a.heads_kv, a.head_dim, g.ring, kv);
    const Partial part = partial_of(a, splits);
    const uint32_t row_codes = a.head_dim / 2, row_scales = a.head_dim / kBits;

    // this split's entries, whole tiles of them; the waves take them in turn
    const int tiles = (keys.n + S::KEYS - 1) / S::KEYS, per = (tiles + splits - 1) / splits;
    const int t0 = split * per, t1 = min(tiles, t0 + per);
    const float scale = a.scale * kLog2e;
    int hi[RT], lo[RT];                                                       // what this lane's query rows see

    // of the summed axis a lane has: 64 values a head, 16 grp + 8 s ..; 128, 32 grp + 8 s ..; 256, 32 (grp + 4 (s / 4)) + 8 (s % 4) ..
    auto dim_of = [&](int s) IDF_INLINE { return DP == 64 ? 16 * grp + 8 * s : DP == 128 ? 32 * grp + 8 * s : 32 * (grp + 4 * (s / 4)) + 8 * (s % 4); };
    bf16x8 q[RT][KS][N];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = 16 * r + col, t = min(row, rows - 1) / group, h = kv * group + min(row, rows - 1) - t * group;
        const int64_t p = g.start + t;
        hi[r] = (int)(p - keys.shift);
        lo[r] = (int)max(p - a.window - keys.shift, (int64_t)-1);
        const T *src = (const T *)a.q.base + (g.begin + t) * a.q.token_stride + h * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < KS; ++s) load_query<PREC>(src + dim_of(s), row < rows ? a.head_dim - dim_of(s) : 0, q[r][s]);
    }

    __bf16 *v_lds = (__bf16 *)(lds + wave * S::WAVE_FLOATS);
    struct Round { uint32_t kc[NT][S::K_WORDS], kp[NT][S::K_POWERS], vp[S::LOADS]; i32x4 vc[S::LOADS]; };
    // Places behind a row's end are those of its first block again: there queries are zeros, and outputs nobody's.  Rounds that lie in one piece are read
    // from one address on, the others (first tokens, the ring's end, the list's) look for the place of each entry.
    uint32_t k_at[S::K_POWERS], k_power_at[S::K_POWERS];
#pragma unroll
    for (int x = 0; x < S::K_POWERS; ++x) {
        const int d = dim_of(4 * x), there = d < a.head_dim ? d : 0;
        k_at[x] = there / 2;
        k_power_at[x] = there / kBits;
    }
    auto load_from = [&](Round &r, const uint8_t *kc, const uint8_t *kp, const uint8_t *vc, const uint8_t *vp, auto slot_of) IDF_INLINE {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t slot = slot_of(16 * t + col);
#pragma unroll
            for (int x = 0; x < S::K_POWERS; ++x) {
                r.kp[t][x] = kp[slot * row_scales + k_power_at[x]];
                if constexpr (DP == 64) {
                    const uint2 w = *(const uint2 *)(kc + (slot * row_codes + k_at[x]));
                    r.kc[t][0] = w.x; r.kc[t][1] = w.y;
                } else {
                    const i32x4 w = *(const i32x4 *)(kc + (slot * row_codes + k_at[x]));
#pragma unroll
                    for (int s = 0; s < 4; ++s) r.kc[t][4 * x + s] = (uint32_t)w[s];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int piece = j * 64 + lane, row = min(piece / S::BLOCKS, S::KEYS - 1), b = piece % S::BLOCKS;
            const uint32_t slot = slot_of(row), block = b * kBits < a.head_dim ? b : 0;
            r.vp[j] = vp[slot * row_scales + block];
            r.vc[j] = *(const i32x4 *)(vc + (slot * row_codes + block * 16));
        }
    };
    auto load = [&](int tile, Round &r) IDF_INLINE {
        const int i0 = tile * S::KEYS;
        uint32_t at = keys.slot0 + (uint32_t)(i0 - keys.n_first);
        if (at >= keys.period) at -= keys.period;
        if (i0 >= keys.n_first && i0 + S::KEYS <= keys.n && at + S::KEYS <= keys.period) {
            const int64_t slot = (int64_t)keys.sinks + at;
            load_from(r, kh.codes + slot * row_codes, kh.scales + slot * row_scales, vh.codes + slot * row_codes, vh.scales + slot * row_scales, [](int e) { return (uint32_t)e; });
        } else {
            load_from(r, kh.codes, kh.scales, vh.codes, vh.scales, [&](int e) { return keys.slot(min(i0 + e, keys.n - 1)); });
        }
    };

    f32x4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -__FLT_MAX__;
        l[r] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto work = [&](int tile, Round &x_) IDF_INLINE {
        const auto &kc = x_.kc; const auto &kp = x_.kp; const auto &vp = x_.vp; const auto &vc = x_.vc;
        f32x4 st[RT][NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int r = 0; r < RT; ++r) st[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 k = values8(kc[t][s], power_of(kp[t][s / 4]));
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int x = N - 1; x >= 0; --x) st[r][t] = M::mma16(k, q[r][s][x], st[r][t]);
            }
        }
        __builtin_amdgcn_wave_barrier();                                      // (LDS serves a wave in order: only the compiler has to keep it)
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int piece = j * 64 + lane, r = piece / S::BLOCKS, b = piece - r * S::BLOCKS;
            const float power = power_of(vp[j]);
            if (S::KEYS * S::BLOCKS % 64 == 0 || piece < S::KEYS * S::BLOCKS)
#pragma unroll
                for (int w = 0; w < 4; ++w) *(bf16x8 *)(v_lds + r * S::STRIDE + b * kBits + 8 * (w ^ step_turn<DP>(r, b))) = values8((uint32_t)vc[j][w], power);
        }
        __builtin_amdgcn_wave_barrier();
        if (tile + WAVES * S::AHEAD < t1) load(tile + WAVES * S::AHEAD, x_);

        bf16x8 pf[RT][N];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float w[NT * 4], top = m[r];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = tile * S::KEYS + 16 * t + 4 * grp + e;
                    const bool seen = i <= hi[r] && (i > lo[r] || i < keys.n_first);
                    w[4 * t + e] = seen ? st[r][t][e] * scale : -__builtin_inff();
                    top = fmaxf(top, w[4 * t + e]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__ballot(top > m[r])) {
                const float fade = __builtin_amdgcn_exp2f(m[r] - top);
                l[r] *= fade;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[r][d] *= fade;
                m[r] = top;
            }
#pragma unroll
            for (int e = 0; e < NT * 4; ++e) { w[e] = __builtin_amdgcn_exp2f(w[e] - m[r]); l[r] += w[e]; }
            in_parts(w, pf[r]);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const bf16x8 v = read_turned<DP>(v_lds, S::STRIDE, d, 4 * grp, 16 + 4 * grp);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int x = N - 1; x >= 0; --x) o[r][d] = M::mma16(v, pf[r][x], o[r][d]);
        }
    };
    Round rounds[S::AHEAD];
#pragma unroll
    for (int x = 0; x < S::AHEAD; ++x)
        if (t0 + wave + WAVES * x < t1) load(t0 + wave + WAVES * x, rounds[x]);
    for (int tile = t0 + wave; tile < t1; tile += WAVES * S::AHEAD)
#pragma unroll
        for (int x = 0; x < S::AHEAD; ++x)
            if (tile + WAVES * x < t1) work(tile + WAVES * x, rounds[x]);

    // the waves' rows joined: [wave][row][value]
    __builtin_amdgcn_wave_barrier();
    float *mine = lds + wave * S::WAVE_FLOATS;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        l[r] += __shfl_xor(l[r], 16);
        l[r] += __shfl_xor(l[r], 32);
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4 *)(mine + (16 * r + col) * S::OUT + 16 * d + 4 * grp) = o[r][d];
        if (grp == 0) { stats[0][wave][16 * r + col] = m[r]; stats[1][wave][16 * r + col] = l[r]; }
    }
    __syncthreads();
    bool bad = false;
    constexpr int V4 = DP / 4;
    for (int x = threadIdx.x; x < rows * V4; x += 64 * WAVES) {
        const int r = x / V4, c = (x - r * V4) * 4;
        float top = -__FLT_MAX__, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stats[0][w][r]);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float fade = __builtin_amdgcn_exp2f(stats[0][w][r] - top);
            sum += fade * stats[1][w][r];
            v += fade * *(const f32x4 *)(lds + w * S::WAVE_FLOATS + r * S::OUT + c);
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
    if ((N > 1 || g.len > 1) && __syncthreads_or(bad))                        // (a single token sees every key of its list; what is infinite is no number in parts)
        for (int r = wave; r < rows; r += WAVES) {
            const int t = r / group;
            exact_row<PREC>(a, g, keys, kv, kv * group + r - t * group, t, t0 * S::KEYS, min(t1 * S::KEYS, keys.n), part, split);
        }
}

// -- many rows --

// A workgroup takes 128 query rows of one segment and key/value head and walks over their keys, 64 at a time; a wave has 32 of the rows.  Codes of a round
// go through registers into LDS as bfloat16, the next round's being asked for while this one's are worked on.  Bound by the matrix instructions and what feeds them: 2
// streams of 8192 tokens on windows of 4096, 32 heads of 128 on 8, in bfloat16 1069 us, 1030 TFLOP/s, 69 % of what a large product reaches (1495); the exponentials
// and the weights' way to bfloat16 are the rest.
// In LDS a block's four pieces of eight values change places, x to x ^ turn: eight lanes that write a piece each, of blocks that follow each other, then write to banks of
// their own (written in order two or four of them met in one; 1113 us where this takes 1069).
template <int DP> struct TileShape {
    static constexpr int KEYS = 64, BLOCKS = DP / kBits;
    static constexpr int K_STRIDE = DP + 8;                                   // neighbouring rows begin 16 bytes apart in the banks
    static constexpr int V_STRIDE = DP + 32;                                  // four rows by 64 bytes are read together: rows begin 16 banks apart
    static constexpr int PIECES = KEYS * BLOCKS;                              // of keys, and as many of values
    static constexpr int LOADS = 2 * PIECES / 256;
    static constexpr int LDS_BYTES = KEYS * (K_STRIDE + V_STRIDE) * 2;
    static __device__ __forceinline__ int k_turn(int block) { return DP == 64 ? 0 : DP == 128 ? block & 2 : block >> 1 & 3; }
    static __device__ __forceinline__ int v_turn(int row, int block) { return DP == 64 ? row & 3 : DP == 128 ? (row & 1) | (block & 2) : block >> 1 & 3; }
};
// read_column of the values over 32 lanes, of a block's columns.
template <int DP> __device__ __forceinline__ bf16x8 read_block(const __bf16 *lds, int block, int r0, int r1)
{
    using S = TileShape<DP>;
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const int lane = threadIdx.x & 31, r = lane >> 2 & 3, at = r * S::V_STRIDE + block * kBits + (((lane >> 3 & 2) | (lane >> 1 & 1)) ^ S::v_turn(r, block)) * 8 + (lane & 1) * 4;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r0 * S::V_STRIDE + at));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r1 * S::V_STRIDE + at));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int PREC, int DP>
__global__ void __launch_bounds__(256, PREC != IDF_PREC_BF16 || DP > 128 ? 1 : DP > 64 ? 2 : 4) k_nibble_tile(idf_nibble_attend_args a, int splits)
{
    using M = Mfma<IDF_PREC_BF16>;
    using T = typename Elem<PREC>::type;
    using S = TileShape<DP>;
    constexpr int KT = S::KEYS / 32, KS = DP / 16, DT = DP / 32, N = Parts<PREC>::N;
    extern __shared__ __align__(16) unsigned char raw[];
    __bf16 *k_lds = (__bf16 *)raw, *v_lds = k_lds + S::KEYS * S::K_STRIDE;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
    const int group = a.heads_q / a.heads_kv;
    const int kv = blockIdx.x % a.heads_kv, seg = blockIdx.x / a.heads_kv;
    const int split = blockIdx.z, tile = gridDim.y - 1 - blockIdx.y;          // long lists first
    const Segment g = segment_of(a, seg, a.starts);
    const int64_t rows = (int64_t)g.len * group, row0 = (int64_t)tile * kTileRows;
    if (row0 >= rows) return;
    const int64_t row_last = min(row0 + kTileRows, rows) - 1;
    const Keys keys(a, g.start + row0 / group, g.start + row_last / group);
    const Held4<const uint8_t> kh(a.ring.k_codes, a.ring.k_scales, a.slots, a.heads_kv, a.head_dim, g.ring, kv), vh(a.ring.v_codes, a.ring.v_scales, a.slots, a.heads_kv, a.head_dim, g.ring, kv);
    const Partial part = partial_of(a, splits);
    const uint32_t row_codes = a.head_dim / 2, row_scales = a.head_dim / kBits;
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

    bf16x8 q[KS][N];
    {
        const T *src = (const T *)a.q.base + token * a.q.token_stride + my_h * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < KS; ++s) load_query<PREC>(src + 16 * s + 8 * half, a.head_dim - 16 * s - 8 * half, q[s]);
    }
    i32x4 codes[S::LOADS];
    uint32_t powers[S::LOADS];
    auto load = [&](int t) IDF_INLINE {
        const int i0 = t * S::KEYS;
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int x = j * 256 + threadIdx.x;
            const bool key = x < S::PIECES;
            const int piece = key ? x : x - S::PIECES, r = piece / S::BLOCKS, b = piece - r * S::BLOCKS;
            const bool there = i0 + r < keys.n && b * kBits < a.head_dim;
            const uint32_t slot = keys.slot(min(i0 + r, keys.n - 1));
            codes[j] = i32x4{0, 0, 0, 0};
            powers[j] = 127u;
            if (there) {
                codes[j] = *(const i32x4 *)((key ? kh.codes : vh.codes) + (slot * row_codes + b * 16));
                powers[j] = (key ? kh.scales : vh.scales)[slot * row_scales + b];
            }
        }
    };
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = -__FLT_MAX__, l = 0.f;
    if (t0 < t1) load(t0);
    for (int t = t0; t < t1; ++t) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < S::LOADS; ++j) {
            const int x = j * 256 + threadIdx.x;
            const bool key = x < S::PIECES;
            const int piece = key ? x : x - S::PIECES, r = piece / S::BLOCKS, b = piece - r * S::BLOCKS;
            __bf16 *to = (key ? k_lds + r * S::K_STRIDE : v_lds + r * S::V_STRIDE) + b * kBits;
            const float power = power_of(powers[j]);
            const int turn = key ? S::k_turn(b) : S::v_turn(r, b);
#pragma unroll
            for (int w = 0; w < 4; ++w) *(bf16x8 *)(to + 8 * (w ^ turn)) = values8((uint32_t)codes[j][w], power);
        }
        __syncthreads();
        if (t + 1 < t1) load(t + 1);

        // a wave in its products goes first: those of another on the same SIMD, in its softmax, fill what it leaves
        __builtin_amdgcn_s_setprio(1);
        f32x16 st[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
            for (int e = 0; e < 16; ++e) st[kt][e] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 k = M::load(k_lds + (32 * kt + col) * S::K_STRIDE + s / 2 * kBits + (((2 * s & 2) | half) ^ S::k_turn(s / 2)) * 8);
#pragma unroll
                for (int x = N - 1; x >= 0; --x) st[kt] = M::mma32(k, q[s][x], st[kt]);
            }
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
            bf16x8 pf[N];
            in_parts(w, pf);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const bf16x8 v = read_block<DP>(v_lds, d, 16 * s + 4 * half, 16 * s + 8 + 4 * half);
#pragma unroll
                for (int x = N - 1; x >= 0; --x) o[d] = M::mma32(v, pf[x], o[d]);
            }
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
}

// ---- host ----

// How a call of the attention is cut: which kernel, and into how many parts the keys go.
struct Plan {
    bool step;
    int64_t rows;              // of the longest segment and a key/value head
    int tiles, splits, waves;
};
bool eight_waves(const idf_nibble_attend_args &a, int64_t groups) { return groups <= 256 && a.head_dim <= 128; }
// Into how many parts a list of keys goes: the number with the least estimated time, as in the window's attention.  Eight waves take a round of 128 keys in half the time of
// four (us, without that and with it: a token of 24 streams on 4096 keys 31.1, 28.8, in float32 42.2, 37.5; 4 of 2 streams on 30,000 22.9, 20.7; one on 16,384 13.6, 12.5).
int splits_of(const idf_nibble_attend_args &a, bool step, int64_t pairs, int64_t keys)
{
    const int64_t round = step ? 128 : 64, rounds = (keys + round - 1) / round, held = 512;
    const double rows = (double)std::min<int64_t>(a.n_tokens, a.n_segments * longest(a)) * a.heads_q;
    int best = 1;
    double least = 0.0;
    for (int64_t per = rounds; per >= 1; per = per > 32 ? per * 7 / 8 : per - 1) {
        const int64_t n = (rounds + per - 1) / per;
        if (n > 1 && (n > kMostSplits || pairs * n > held)) break;
        const double each = !step ? 1.0 + 0.006 * a.head_dim : eight_waves(a, pairs * n) ? 0.65 : 1.25;
        const double us = per * each + (n > 1 ? (step ? 4.2 : 5.0) + rows * (1.6e-3 + 1e-6 * n * a.head_dim) : 0.0);
        if (n == 1 || us < least) { least = us; best = (int)n; }
    }
    return best;
}

Plan plan_of(const idf_nibble_attend_args &a)
{
    Plan p;
    p.rows = longest(a) * (a.heads_q / a.heads_kv);
    p.step = p.rows <= (a.precision == IDF_PREC_F32 && a.head_dim > 128 ? kStepRows / 2 : kStepRows);
    p.tiles = p.step ? 1 : (int)((p.rows + kTileRows - 1) / kTileRows);
    const int64_t pairs = (int64_t)a.n_segments * a.heads_kv * p.tiles;
    const int64_t own = p.step ? longest(a) : std::min<int64_t>(longest(a), kTileRows / (a.heads_q / a.heads_kv) + 1);
    p.splits = splits_of(a, p.step, pairs, std::min<int64_t>(a.window + own, a.slots) + a.sinks);
    p.waves = eight_waves(a, pairs * p.splits) ? 8 : 4;
    return p;
}

template <int PREC, int DP, int RT, int WAVES>
hipError_t step(const idf_nibble_attend_args &a, const Plan &p, const LaunchCtx &lc)
{
    constexpr int bytes = WAVES * StepShape<PREC, DP, RT, WAVES>::WAVE_FLOATS * (int)sizeof(float);
    if (bytes > 60000)
        if (const hipError_t e = allow_lds<bytes>(Kernel<k_nibble_step<PREC, DP, RT, WAVES>>{})) return e;
    return launch(k_nibble_step<PREC, DP, RT, WAVES>, dim3(p.splits, a.heads_kv, a.n_segments), dim3(64 * WAVES), bytes, lc, a, p.splits);
}

template <int PREC, int DP>
hipError_t attend(const idf_nibble_attend_args &a, const Plan &p, const LaunchCtx &lc)
{
    if (p.step) {
        // (what eight waves, or 32 rows, leave of the registers has to hold a round)
        if constexpr (DP <= 128)
            if (p.waves == 8) return p.rows <= 16 ? step<PREC, DP, 1, 8>(a, p, lc) : step<PREC, DP, 2, 8>(a, p, lc);
        if constexpr (DP <= 128 || PREC == IDF_PREC_BF16)
            if (p.rows > 16) return step<PREC, DP, 2, 4>(a, p, lc);
        return step<PREC, DP, 1, 4>(a, p, lc);
    }
    constexpr int bytes = TileShape<DP>::LDS_BYTES;
    if (bytes > 65536)
        if (const hipError_t e = allow_lds<bytes>(Kernel<k_nibble_tile<PREC, DP>>{})) return e;
    return launch(k_nibble_tile<PREC, DP>, dim3(a.n_segments * a.heads_kv, p.tiles, p.splits), dim3(256), bytes, lc, a, p.splits);
}

template <int PREC>
hipError_t by_dim(const idf_nibble_attend_args &a, const LaunchCtx &lc)
{
    const Plan p = plan_of(a);
    const hipError_t e = a.head_dim <= 64 ? attend<PREC, 64>(a, p, lc) : a.head_dim <= 128 ? attend<PREC, 128>(a, p, lc) : attend<PREC, 256>(a, p, lc);
    return e == hipSuccess && p.splits > 1 ? join_splits<PREC>(a, p.splits, lc) : e;
}

template <int PREC>
hipError_t append(const idf_nibble_append_args &a, const LaunchCtx &lc)
{
    const int eb = PREC == IDF_PREC_F32 ? 4 : 2;
    bool aligned = true;
    for (const idf_tokens *t : {&a.k, &a.v}) aligned = aligned && (uintptr_t)t->base % (8 * eb) == 0 && t->token_stride % 8 == 0 && t->head_stride % 8 == 0;
    int lanes_log2 = 2;
    while (8 << lanes_log2 < a.head_dim) ++lanes_log2;
    // workgroups for every compute unit first, then as many tokens as share a barrier
    const int64_t n = longest(a);
    const int per = (int)std::max<int64_t>(1, std::min<int64_t>({std::min<int64_t>(a.n_tokens, n * a.n_segments) / 1024, kMostTokens, n}));
    const dim3 grid((unsigned)((n + per - 1) / per), a.n_segments);
    const size_t lds = (size_t)per * (a.rotary_dim / 2) * sizeof(double2);
    return aligned ? launch(k_nibble_append<PREC, true>, grid, dim3(256), lds, lc, a, lanes_log2, per) : launch(k_nibble_append<PREC, false>, grid, dim3(256), lds, lc, a, lanes_log2, per);
}

}  // namespace

hipError_t launch_nibble_append(const idf_nibble_append_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? append<IDF_PREC_F32>(a, lc) : append<IDF_PREC_BF16>(a, lc);
}

hipError_t launch_nibble_values(const idf_nibble_values_args &a, const LaunchCtx &lc)
{
    const int rows = 256 / (a.head_dim / 8);
    const int64_t heads = (int64_t)a.n_streams * a.heads_kv;
    // (a launch's second axis: more heads go in several launches)
    for (int64_t first = 0; first < heads; first += 65536 / a.heads_kv * a.heads_kv - a.heads_kv) {
        idf_nibble_values_args part = a;
        const int64_t n = std::min<int64_t>(heads - first, 65536 / a.heads_kv * a.heads_kv - a.heads_kv), row = first * a.slots;
        const int eb = a.precision == IDF_PREC_F32 ? 4 : 2;
        part.ring = {a.ring.k_codes + row * (a.head_dim / 2), a.ring.k_scales + row * (a.head_dim / kBits), a.ring.v_codes + row * (a.head_dim / 2), a.ring.v_scales + row * (a.head_dim / kBits)};
        part.k = (char *)a.k + row * a.head_dim * eb;
        part.v = (char *)a.v + row * a.head_dim * eb;
        const dim3 grid((unsigned)std::min<int64_t>((a.slots + rows * 4 - 1) / (rows * 4), std::max<int64_t>(1, 8192 / n)), (unsigned)n, 2);
        const hipError_t e = a.precision == IDF_PREC_F32 ? launch(k_nibble_values<IDF_PREC_F32>, grid, dim3(256), 0, lc, part) : launch(k_nibble_values<IDF_PREC_BF16>, grid, dim3(256), 0, lc, part);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

size_t nibble_attend_workspace(const idf_nibble_attend_args &a) { return split_workspace(a, plan_of(a).splits); }

hipError_t launch_nibble_attend(const idf_nibble_attend_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? by_dim<IDF_PREC_F32>(a, lc) : by_dim<IDF_PREC_BF16>(a, lc);
}

}  // namespace idf
