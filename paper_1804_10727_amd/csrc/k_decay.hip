// Linear attention with a decay per head (idf_decay_attend).
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

// The recurrence itself, token by token.  A wave owns 32 columns of the state of one key/value head: eight lanes side by side hold four
// columns each, eight lanes below each other ROWS rows each, so that a token costs two multiply-adds per value of the state and a sum
// over eight lanes per query; nothing is shared between waves.
template <int PREC, int ROWS>
__global__ void __launch_bounds__(256) k_decay_tokens(idf_decay_args a, int column_groups)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int kv = wave / column_groups, c0 = (wave - kv * column_groups) * 32 + (lane & 7) * 4, r0 = (lane >> 3) * ROWS;
    if (kv >= a.heads_kv) return;
    const Segment g = segment_of(a, blockIdx.y, nullptr);
    if (!g.valid) return;
    const int queries = a.heads_q / a.heads_kv;
    const float lambda = expf(a.log_decay[kv]);
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
            for (int e = 0; e < 4; ++e) s[r][e] = __builtin_fmaf(kr, vv[e], lambda * s[r][e]);
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

template <int PREC>
hipError_t tokens(const idf_decay_args &a, const LaunchCtx &lc)
{
    const int column_groups = (a.dim_v + 31) / 32;
    const dim3 grid((unsigned)(((int64_t)a.heads_kv * column_groups + 3) / 4), a.n_segments);
    if (a.dim_k <= 64) return launch(k_decay_tokens<PREC, 8>, grid, dim3(256), 0, lc, a, column_groups);
    if (a.dim_k <= 128) return launch(k_decay_tokens<PREC, 16>, grid, dim3(256), 0, lc, a, column_groups);
    return launch(k_decay_tokens<PREC, 32>, grid, dim3(256), 0, lc, a, column_groups);
}

}  // namespace

size_t decay_workspace(const idf_decay_args &) { return 0; }

hipError_t launch_decay(const idf_decay_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? tokens<IDF_PREC_F32>(a, lc) : tokens<IDF_PREC_BF16>(a, lc);
}

}  // namespace idf
