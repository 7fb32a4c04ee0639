// Attention over a sliding window and first tokens, with the ring that caches keys and values (idf_window_attend).
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Where the key or value of a position lies: with the segment's own tokens, or in the ring.
template <class T>
__device__ __forceinline__ const T *held_row(const idf_window_args &a, const Segment &g, int64_t pos, const idf_tokens &own, const void *ring, int kv)
{
    if (pos >= g.start) return (const T *)own.base + (g.begin + (pos - g.start)) * own.token_stride + kv * own.head_stride;
    const int64_t slot = pos < a.sinks ? pos : a.sinks + (pos - a.sinks) % (a.slots - a.sinks);
    return (const T *)ring + ((g.ring * a.slots + slot) * a.heads_kv + kv) * a.head_dim;
}

// One query row by one wave, key by key: scores of 64 keys at a time, a lane each, then the sum with a lane for every 64th value.  Only
// keys that the query sees are read, so that whatever lies in the others cannot reach it.
template <int PREC>
__global__ void __launch_bounds__(64) k_window_rows(idf_window_args a)
{
    using E = Elem<PREC>;
    using T = typename E::type;
    const int lane = threadIdx.x, h = blockIdx.y, kv = h / (a.heads_q / a.heads_kv);
    const Segment g = segment_of(a, blockIdx.z, a.starts);
    for (int t = blockIdx.x; t < g.len; t += gridDim.x) {
        const int64_t p = g.start + t, floor = a.k_ring ? 0 : g.start;               // (without a ring nothing is held from before the segment)
        const int64_t first = min((int64_t)a.sinks, p + 1), low = max(max(first, p - a.window + 1), floor), skip = min(first, floor);
        const int64_t n_first = first - skip, n = n_first + max(p - low + 1, (int64_t)0);
        const T *q = (const T *)a.q.base + (g.begin + t) * a.q.token_stride + h * a.q.head_stride;
        float m = -__FLT_MAX__, l = 0.f, o[4] = {};
        for (int64_t i0 = 0; i0 < n; i0 += 64) {
            const int64_t i = min(i0 + lane, n - 1), pos = i < n_first ? skip + i : low + i - n_first;
            const T *k = held_row<T>(a, g, pos, a.k, a.k_ring, kv);
            float s = 0.f;
            for (int d = 0; d < a.head_dim; ++d) s += E::to_f32(q[d]) * E::to_f32(k[d]);
            s = i0 + lane < n ? s * (a.scale * kLog2e) : -__builtin_inff();
            const float m2 = fmaxf(m, wave_max(s)), w = exp2f(s - m2), fade = exp2f(m - m2);
            m = m2;
            l = l * fade + wave_sum(w);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] *= fade;
            for (int j = 0; j < 64 && i0 + j < n; ++j) {
                const int64_t i = i0 + j, pos = i < n_first ? skip + i : low + i - n_first;
                const T *v = held_row<T>(a, g, pos, a.v, a.v_ring, kv);
                const float wj = __shfl(w, j);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (lane + 64 * c < a.head_dim) o[c] += wj * E::to_f32(v[lane + 64 * c]);
            }
        }
        T *out = (T *)a.out.base + (g.begin + t) * a.out.token_stride + h * a.out.head_stride;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < a.head_dim) out[lane + 64 * c] = E::from_f32(o[c] / l);
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

}  // namespace

size_t window_workspace(const idf_window_args &) { return 0; }

hipError_t launch_window(const idf_window_args &a, const LaunchCtx &lc)
{
    const dim3 grid((unsigned)std::min<int64_t>(a.max_tokens, 16384), a.heads_q, a.n_segments);
    hipError_t e = a.precision == IDF_PREC_F32 ? launch(k_window_rows<IDF_PREC_F32>, grid, dim3(64), 0, lc, a)
                                               : launch(k_window_rows<IDF_PREC_BF16>, grid, dim3(64), 0, lc, a);
    if (e == hipSuccess && a.k_ring) {
        const int elem16 = a.precision == IDF_PREC_F32 ? 4 : 8, row16 = a.heads_kv * a.head_dim / elem16;
        const dim3 g((unsigned)std::min<int64_t>((a.max_tokens * row16 + 255) / 256, 4096), a.n_segments);
        e = launch(k_window_append, g, dim3(256), 0, lc, a, row16, elem16);
    }
    return e;
}

}  // namespace idf
