// Attention whose lists of keys are cut into parts: partial results in the workspace, and the launch that joins them.
#pragma once

#include <algorithm>

#include "seq_mfma.h"

namespace idf {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMostSplits = 128;                   // parts of a list of keys: a wave joins them, a lane has two

// Partial results of rows whose keys are split over workgroups: [split][token][head][head_dim] sums, then [split][token][head] maximum (of
// scores in units of log 2) and sum of weights.
struct Partial {
    float *o, *ml;
    int splits;
};
template <class Args> __device__ __host__ __forceinline__ Partial partial_of(const Args &a, int splits)
{
    Partial p;
    p.splits = splits;
    p.o = (float *)a.workspace;
    p.ml = p.o + (int64_t)splits * a.n_tokens * a.heads_q * a.head_dim;
    return p;
}

template <class Args> size_t split_workspace(const Args &a, int splits)
{
    return splits > 1 ? (size_t)splits * a.n_tokens * a.heads_q * (a.head_dim + 2) * sizeof(float) : 0;
}

// Splits joined.  A workgroup takes a row, each of its waves every fourth split: its lanes first the maximum and sum of a split each, whose
// shares then go from lane to lane while a lane adds up four values of the row, with splits side by side where the row leaves lanes.  All of
// a wave's reads are on their way together: one after the other, each would wait for memory.
template <int PREC, class Args>
__global__ void __launch_bounds__(256) k_window_join(Args a, int splits, int lanes_log2)
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

template <int PREC, class Args> hipError_t join_splits(const Args &a, int splits, const LaunchCtx &lc)
{
    int lanes_log2 = 0;
    while (4 << lanes_log2 < a.head_dim) ++lanes_log2;
    return launch(k_window_join<PREC, Args>, dim3((unsigned)std::min<int64_t>(longest(a) * a.heads_q, 8192), a.n_segments), dim3(256), 0, lc, a, splits, lanes_log2);
}

}  // namespace

}  // namespace idf
