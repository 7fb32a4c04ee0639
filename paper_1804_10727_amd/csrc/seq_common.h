// What the kernels that mix the tokens of streams share: loads and roundings of the two precisions, the segment that a workgroup
// works on, and the rows of the cache that a query sees.
#pragma once

#include "idf_kernels.h"
#include "mfma_tile.h"

namespace idf {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

// Elements as they lie in memory: VL of them in 16 bytes.
template <int PREC> struct Elem;
template <> struct Elem<IDF_PREC_F32> {
    using type = float;
    static constexpr int VL = 4;
    static __device__ __forceinline__ float to_f32(float v) { return v; }
    static __device__ __forceinline__ float from_f32(float v) { return v; }
};
template <> struct Elem<IDF_PREC_BF16> {
    using type = __bf16;
    static constexpr int VL = 8;
    static __device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }
    static __device__ __forceinline__ __bf16 from_f32(float v) { return (__bf16)v; }          // to nearest, ties to even
};

template <class T, int N> struct alignas(N * sizeof(T)) Pack { T v[N]; };

// A segment of packed tokens as a workgroup sees it.  Nothing that the device alone can see is trusted: whatever offsets, starts
// and ids hold, [begin, begin + len) lies in the tokens and ring among the streams.
struct Segment {
    int64_t begin;             // its first token
    int64_t start;             // position of that token in the stream
    int len;
    int ring;                  // its stream; a segment whose stream is none has no tokens
    bool valid;
};

template <class Args>
__device__ __forceinline__ Segment segment_of(const Args &a, int s, const int64_t *starts)
{
    Segment g;
    if (a.offsets) {
        const int64_t b = min(max(a.offsets[s], (int64_t)0), a.n_tokens), e = min(max(a.offsets[s + 1], b), a.n_tokens);
        g.begin = b;
        g.len = (int)min(e - b, a.max_tokens);
    } else {
        g.begin = (int64_t)s * a.max_tokens;
        g.len = (int)a.max_tokens;
    }
    g.start = starts ? starts[s] : 0;
    g.ring = a.stream_ids ? a.stream_ids[s] : s;
    g.valid = g.ring >= 0 && g.ring < a.n_streams && g.start >= 0 && g.start <= (int64_t)1 << 62;
    if (!g.valid) { g.len = 0; g.start = 0; g.ring = 0; }
    return g;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

}  // namespace

}  // namespace idf
