// Matrix-core pieces of the kernels that mix tokens.  A fragment is eight values of a lane along the summed axis; the two precisions
// share every layout: one bfloat16 instruction takes a whole fragment, eight float32 instructions take one value of it each (which values
// meet in one instruction does not matter as long as both operands agree).
#pragma once

#include "seq_common.h"

namespace idf {

namespace {

typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

template <int PREC> struct Mfma;
template <> struct Mfma<IDF_PREC_BF16> {
    using T = __bf16;
    using frag = bf16x8;
    static constexpr int VL = 8;
    static __device__ __forceinline__ frag zero() { return __builtin_bit_cast(frag, i32x4{0, 0, 0, 0}); }
    static __device__ __forceinline__ frag load(const T *p) { return *(const frag *)p; }
    // of a row that has n values from p on (n a multiple of VL; zeros behind them, nothing read there)
    static __device__ __forceinline__ frag load(const T *p, int n) { return n > 0 ? load(p) : zero(); }
    // D[16][16] += A[16][32] B[32][16]: a lane holds row (A) or column (B) lane % 16 and, of the summed axis, 8 (lane / 16) + 0 .. 7; of D column
    // lane % 16, rows 4 (lane / 16) + 0 .. 3
    static __device__ __forceinline__ f32x4 mma16(const frag &a, const frag &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    // D[32][32] += A[32][16] B[16][32]: row or column lane % 32, summed axis 8 (lane / 32) + 0 .. 7; of D column lane % 32, register i is row 8 (i / 4) + 4 (lane / 32) + i % 4
    static __device__ __forceinline__ f32x16 mma32(const frag &a, const frag &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ frag pack(const float *v)
    {
        frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (__bf16)v[i];
        return f;
    }
};
template <> struct Mfma<IDF_PREC_F32> {
    using T = float;
    using frag = f32x8;
    static constexpr int VL = 4;
    static __device__ __forceinline__ frag zero() { return frag{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
    static __device__ __forceinline__ frag load(const T *p)
    {
        const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ frag load(const T *p, int n)
    {
        f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
        if (n > 0) a = *(const f32x4 *)p;
        if (n > 4) b = *(const f32x4 *)(p + 4);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ f32x4 mma16(const frag &a, const frag &b, f32x4 c)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ f32x16 mma32(const frag &a, const frag &b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ frag pack(const float *v)
    {
        frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i];
        return f;
    }
};

// Values [row][column] in LDS, read along the rows: eight values of one column, rows r0 .. r0 + 3 and r1 .. r1 + 3.  The lanes of a group of
// 16 ask for columns c .. c + 15 and the same rows.  bfloat16: the transposing read, in which lane 4 r + x of a group points at row r, columns
// 4 x .. 4 x + 3 of the four rows by sixteen columns that the group gets.  stride in elements, a multiple of four.
__device__ __forceinline__ bf16x8 read_column(const __bf16 *lds, int stride, int c, int r0, int r1)
{
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const int lane = threadIdx.x & 15, at = (lane >> 2) * stride + c + (lane & 3) * 4;
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r0 * stride + at));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r1 * stride + at));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ f32x8 read_column(const float *lds, int stride, int c, int r0, int r1)
{
    const float *at = lds + c + (threadIdx.x & 15);
    f32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = at[(r0 + i) * stride]; f[4 + i] = at[(r1 + i) * stride]; }
    return f;
}

// The same with columns c + 4 .. c + 7 and c + 8 .. c + 11 of each 16 in each other's place: as rows of a 32 x 32 product they put eight
// columns in order into a lane's registers.
__device__ __forceinline__ bf16x8 read_rows_swapped(const __bf16 *lds, int stride, int c, int r0, int r1)
{
    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
    const int lane = threadIdx.x & 15, x = lane & 3, at = (lane >> 2) * stride + c + ((x & 1) << 3 | (x & 2) << 1);
    const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r0 * stride + at));
    const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + r1 * stride + at));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ f32x8 read_rows_swapped(const float *lds, int stride, int c, int r0, int r1)
{
    const int lane = threadIdx.x & 15, x = lane >> 2;
    const float *at = lds + c + ((x & 1) << 3 | (x & 2) << 1 | (lane & 3));
    f32x8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = at[(r0 + i) * stride]; f[4 + i] = at[(r1 + i) * stride]; }
    return f;
}

}  // namespace

}  // namespace idf
