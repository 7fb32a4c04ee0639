// Rows times 8-bit weights (idf_quantize_rows, idf_project_rows).
//
//   out[r][n] = s_r t_n sum_c x[r][c] w[n][c] + bias[n],  sums of 8-bit codes in 32-bit integers: exact, whatever their order, so that every way
// of cutting a call gives the same bits.
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

typedef __attribute__((ext_vector_type(2))) int i32x2;

inline __host__ __device__ int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// ---- rows to codes ----

// The whole number nearest to 127 x / most, the even one halfway.  The quotient is formed in 64 bits; where it comes within 2^-30 of a middle, products that
// are exact in 64 bits decide (24 + 7 bits on one side, 24 + 8 on the other).
__device__ __forceinline__ int code_of(float x, double per, float most)
{
    const double q = (double)x * per, whole = __builtin_rint(q), off = q - whole;
    int c = (int)whole;
    if (__builtin_fabs(__builtin_fabs(off) - 0.5) < 0x1p-30) {
        const double low = __builtin_floor(q);     // (the middle is low + 0.5)
        const double far = 127.0 * (double)x - (low + 0.5) * (double)most;
        c = (int)low + (far > 0.0 || (far == 0.0 && ((int)low & 1)));
    }
    return c;
}

// A row by THREADS threads, which keep as many of its values as their registers hold, and read the others a second time.
template <int PREC, int THREADS>
__global__ void __launch_bounds__(256) k_quantize_rows(idf_quantize_args a, bool aligned)
{
    using T = typename Elem<PREC>::type;
    constexpr int kKeep = 4, N = 8;                // pieces of eight values
    using P = Pack<T, N>;
    __shared__ float top[256 / 64];
    const int lane = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS;
    const bool there = row < a.n_rows;
    const T *src = (const T *)a.x.base + (there ? row : a.n_rows - 1) * a.x.row_stride;
    auto load = [&](int c) IDF_INLINE {
        P p;
        if (aligned && c + N <= a.cols) return *(const P *)(src + c);
#pragma unroll
        for (int i = 0; i < N; ++i) p.v[i] = c + i < a.cols ? src[c + i] : Elem<PREC>::from_f32(0.f);
        return p;
    };
    P kept[kKeep];
    float most = 0.f;
    bool fine = true;
    auto look = [&](const P &p) IDF_INLINE {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float v = __builtin_fabsf(Elem<PREC>::to_f32(p.v[i]));
            fine = fine && v < __builtin_inff();
            most = fmaxf(most, v);
        }
    };
#pragma unroll
    for (int k = 0; k < kKeep; ++k) {
        const int c = (k * THREADS + lane) * N;
        kept[k] = P{};
        if (c < a.cols) kept[k] = load(c);
    }
#pragma unroll
    for (int k = 0; k < kKeep; ++k) look(kept[k]);
    for (int c = (kKeep * THREADS + lane) * N; c < a.cols; c += THREADS * N) look(load(c));
    if (!fine) most = __builtin_inff();
    most = wave_max(most);
    if (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = most;
        __syncthreads();
        most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    }
    if (!there) return;
    fine = most < __builtin_inff();
    const double per = most > 0.f && fine ? 127.0 / (double)most : 0.0;
    int8_t *to = a.codes + row * up16(a.cols);
    auto store = [&](int c, const P &p) IDF_INLINE {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < N; ++i) w[i / 4] |= (uint32_t)(per > 0.0 ? code_of(Elem<PREC>::to_f32(p.v[i]), per, most) & 255 : 0) << 8 * (i % 4);
        *(i32x2 *)(to + c) = i32x2{(int)w[0], (int)w[1]};
    };
    const int padded = (int)up16(a.cols);
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
        if (const int c = (k * THREADS + lane) * N; c < padded) store(c, kept[k]);
    for (int c = (kKeep * THREADS + lane) * N; c < padded; c += THREADS * N) store(c, c < a.cols ? load(c) : P{});
    if (lane == 0) a.scales[row] = fine ? most / 127.f : __builtin_nanf("");
}

// ---- the product ----

// What a kernel of the product takes: codes with rows of ld bytes, a multiple of 16.
struct Product {
    const int8_t *x, *w;
    int64_t x_ld, n_rows;
    int w_ld, n_out;                               // (rows of weights lie behind each other)
    const float *x_scales, *w_scales, *bias;
    void *out;
    int64_t out_stride;
};

template <class T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __bf16 rounded<__bf16>(float v) { return (__bf16)v; }

__device__ __attribute__((aligned(16))) const int8_t kZeros[16] = {};

// A workgroup takes BM rows of x by BN outputs, a wave 16 MT by 16 NT of them; codes go from memory into LDS directly, 128 of a row at a time, the
// next ones while these are multiplied.  A row's eight pieces of 16 bytes lie in LDS at place piece ^ (row & 7): what a matrix instruction's lanes read together,
// 16 rows by four neighbouring pieces, lies in banks of its own.
template <class Out, int WM, int WN, int MT, int NT>
__global__ void __launch_bounds__(64 * WM * WN) k_project_tile(Product a)
{
    constexpr int BM = WM * MT * 16, BN = WN * NT * 16, WAVES = WM * WN, KEYS = (BM + BN) * 128;
    constexpr int LOADS = (BM + BN) / 8 / WAVES;   // of eight rows each
    static_assert((BM + BN) / 8 % WAVES == 0 && BM / 8 % WAVES == 0, "a wave's loads are of one matrix each");
    extern __shared__ __align__(16) int8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles_n = (a.n_out + BN - 1) / BN;
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * BM;
    const int n0 = (int)(blockIdx.x % tiles_n) * BN;
    // lane's row among eight and the piece of 16 bytes that lies at its place
    const int lrow = lane >> 3, piece = (lane & 7) ^ lrow;
    const int8_t *src[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int row = (j * WAVES + wave) * 8 + lrow;
        src[j] = j * WAVES * 8 < BM ? a.x + min(m0 + row, a.n_rows - 1) * a.x_ld : a.w + (int64_t)min(n0 + row - BM, a.n_out - 1) * a.w_ld;
    }
    auto load = [&](int k0, int buffer) IDF_INLINE {
        const bool there = k0 + piece * 16 < a.w_ld;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int8_t *from = there ? src[j] + k0 + piece * 16 : kZeros;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(lds + buffer * KEYS + (j * WAVES + wave) * 1024), 16, 0, 0);
        }
    };
    i32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int wm = wave / WN, wn = wave % WN, col = lane & 15, grp = lane >> 4;
    load(0, 0);
    int buffer = 0;
    for (int k0 = 0; k0 < a.w_ld; k0 += 128, buffer ^= 1) {
        __syncthreads();                           // (waits for the loads, too)
        if (k0 + 128 < a.w_ld) load(k0 + 128, buffer ^ 1);
        const int8_t *xs = lds + buffer * KEYS + (wm * MT * 16 + col) * 128, *ws = lds + buffer * KEYS + (BM + wn * NT * 16 + col) * 128;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = ((s * 4 + grp) ^ (col & 7)) * 16;
            i32x4 x[MT], w[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) x[i] = *(const i32x4 *)(xs + i * 16 * 128 + at);
#pragma unroll
            for (int j = 0; j < NT; ++j) w[j] = *(const i32x4 *)(ws + j * 16 * 128 + at);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[i], acc[i][j], 0, 0, 0);
        }
    }
    // a lane has one row of x and four neighbouring outputs
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t r = m0 + (wm * MT + i) * 16 + col;
        if (r >= a.n_rows) continue;
        const float sx = a.x_scales[r];
        Out *out = (Out *)a.out + r * a.out_stride;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = n0 + (wn * NT + j) * 16 + grp * 4 + e;
                if (n < a.n_out) out[n] = rounded<Out>((float)acc[i][j][e] * a.w_scales[n] * sx + (a.bias ? a.bias[n] : 0.f));
            }
    }
}

template <class Out>
hipError_t product(const Product &p, const LaunchCtx &lc)
{
    constexpr int BM = 128, BN = 128;
    return launch(k_project_tile<Out, 2, 2, 4, 4>, dim3((unsigned)((p.n_rows + BM - 1) / BM * ((p.n_out + BN - 1) / BN))), dim3(256), 2 * (BM + BN) * 128, lc, p);
}

template <int PREC>
hipError_t quantize(const idf_quantize_args &a, const LaunchCtx &lc)
{
    const int eb = PREC == IDF_PREC_F32 ? 4 : 2;
    const bool aligned = (uintptr_t)a.x.base % (8 * eb) == 0 && a.x.row_stride % 8 == 0;
    if (a.cols <= 2048) return launch(k_quantize_rows<PREC, 64>, dim3((unsigned)((a.n_rows + 3) / 4)), dim3(256), 0, lc, a, aligned);
    return launch(k_quantize_rows<PREC, 256>, dim3((unsigned)a.n_rows), dim3(256), 0, lc, a, aligned);
}

}  // namespace

hipError_t launch_quantize_rows(const idf_quantize_args &a, const LaunchCtx &lc)
{
    return a.precision == IDF_PREC_F32 ? quantize<IDF_PREC_F32>(a, lc) : quantize<IDF_PREC_BF16>(a, lc);
}

// Codes, then scales.
size_t project_workspace(const idf_project_args &a)
{
    return a.precision == IDF_PREC_I8 ? 0 : (size_t)a.n_rows * (size_t)up16(a.cols) + (size_t)a.n_rows * sizeof(float);
}

hipError_t launch_project_rows(const idf_project_args &a, const LaunchCtx &lc)
{
    const int64_t ld = up16(a.cols);
    Product p = {(const int8_t *)a.x.base, a.weights, a.x.row_stride, a.n_rows, (int)ld, a.n_out, a.x_scales, a.weight_scales, a.bias, a.out.base, a.out.row_stride};
    if (a.precision != IDF_PREC_I8) {
        idf_quantize_args q = {a.precision, a.cols, a.n_rows, a.x, (int8_t *)a.workspace, (float *)((int8_t *)a.workspace + a.n_rows * ld)};
        if (const hipError_t e = launch_quantize_rows(q, lc)) return e;
        p.x = q.codes; p.x_ld = ld; p.x_scales = q.scales;
    }
    return a.out_precision == IDF_PREC_F32 ? product<float>(p, lc) : product<__bf16>(p, lc);
}

}  // namespace idf
