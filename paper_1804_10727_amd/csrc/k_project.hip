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

// The whole number nearest to 127 x / most, the even one halfway.  The quotient by 32-bit numbers (off by less than 2^-14) decides unless it comes near a
// middle: there products that are exact in 64 bits do (24 + 7 bits on one side, 24 + 8 on the other).
__device__ __forceinline__ int code_of(float x, float per, float most)
{
    const float q = x * per, whole = __builtin_rintf(q);
    int c = (int)whole;
    if (__builtin_fabsf(__builtin_fabsf(q - whole) - 0.5f) < 0x1p-12f) {
        const double low = __builtin_floorf(q);    // (the middle is low + 0.5)
        const double far = 127.0 * (double)x - (low + 0.5) * (double)most;
        c = (int)low + (far > 0.0 || (far == 0.0 && ((int)low & 1)));
    }
    return c;
}

// A row by THREADS threads, which keep as many of its values as their registers hold, and read the others a second time.  Many rows are bound by memory: 16384 x 4096 from
// bfloat16 in 48 us, 4.2 TB/s, from float32 in 60, 5.6.  Few ones by its latency, 64 x 4096 in 4: a piece is a whole one or single values, which the compiler joins in scratch memory
// (32 or 64 bytes a lane), so that each waits for its own loads before the next one is asked for.
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
        const float *mine = top + threadIdx.x / THREADS * (THREADS / 64);
        most = fmaxf(mine[0], mine[1]);
        if (THREADS == 256) most = fmaxf(most, fmaxf(mine[2], mine[3]));
    }
    if (!there) return;
    fine = most < __builtin_inff();
    // rows of very small values are taken up by a power of two first: a quotient by them is no float32
    const float up = most < 0x1p-100f ? 0x1p120f : 1.f;
    const float top_up = most * up, per = most > 0.f && fine ? 127.f / top_up : 0.f;
    int8_t *to = a.codes + row * up16(a.cols);
    auto store = [&](int c, const P &p) IDF_INLINE {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < N; ++i) w[i / 4] |= (uint32_t)(per > 0.f ? code_of(Elem<PREC>::to_f32(p.v[i]) * up, per, top_up) & 255 : 0) << 8 * (i % 4);
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
    bool fours, whole;                             // rows of out begin at multiples of four values, or of 16 bytes, and have so many
};

template <class T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __bf16 rounded<__bf16>(float v) { return (__bf16)v; }

// Scales and biases of four neighbouring outputs, and those outputs of a row.
struct Four { float scale[4], bias[4]; };
__device__ __forceinline__ Four four_of(const Product &a, int n)
{
    Four f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool there = n + e < a.n_out;
        f.scale[e] = there ? a.w_scales[n + e] : 0.f;
        f.bias[e] = there && a.bias ? a.bias[n + e] : 0.f;
    }
    return f;
}
template <class Out> __device__ __forceinline__ void store_four(const Product &a, int64_t r, int n, float sx, const i32x4 &sum, const Four &f)
{
    Pack<Out, 4> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v.v[e] = rounded<Out>((float)sum[e] * f.scale[e] * sx + f.bias[e]);
    Out *to = (Out *)a.out + r * a.out_stride + n;
    if (a.fours) {
        if (n < a.n_out) *(Pack<Out, 4> *)to = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.n_out) to[e] = v.v[e];
    }
}

// What a row has no more of is read from here.
__device__ const int8_t kZeros[16] __attribute__((aligned(16))) = {};

// A workgroup takes BM rows of x by BN outputs, a wave 16 MT by 16 NT of them; codes go from memory into LDS directly, 128 of a row at a time, those of the next
// STAGES times on their way while these are multiplied.  A row's eight pieces of 16 bytes lie in LDS at place piece ^ (row & 7): what a matrix instruction's
// lanes read together, 16 rows by four neighbouring pieces, lies in banks of its own.  Workgroups of one die (every eighth) take tiles next to each other.
// Results leave by way of LDS, whole lines of a row at a time.  Many rows are bound by the matrix instructions (16384 x 4096 x 6144: 370 us, 2,230 TOP/s, as fast as the library's
// product of 8-bit numbers alone), few ones by the weights (64 x 4096 x 6144: 25 MB in 9.4 us).
template <int N> __device__ __forceinline__ void wait_and_meet()
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
#endif
}

constexpr int BK = 128;

template <class Out, int WM, int WN, int MT, int NT, int STAGES> struct TileShape {
    static constexpr int BM = WM * MT * 16, BN = WN * NT * 16, WAVES = WM * WN, STAGE = (BM + BN) * BK;
    static constexpr int ROWS = 8;                                            // of a wave's load
    static constexpr int LOADS = (BM + BN) / ROWS / WAVES;
    static constexpr int OUT_STRIDE = NT * 16 * (int)sizeof(Out) + 16;        // of a row of results in LDS
    static constexpr int OUT_ROWS = MT * 16 * OUT_STRIDE * WAVES <= STAGES * STAGE ? MT * 16 : 16;      // that a wave has there at a time
    static constexpr int LDS_BYTES = STAGES * STAGE;
    static_assert((BM + BN) / ROWS % WAVES == 0 && BM / ROWS % WAVES == 0, "a wave's loads are of one matrix each");
    static_assert(64 * 16 / (NT * 16 * (int)sizeof(Out)) <= OUT_ROWS, "a wave's store is of its own rows");
    static_assert(OUT_ROWS * OUT_STRIDE * WAVES <= STAGES * STAGE, "results of 16 rows fit");
};

template <class Out, int WM, int WN, int MT, int NT, int STAGES, int PER_CU>
__global__ void __launch_bounds__(64 * WM * WN, PER_CU * WM * WN / 4) k_project_tile(Product a)
{
    using S = TileShape<Out, WM, WN, MT, NT, STAGES>;
    constexpr int BM = S::BM, BN = S::BN, WAVES = S::WAVES, STAGE = S::STAGE, LOADS = S::LOADS, kBand = 8;
    extern __shared__ __align__(16) int8_t lds[];
    __shared__ float x_scale[BM], w_scale[BN], bias[BN];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles_n = (a.n_out + BN - 1) / BN, tiles_m = (int)((a.n_rows + BM - 1) / BM);
    int tm, tn;
    {
        const int whole = gridDim.x / 8, rest = gridDim.x % 8, die = blockIdx.x % 8, at = blockIdx.x / 8;
        const int id = die * whole + min(die, rest) + at;                     // each die's behind each other
        const int band = id / (kBand * tiles_n), m0 = band * kBand, high = min(kBand, tiles_m - m0), in = id - band * kBand * tiles_n;
        tm = m0 + in % high;
        tn = in / high;
    }
    const int64_t m0 = (int64_t)tm * BM;
    const int n0 = tn * BN;
    // a lane's row among those of a load, and the piece of 16 bytes that lies at its place
    const int lrow = lane / 8, piece = (lane % 8) ^ lrow;
    const int8_t *src[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int row = (j * WAVES + wave) * S::ROWS + lrow;
        src[j] = (j * WAVES * S::ROWS < BM ? a.x + min(m0 + row, a.n_rows - 1) * a.x_ld : a.w + (int64_t)min(n0 + row - BM, a.n_out - 1) * a.w_ld) + piece * 16;
    }
    auto load = [&](int k0, int stage) IDF_INLINE {
        int8_t *to = lds + stage * STAGE + wave * 1024;
        if (k0 + BK <= a.w_ld) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src[j] + k0), (__attribute__((address_space(3))) void *)(to + j * WAVES * 1024), 16, 0, 0);
        } else {
            const bool there = k0 + piece * 16 < a.w_ld;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const uintptr_t from = there ? (uintptr_t)(src[j] + k0) : (uintptr_t)kZeros;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)(to + j * WAVES * 1024), 16, 0, 0);
            }
        }
    };
    for (int i = threadIdx.x; i < BM; i += 64 * WAVES) x_scale[i] = a.x_scales[min(m0 + i, a.n_rows - 1)];
    for (int i = threadIdx.x; i < BN; i += 64 * WAVES) {
        const int n = min(n0 + i, a.n_out - 1);
        w_scale[i] = a.w_scales[n];
        bias[i] = a.bias ? a.bias[n] : 0.f;
    }
    i32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int wm = wave / WN, wn = wave % WN, col = lane & 15, grp = lane >> 4;
    const int steps = (a.w_ld + BK - 1) / BK;
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < steps) load(s * BK, s);
    const int8_t *const xs = lds + (wm * MT * 16 + col) * BK, *const ws = lds + (BM + wn * NT * 16 + col) * BK;
    struct Part { i32x4 x[MT], w[NT]; };           // 64 codes of the summed axis
    auto read = [&](int stage, int h, Part &p) IDF_INLINE {
        const int at = stage * STAGE + ((h * 4 + grp) ^ (col & 7)) * 16;
#pragma unroll
        for (int j = 0; j < NT; ++j) p.w[j] = *(const i32x4 *)(ws + j * 16 * BK + at);
#pragma unroll
        for (int i = 0; i < MT; ++i) p.x[i] = *(const i32x4 *)(xs + i * 16 * BK + at);
    };
    auto multiply = [&](const Part &p) IDF_INLINE {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(p.w[j], p.x[i], acc[i][j], 0, 0, 0);
    };
    // While one part is multiplied the next one is read; every wave has read a stage before any wave asks for what takes its place.
    Part first, second;
    int stage = 0, s = 0;
    auto go_on = [&](Part &next) IDF_INLINE {      // from step s to the one behind it
        if (s + 1 < steps) {
            const int to = stage + 1 == STAGES ? 0 : stage + 1;
            if (s + STAGES <= steps) wait_and_meet<LOADS * (STAGES - 2)>();
            else wait_and_meet<0>();
            if (s + STAGES < steps) load((s + STAGES) * BK, stage);
            read(to, 0, next);
            stage = to;
        }
        ++s;
    };
    if (steps >= STAGES) wait_and_meet<LOADS * (STAGES - 1)>();
    else wait_and_meet<0>();
    read(0, 0, first);
    while (s < steps) {
        read(stage, 1, second);
        multiply(first);
        go_on(first);
        multiply(second);
    }

    // a lane has one row of x and four neighbouring outputs
    __syncthreads();
    int8_t *const mine = lds + wave * S::OUT_ROWS * S::OUT_STRIDE;
    constexpr int TILES = S::OUT_ROWS / 16, LINE = NT * 16 * (int)sizeof(Out) / 16, AT_ONCE = 64 / LINE;       // a row is so many pieces of 16 bytes
    const int nw = n0 + wn * NT * 16;
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += TILES) {
#pragma unroll
        for (int i = i0; i < i0 + TILES; ++i) {
            const float sx = x_scale[(wm * MT + i) * 16 + col];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int at = (wn * NT + j) * 16 + grp * 4;
                const f32x4 f = *(const f32x4 *)(w_scale + at), b = *(const f32x4 *)(bias + at);
                Pack<Out, 4> v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v.v[e] = rounded<Out>((float)acc[i][j][e] * f[e] * sx + b[e]);
                *(Pack<Out, 4> *)(mine + ((i - i0) * 16 + col) * S::OUT_STRIDE + (j * 16 + grp * 4) * (int)sizeof(Out)) = v;
            }
        }
        __builtin_amdgcn_wave_barrier();           // (LDS serves a wave in order)
        const int line = lane / LINE, at = (lane % LINE) * (16 / (int)sizeof(Out));
#pragma unroll
        for (int r0 = 0; r0 < S::OUT_ROWS; r0 += AT_ONCE) {
            const int64_t r = m0 + (wm * MT + i0) * 16 + r0 + line;
            const Pack<Out, 16 / (int)sizeof(Out)> v = *(const Pack<Out, 16 / (int)sizeof(Out)> *)(mine + (r0 + line) * S::OUT_STRIDE + at * (int)sizeof(Out));
            if (r >= a.n_rows) continue;
            Out *to = (Out *)a.out + r * a.out_stride + nw + at;
            if (a.whole) {
                if (nw + at < a.n_out) *(Pack<Out, 16 / (int)sizeof(Out)> *)to = v;
            } else {
#pragma unroll
                for (int e = 0; e < 16 / (int)sizeof(Out); ++e)
                    if (nw + at + e < a.n_out) to[e] = v.v[e];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Up to 16 rows: what is read is the weights.  A workgroup takes 16 outputs, its WAVES waves a part of the summed axis each; codes go from memory
// straight into the layout of the matrix instruction, whole batches of them on their way at a time, and the waves' sums are added up in LDS.
template <class Out, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_project_few(Product a)
{
    constexpr int kAhead = 8;                      // steps of 64 codes
    __shared__ __align__(16) i32x4 sums[WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    const int n0 = blockIdx.x * 16;
    const int steps = (a.w_ld + 63) / 64, per = (steps + WAVES - 1) / WAVES, s0 = min(steps, wave * per), s1 = min(steps, s0 + per);
    const int8_t *const w = a.w + (int64_t)min(n0 + col, a.n_out - 1) * a.w_ld + grp * 16, *const x = a.x + min((int64_t)col, a.n_rows - 1) * a.x_ld + grp * 16;
    i32x4 acc = {0, 0, 0, 0};
    int s = s0;
    for (; s + kAhead <= s1 && (s + kAhead) * 64 <= a.w_ld; s += kAhead) {
        i32x4 wf[kAhead], xf[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) wf[u] = *(const i32x4 *)(w + (s + u) * 64);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) xf[u] = *(const i32x4 *)(x + (s + u) * 64);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[u], xf[u], acc, 0, 0, 0);
    }
    for (; s < s1; ++s) {
        const bool there = s * 64 + grp * 16 < a.w_ld;
        const i32x4 wf = there ? *(const i32x4 *)(w + s * 64) : i32x4{0, 0, 0, 0}, xf = there ? *(const i32x4 *)(x + s * 64) : i32x4{0, 0, 0, 0};
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf, xf, acc, 0, 0, 0);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    i32x4 sum = sums[0][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) sum += sums[v][lane];
    if (col < a.n_rows) store_four<Out>(a, col, n0 + grp * 4, a.x_scales[col], sum, four_of(a, n0 + grp * 4));
}

template <class Out, int WM, int WN, int MT, int NT, int STAGES, int PER_CU> hipError_t tile(const Product &p, const LaunchCtx &lc)
{
    using S = TileShape<Out, WM, WN, MT, NT, STAGES>;
    constexpr auto kernel = k_project_tile<Out, WM, WN, MT, NT, STAGES, PER_CU>;
    if (S::LDS_BYTES > 60000)
        if (const hipError_t e = allow_lds<S::LDS_BYTES>(Kernel<k_project_tile<Out, WM, WN, MT, NT, STAGES, PER_CU>>{})) return e;
    return launch(kernel, dim3((unsigned)((p.n_rows + S::BM - 1) / S::BM * ((p.n_out + S::BN - 1) / S::BN))), dim3(64 * WM * WN), S::LDS_BYTES, lc, p);
}
template <class Out, int WAVES> hipError_t few(const Product &p, const LaunchCtx &lc)
{
    return launch(k_project_few<Out, WAVES>, dim3((p.n_out + 15) / 16), dim3(64 * WAVES), 0, lc, p);
}

// Which tiles a product goes in: those of the least estimated time.  A step of BK codes takes a workgroup that has its compute unit to itself `alone` us, and `full` us
// per_cu of them that share it; 256 x 256 always has one to itself (measured with weights that come from memory; rows x columns x outputs, us by 64 x 32, 64 x 64, 64 x 128, 128 x 128, 256 x 256: 64 x 4096 x 6144
// 10.7, 13.0, -, -, -; 256 23, 20, 18.5, 31, -; 1024 -, -, 43, 40, 53; 2048 -, -, 78, 70, 58; 16384 -, -, -, 445, 370, 2,230 TOP/s).  One workgroup of 16 rows has no
// tile: their weights are read by waves that share the summed axis (16 x 8192 x 1024 9.3, in tiles 14.8; 16 x 4096 x 6144 10.5 and 9.9).
struct Tiles { int rows, outs, per_cu; float alone, full; };
constexpr Tiles kTiles[] = {{64, 32, 2, 0.26f, 0.39f}, {64, 64, 2, 0.33f, 0.54f}, {64, 128, 2, 0.50f, 0.82f}, {128, 128, 2, 0.90f, 1.15f}, {256, 256, 1, 1.93f, 1.93f}};
int tiles_of(const Product &p)
{
    int best = 0;
    float least = 0.f;
    for (int i = 0; i < 5; ++i) {
        const Tiles &t = kTiles[i];
        const int64_t n = ((p.n_rows + t.rows - 1) / t.rows * ((p.n_out + t.outs - 1) / t.outs) + 255) / 256, rest = n % t.per_cu;
        const float us = (float)(n / t.per_cu) * t.full + (rest ? t.alone : 0.f);
        if (i == 0 || us < least) { least = us; best = i; }
    }
    return best;
}

template <class Out>
hipError_t product(const Product &p, const LaunchCtx &lc)
{
    if (p.n_rows <= 16) return few<Out, 8>(p, lc);
    switch (tiles_of(p)) {
    case 0: return tile<Out, 2, 2, 2, 1, 6, 2>(p, lc);
    case 1: return tile<Out, 2, 2, 2, 2, 4, 2>(p, lc);
    case 2: return tile<Out, 2, 2, 2, 4, 3, 2>(p, lc);
    case 3: return tile<Out, 2, 2, 4, 4, 2, 2>(p, lc);
    default: return tile<Out, 4, 2, 4, 8, 2, 1>(p, lc);
    }
}

template <int PREC>
hipError_t quantize(const idf_quantize_args &a, const LaunchCtx &lc)
{
    const int eb = PREC == IDF_PREC_F32 ? 4 : 2;
    const bool aligned = (uintptr_t)a.x.base % (8 * eb) == 0 && a.x.row_stride % 8 == 0;
    // many rows: as few threads as keep all of one; few rows: as many threads as share one (us by 64, 128, 256; bfloat16, 16384 x 2048 26.5, 27.7, 35.7; 16384 x 4096
    // 63, 48, 57; 777 x 1096 5.1, 4.8, 4.4; 64 x 4096 12.5, 7.2, 4.7; 64 x 512 3.6, 3.5, 3.9)
    const int threads = a.n_rows >= 2048 ? (a.cols <= 2048 ? 64 : a.cols <= 4096 ? 128 : 256) : a.cols <= 512 ? 64 : 256;
    const dim3 grid((unsigned)((a.n_rows * threads + 255) / 256));
    if (threads == 64) return launch(k_quantize_rows<PREC, 64>, grid, dim3(256), 0, lc, a, aligned);
    if (threads == 128) return launch(k_quantize_rows<PREC, 128>, grid, dim3(256), 0, lc, a, aligned);
    return launch(k_quantize_rows<PREC, 256>, grid, dim3(256), 0, lc, a, aligned);
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
    Product p = {(const int8_t *)a.x.base, a.weights, a.x.row_stride, a.n_rows, (int)ld, a.n_out, a.x_scales, a.weight_scales, a.bias, a.out.base, a.out.row_stride, false, false};
    const int eb = a.out_precision == IDF_PREC_F32 ? 4 : 2;
    auto pieces = [&](int n) { return a.n_out % n == 0 && a.out.row_stride % n == 0 && (uintptr_t)a.out.base % (n * eb) == 0; };
    p.whole = pieces(16 / eb);
    p.fours = pieces(4);
    if (a.precision != IDF_PREC_I8) {
        idf_quantize_args q = {a.precision, a.cols, a.n_rows, a.x, (int8_t *)a.workspace, (float *)((int8_t *)a.workspace + a.n_rows * ld)};
        if (const hipError_t e = launch_quantize_rows(q, lc)) return e;
        p.x = q.codes; p.x_ld = ld; p.x_scales = q.scales;
    }
    return a.out_precision == IDF_PREC_F32 ? product<float>(p, lc) : product<__bf16>(p, lc);
}

}  // namespace idf
