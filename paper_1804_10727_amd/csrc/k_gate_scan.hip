// A gated recurrence per channel and its gradients (idf_gate_scan, idf_gate_scan_backward).
//
//   h_t = a_t h_{t-1} + b_t x_t,  a = sigmoid(g), b = 1 - a.  Of a and b the smaller one, e / (1 + e) with e = exp(-|g|), is formed, and a step taken as
// h + b (x - h) or x + a (h - x): the larger one, rounded to a number near one, would be off in the same direction again and again where gates stay the
// same.  A part of a segment takes a state h to k h + n, with n what the part gives from nothing and k the product of its a, formed in the same way.
//   A lane has V neighbouring channels, a wave 64 V of them and 16 or 32 tokens, which it reads once: they stay in registers with their gates while the state that
// they begin with is found out.  A tile is up to eight waves behind each other, one workgroup; a long segment has many, which hand summaries on through memory.
// States within a segment before every 16th token are what the backward pass starts from: it forms the 16 states of a block anew, in registers, and
// goes back through them.
//   What infinite values and gates that are no numbers ask for is done where a block has any: once more for that block, by the definition and from memory.
#include <algorithm>

#include "idf.h"
#include "seq_common.h"

namespace idf {

namespace {

constexpr int kBlock = 16;                         // tokens of a block
constexpr float kGateMost = 87.f;

// The smaller one of what a gate keeps and takes in, with the gate's sign: above zero it is what is taken in.
struct Gate {
    float s;
    __device__ __forceinline__ bool open() const { return __builtin_bit_cast(int, s) >= 0; }
    __device__ __forceinline__ float big() const { return 1.f - __builtin_fabsf(s); }
    __device__ __forceinline__ float take() const { return open() ? s : big(); }
};
template <int PREC> __device__ __forceinline__ Gate gate_of(float g)
{
    constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.9259629911e-8f, kLn2 = 0.6931471805599453f;
    const float size = __builtin_fabsf(g), p = size * -kLog2e;
    float t = __builtin_amdgcn_exp2f(p);
    // the rounding of the product counts by its size: 5e-6 of t where |g| is 87
    if (PREC == IDF_PREC_F32) t = __builtin_fmaf(t, kLn2 * (__builtin_fmaf(size, -kLog2e, -p) - size * kLog2eLow), t);
    const float r = __builtin_amdgcn_rcpf(1.f + t);
    return {__builtin_copysignf(t * r, g)};
}
__device__ __forceinline__ bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }

// The next state, and what flows to the token before it (l: what comes to this one).
__device__ __forceinline__ float step_of(const Gate &w, float x, float h) { return __builtin_fmaf(w.s, x - h, w.open() ? h : x); }
__device__ __forceinline__ float kept_of(const Gate &w, float l) { return __builtin_fmaf(-w.s, l, w.open() ? l : 0.f); }

// What a gate's gradient goes by: a (1 - a).
__device__ __forceinline__ float slope_of(const Gate &w) { return __builtin_fabsf(w.s) * w.big(); }

// The same from the definition, for what the above would make no number: differences of infinite values, gates held to +-87.
template <int PREC> struct Slow {
    float keep, take;
    Gate w;
    __device__ __forceinline__ Slow(float g)
    {
        g = g > kGateMost ? kGateMost : g;         // (comparisons, so that what is not a number stays)
        g = g < -kGateMost ? -kGateMost : g;
        w = gate_of<PREC>(g);
        keep = w.open() ? w.big() : __builtin_fabsf(w.s);
        take = w.take();
    }
    __device__ __forceinline__ float step(float x, float h) const
    {
        const float next = step_of(w, x, h);
        return finite(next) ? next : keep * h + take * x;
    }
    __device__ __forceinline__ float kept(float l) const
    {
        const float next = kept_of(w, l);
        return finite(next) ? next : keep * l;
    }
};

// What a part makes of the state before it: keep * h + made.
struct Summary { float keep, made; };
__device__ __forceinline__ float through(const Summary &s, float h)
{
    return (s.keep == 0.f && !finite(h) ? h : s.keep * h) + s.made;            // (no product of gates is nothing, but 32 bits may say so)
}
__device__ __forceinline__ Summary join(const Summary &first, const Summary &then) { return {first.keep * then.keep, through(then, first.made)}; }

// V values as they lie in memory: two of 16 bits stay in one register until they are asked for.
template <int PREC, int V> struct Raw {
    using T = typename Elem<PREC>::type;
    T bits;
    __device__ __forceinline__ float get(int) const { return Elem<PREC>::to_f32(bits); }
};
template <> struct Raw<IDF_PREC_BF16, 2> {
    uint32_t bits;
    __device__ __forceinline__ float get(int v) const { return __builtin_bit_cast(float, v ? bits & 0xffff0000u : bits << 16); }
};

// A matrix from a segment's first row on: an address that is the wave's own per block, and offsets of 32 bits in it (rows lie at most 2^25 values apart).
template <int PREC, int V> struct Rows {
    using T = typename Elem<PREC>::type;
    using P = Raw<PREC, V>;
    const char *base;
    uint32_t stride, lane;                         // in bytes
    __device__ __forceinline__ Rows(const idf_rows &r, int64_t row, int c)
        : base((const char *)r.base + row * r.row_stride * (int64_t)sizeof(T)), stride((uint32_t)r.row_stride * (uint32_t)sizeof(T)), lane((uint32_t)c * (uint32_t)sizeof(T)) {}
    // rows t .. t + kBlock - 1, of which there are those below n (the last one again in place of the others)
    __device__ __forceinline__ void load(P (&to)[kBlock], int t, int n) const
    {
        const char *at = base + (int64_t)t * stride;
        if (t + kBlock <= n) {
#pragma unroll
            for (int u = 0; u < kBlock; ++u) to[u] = *(const P *)(at + (lane + u * stride));
        } else {
#pragma unroll
            for (int u = 0; u < kBlock; ++u) to[u] = *(const P *)(at + (lane + (uint32_t)min(u, n - 1 - t) * stride));
        }
    }
    __device__ __forceinline__ P row(int t) const { return *(const P *)(base + (int64_t)t * stride + lane); }
    __device__ __forceinline__ void store(int t, int u, const float (&v)[V]) const
    {
        Pack<T, V> p;
#pragma unroll
        for (int i = 0; i < V; ++i) p.v[i] = Elem<PREC>::from_f32(v[i]);
        *(Pack<T, V> *)(const_cast<char *>(base) + (int64_t)t * stride + (lane + u * stride)) = p;
    }
};

// What a wave works on: V channels from c on in each lane, tokens t0 <= t < t1 of the segment.
struct Work {
    Segment g;
    int segment, group, wave, c, t0, t1;
    bool on;
};
// the first token of a segment has a row of marks of its own, whatever the others' lengths are
__device__ __forceinline__ float *marks_at(float *marks, const Work &w, int t, int channels)
{
    return marks + (w.g.begin / kBlock + w.segment + t / kBlock) * channels + w.c;
}

// ---- tiles ----

// A tile is W waves of K blocks each, one behind the other.  Its tokens are read once and stay in registers with their gates: every wave first makes its summary, and goes
// through its tokens again when it knows what it begins with.  A segment of one tile needs no more than its workgroup for that.  Tiles of longer ones tell
// each other through memory: each makes its summary known, and gathers those of the tiles since the last row whose number is a multiple of chain_of(K), in front of
// which a state is made known too (that way follows the tokens one by one, 4096 in 2.5 us; eight rows to a state left 65536 tokens of 1024 channels at 162 us instead of 108).
// What is combined and in what order does not depend on who comes first.  A word that is not there yet is all ones (no
// number that is stored has these bits) and holds all that it tells, so that nothing else has to be seen with it.  Tiles are numbered in the order in which workgroups begin,
// and wait for lower numbers only, which have begun; a tile makes known what others may wait for whatever its segment looks like.
//   Bound by memory: x, gates and results once, and 4 to 12 bytes a channel that tiles tell each other for every 128 or 256 tokens.  65536 tokens of 2048 channels, bfloat16:
// forward 185 us, 4.35 TB/s, backward 291, 4.6; 262144 of 2048 in float32 5.7 TB/s both.  (Summaries in a launch of their own, and everything read again from
// the states that they give, 308 and 436.)  All of it in 128 registers, for two workgroups to a compute unit: what one waits for the other hides.  (Backward with two channels to a lane
// it is 3 to 6 more, which go to scratch memory.)
constexpr int kTileWaves = 8;
constexpr int each_of(int blocks) { return 4 / blocks; }                     // tiles that a wave gathers
constexpr int chain_of(int blocks) { return kTileWaves * each_of(blocks); }
constexpr int kMostTries = 1 << 22;                // seconds; what is not there then is taken as no number
constexpr uint64_t kAbsent = ~(uint64_t)0;
struct Tiling {
    int span, cols;                                // tokens of a tile, tiles side by side
    int64_t rows;                                  // of tiles behind each other
};
// In the workspace: a counter in 256 bytes, [row][channels] summaries of 8 bytes, [row / kChain][channels] states.
__device__ __forceinline__ uint64_t *told_at(void *workspace, int64_t row, int channels) { return (uint64_t *)((char *)workspace + 256) + row * channels; }
__device__ __forceinline__ uint32_t *state_at(void *workspace, const Tiling &tl, int64_t link, int channels)
{
    return (uint32_t *)told_at(workspace, tl.rows, channels) + link * channels;
}
__device__ __forceinline__ uint32_t told(float v) { return v == v ? __builtin_bit_cast(uint32_t, v) : 0x7fc00000u; }

template <class Word> __device__ __forceinline__ void tell(Word *to, Word w) { __hip_atomic_store(to, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// V neighbouring words of each of n rows that lie `apart` words from each other, once all that the wave asks for are there
template <int V, int N, class Word> __device__ __forceinline__ void hear(const Word *from, int64_t apart, int n, Word (&to)[N][V])
{
    for (int tries = 0;; ++tries) {
        bool there = true;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    to[i][v] = __hip_atomic_load(from + i * apart + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    there = there && to[i][v] != (Word)kAbsent;
                }
        if (__all(there) || tries == kMostTries) return;
        __builtin_amdgcn_s_sleep(1);
    }
}

__global__ void __launch_bounds__(256) k_gate_absent(uint4 *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = uint4{~0u, ~0u, ~0u, ~0u};
}

// The segment that a row of tiles is one of: the last one whose first row is not behind it.
template <class Args> __device__ __forceinline__ int64_t first_row(const Args &a, const Tiling &tl, int s)
{
    const int64_t begin = a.offsets ? min(max(a.offsets[s], (int64_t)0), a.n_tokens) : s * a.max_tokens;
    return (uint32_t)begin / (uint32_t)tl.span + s;
}
template <class Args> __device__ __forceinline__ int segment_at(const Args &a, const Tiling &tl, int64_t row)
{
    int at = 0, n = a.n_segments;
    while (n > 1) {
        const int step = (n + 63) / 64, i = (threadIdx.x & 63) * step;
        const uint64_t below = __ballot(i < n && first_row(a, tl, at + min(i, n - 1)) <= row);
        const int k = below ? (63 - __builtin_clzll(below)) * step : 0;
        at += k;
        n = min(step, n - k);
    }
    return __builtin_amdgcn_readfirstlane(at);
}

// What a workgroup's waves tell each other: summaries of the waves, then of the tiles before this one, and what all of them begin with.
template <int V> struct alignas(16) Board {
    alignas(16) float own[kTileWaves][64][2 * V], before[kTileWaves][64][2 * V], start[64][V];
};
template <int V> __device__ __forceinline__ void pin(float (&at)[2 * V], const Summary (&s)[V])
{
    Pack<float, 2 * V> p;                          // (in one piece: four lanes would meet in a bank)
#pragma unroll
    for (int v = 0; v < V; ++v) { p.v[2 * v] = s[v].keep; p.v[2 * v + 1] = s[v].made; }
    *(Pack<float, 2 * V> *)at = p;
}
template <int V> __device__ __forceinline__ void through(const float (&at)[2 * V], float (&h)[V])
{
    const Pack<float, 2 * V> p = *(const Pack<float, 2 * V> *)at;
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = through(Summary{p.v[2 * v], p.v[2 * v + 1]}, h[v]);
}

// f(0) .. f(n - 1), as the compiler unrolls it or step by step (unrolled, the forward pass spills: 198 us where it takes 185; step by step, the backward pass takes 318 and not 292).
template <bool UNROLL, class F> __device__ __forceinline__ void go(int n, F f)
{
    if constexpr (UNROLL) {
        for (int i = 0; i < n; ++i) f(i);
    } else {
#pragma unroll 1
        for (int i = 0; i < n; ++i) f(i);
    }
}

// A tile's place: which row and channels, and the tokens of each wave.
struct Tile {
    Work w;
    int64_t row, place;                            // place: of the row among the segment's
    int order, waves;                              // order: of this wave among its tile's, in the direction that the states go
    bool edge;                                     // nothing of the segment comes before it in that direction
    int links;                                     // tiles before it, as far as the state that it begins with, and whether there is one
    bool linked;
};
template <int V, int K, bool CHAIN, bool BACK, class Args> __device__ __forceinline__ bool tile_of(const Args &a, const Tiling &tl, Tile &x)
{
    constexpr int kChain = chain_of(K);
    x.waves = blockDim.x >> 6;
    int col = blockIdx.x, segment = blockIdx.y;
    x.row = 0;
    if (CHAIN) {
        __shared__ uint32_t ticket;
        if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add((uint32_t *)a.workspace, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u;
        __syncthreads();
        const uint32_t n = __builtin_amdgcn_readfirstlane(ticket);
        const int64_t row = n / (uint32_t)tl.cols;
        if (row >= tl.rows) return false;
        col = (int)(n - (uint32_t)row * (uint32_t)tl.cols);
        x.row = BACK ? tl.rows - 1 - row : row;
        segment = segment_at(a, tl, x.row);
    }
    Work &w = x.w;
    w.segment = segment;
    w.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    w.g = segment_of(a, segment, nullptr);
    w.c = (col * 64 + (int)(threadIdx.x & 63)) * V;
    w.on = w.c < a.channels;
    if (!w.on) w.c = a.channels - V;
    const int64_t first = CHAIN ? first_row(a, tl, segment) : 0, tokens = K * kBlock;
    x.place = x.row - first;
    w.group = (int)x.place;
    if (w.group < 0) { w.group = 1; w.g.len = 0; w.g.valid = false; }             // (offsets that do not go up)
    const int64_t t0 = (int64_t)w.group * tl.span + w.wave * tokens;
    w.t0 = (int)min((int64_t)w.g.len, t0);
    w.t1 = (int)min((int64_t)w.g.len, t0 + tokens);
    x.order = BACK ? x.waves - 1 - w.wave : w.wave;
    const int64_t last = first + (w.g.len > 0 ? (w.g.len - 1) / tl.span : 0);
    x.edge = BACK ? x.row == last : w.group == 0;
    const int64_t block = x.row / kChain * kChain;
    x.links = (int)(BACK ? min(last, block + kChain - 1) - x.row : x.row - max(first, block));
    x.linked = BACK ? block + kChain - 1 < last : first < block;
    return true;
}

// From the waves' summaries to what each begins with.  All waves of a workgroup come here.
template <int V, int K, bool CHAIN, bool BACK, class Args>
__device__ __forceinline__ void begin_of(const Args &a, const Tiling &tl, const Tile &x, Board<V> &b, const float *begin, const Summary (&s)[V], float (&h)[V])
{
    constexpr int kEach = each_of(K), kChain = chain_of(K);
    const int lane = threadIdx.x & 63, c = x.w.c;
    if (x.order == x.waves - 1 && (!CHAIN || x.edge)) {
#pragma unroll
        for (int v = 0; v < V; ++v) b.start[lane][v] = begin ? begin[(int64_t)x.w.g.ring * a.channels + c + v] : 0.f;
    }
    pin<V>(b.own[x.order][lane], s);
    lds_barrier();
    if (CHAIN) {
        if (x.order == 0) {
            Summary all[V];
#pragma unroll
            for (int v = 0; v < V; ++v) all[v] = {1.f, 0.f};
            go<BACK>(x.waves, [&](int i) IDF_INLINE {
#pragma unroll
                for (int v = 0; v < V; ++v) all[v] = join(all[v], Summary{b.own[i][lane][2 * v], b.own[i][lane][2 * v + 1]});
            });
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (x.edge) all[v] = {0.f, through(all[v], b.start[lane][v])};         // (whatever comes before is another segment's)
                if (x.w.on) tell(told_at(a.workspace, x.row, a.channels) + c + v, told(all[v].keep) | (uint64_t)told(all[v].made) << 32);
            }
        }
        // the tiles before this one, kEach to a wave
        if (x.order * kEach < x.links) {
            const int from = x.order * kEach, n = min(kEach, x.links - from);
            const int64_t row = BACK ? x.row + x.links - from : x.row - x.links + from;
            uint64_t word[kEach][V];
            hear<V, kEach>(told_at(a.workspace, row, a.channels) + c, BACK ? -(int64_t)a.channels : a.channels, n, word);
            Summary all[V];
#pragma unroll
            for (int v = 0; v < V; ++v) all[v] = {1.f, 0.f};
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (i < n)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        all[v] = join(all[v], Summary{__builtin_bit_cast(float, (uint32_t)word[i][v]), __builtin_bit_cast(float, (uint32_t)(word[i][v] >> 32))});
            pin<V>(b.before[x.order][lane], all);
        }
        if (x.order == x.waves - 1 && !x.edge) {
            uint32_t word[1][V] = {};
            if (x.linked) hear<V, 1>(state_at(a.workspace, tl, x.row / kChain, a.channels) + c, 0, 1, word);
#pragma unroll
            for (int v = 0; v < V; ++v) b.start[lane][v] = __builtin_bit_cast(float, word[0][v]);
        }
        lds_barrier();
    }
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = b.start[lane][v];
    if (CHAIN) {
        go<BACK>((x.links + kEach - 1) / kEach, [&](int i) IDF_INLINE { through<V>(b.before[i][lane], h); });
        const int64_t next = BACK ? x.row / kChain - 1 : x.row / kChain + 1;
        if (x.order == 0 && x.row % kChain == (BACK ? 0 : kChain - 1) && next >= 0) {
            float end[V];
#pragma unroll
            for (int v = 0; v < V; ++v) end[v] = h[v];
            go<BACK>(x.waves, [&](int i) IDF_INLINE { through<V>(b.own[i][lane], end); });
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (x.w.on) tell(state_at(a.workspace, tl, next, a.channels) + c + v, told(end[v]));
        }
    }
    go<BACK>(x.order, [&](int i) IDF_INLINE { through<V>(b.own[i][lane], h); });
}
// A tile without tokens makes known that it changes nothing.
template <int V, int K, bool BACK, class Args> __device__ __forceinline__ void pass_over(const Args &a, const Tiling &tl, const Tile &x)
{
    constexpr int kChain = chain_of(K);
    if (x.w.wave != 0 || !x.w.on) return;
    const int64_t next = BACK ? x.row / kChain - 1 : x.row / kChain + 1;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        tell(told_at(a.workspace, x.row, a.channels) + x.w.c + v, (uint64_t)told(1.f));
        if (x.row % kChain == (BACK ? 0 : kChain - 1) && next >= 0) tell(state_at(a.workspace, tl, next, a.channels) + x.w.c + v, told(0.f));
    }
}

// A gate held to its bounds.
template <int PREC> __device__ __forceinline__ Gate held_gate(float g)
{
    return gate_of<PREC>(__builtin_fabsf(g) > kGateMost ? __builtin_copysignf(kGateMost, g) : g);
}

// Rows that no segment has, which are cleared where somebody asks for it, and always of gradients: those in front of the first segment, and from a segment's last token to
// the next one.  In a chain a wave clears what lies where its tokens would be, else the waves of all workgroups of the segment share them (65,472 rows behind 64
// single tokens of 1024 channels, backward: 2,415 us by one wave, 131 so; behind 4 segments of 1000 2,326 and 76).
template <int K, bool CHAIN, class Args, class Clear> __device__ __forceinline__ void rows_between(const Args &a, const Tiling &tl, const Tile &x, Clear clear)
{
    constexpr int kTokens = K * kBlock;            // of a wave
    const Work &w = x.w;
    const int64_t end = w.g.begin + w.g.len;
    const int64_t next = w.segment + 1 == a.n_segments ? a.n_tokens : a.offsets ? min(max(a.offsets[w.segment + 1], (int64_t)0), a.n_tokens) : w.g.begin + a.max_tokens;
    if (CHAIN) {
        const int64_t mine = w.wave * kTokens, behind = w.g.begin + x.place * tl.span + mine;
        if (x.place >= 0) clear(max(end, behind), min(next, behind + kTokens));
        // (rows of tiles in front of the first segment's, and what that one leaves of the tile it begins in)
        const int64_t front = x.row * tl.span + mine;
        if (w.segment == 0 && x.place <= 0) clear(front, min(w.g.begin, front + kTokens));
    } else {
        const int64_t of = (int64_t)gridDim.z * x.waves, i = (int64_t)blockIdx.z * x.waves + w.wave;
        auto share = [&](int64_t from, int64_t to) { if (to > from) clear(from + (to - from) * i / of, from + (to - from) * (i + 1) / of); };
        share(end, next);
        if (w.segment == 0) share(0, w.g.begin);
    }
}
template <int PREC, int V> __device__ __forceinline__ void clear_rows(const idf_rows &r, const Work &w, int64_t from, int64_t to)
{
    const float zero[V] = {};
    for (int64_t t = from; t < to; ++t)
        if (w.on) Rows<PREC, V>(r, t, w.c).store(0, 0, zero);
}

template <int PREC, int V, int K, bool CHAIN>
__global__ void __launch_bounds__(64 * kTileWaves, 4) k_gate_tile(idf_gate_scan_args a, Tiling tl)
{
    __shared__ Board<V> board;
    Tile tile;
    if (!tile_of<V, K, CHAIN, false>(a, tl, tile)) return;
    const Work &w = tile.w;
    if (a.clear_rows) rows_between<K, CHAIN>(a, tl, tile, [&](int64_t from, int64_t to) IDF_INLINE { clear_rows<PREC, V>(a.out, w, from, to); });
    if (!CHAIN && blockIdx.z > 0) return;
    if (w.g.len <= (int64_t)w.group * tl.span) {
        if (CHAIN) pass_over<V, K, false>(a, tl, tile);
        if (w.g.valid && w.group == 0 && w.wave == 0 && w.on && a.state_out)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t i = (int64_t)w.g.ring * a.channels + w.c + v;
                a.state_out[i] = a.state_in ? a.state_in[i] : 0.f;
            }
        return;
    }
    using R = Rows<PREC, V>;
    const R x(a.x, w.g.begin, w.c), g(a.gates, w.g.begin, w.c), out(a.out, w.g.begin, w.c);
    typename R::P xs[K][kBlock], gs[K][kBlock];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (w.t0 + k * kBlock < w.t1) { g.load(gs[k], w.t0 + k * kBlock, w.t1); x.load(xs[k], w.t0 + k * kBlock, w.t1); }
    float gate[K][kBlock][V], h[V];
    Summary s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { s[v] = {1.f, 0.f}; h[v] = 0.f; }
    // the rows of a block by the definition, from memory: h, and each row's gates
    auto slow = [&](int t, int n, auto each) IDF_INLINE {
        for (int u = 0; u < n; ++u) {
            const typename R::P xr = x.row(t + u), gr = g.row(t + u);
            Gate one[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Slow<PREC> it(gr.get(v));
                h[v] = it.step(xr.get(v), h[v]);
                one[v] = it.w;
            }
            each(u, one);
        }
    };
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int t = w.t0 + k * kBlock, n = w.t1 - t;
        if (n <= 0) break;
        float was[V], kept[V];
        bool fine = true;
#pragma unroll
        for (int v = 0; v < V; ++v) { was[v] = h[v]; kept[v] = s[v].keep; }
#pragma unroll
        for (int u = 0; u < kBlock; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // (a row that is not there leaves the state as it is)
                const Gate one = u < n ? held_gate<PREC>(gs[k][u].get(v)) : Gate{0.f};
                gate[k][u][v] = one.s;
                h[v] = step_of(one, xs[k][u].get(v), h[v]);
                s[v].keep = kept_of(one, s[v].keep);
            }
#pragma unroll
        for (int v = 0; v < V; ++v) fine = fine && finite(h[v]);
        if (!fine) {
#pragma unroll
            for (int v = 0; v < V; ++v) { h[v] = was[v]; s[v].keep = kept[v]; }
            slow(t, min(n, kBlock), [&](int, Gate (&one)[V]) IDF_INLINE {
#pragma unroll
                for (int v = 0; v < V; ++v) s[v].keep = kept_of(one[v], s[v].keep);
            });
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) s[v].made = h[v];
    begin_of<V, K, CHAIN, false>(a, tl, tile, board, a.state_in, s, h);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int t = w.t0 + k * kBlock, n = w.t1 - t;
        if (n <= 0) break;
        if (a.marks && w.on) {
            float *to = marks_at(a.marks, w, t, a.channels);
#pragma unroll
            for (int v = 0; v < V; ++v) to[v] = h[v];
        }
        float was[V];
        bool fine = true;
#pragma unroll
        for (int v = 0; v < V; ++v) was[v] = h[v];
#pragma unroll
        for (int u = 0; u < kBlock; ++u) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = step_of(Gate{gate[k][u][v]}, xs[k][u].get(v), h[v]);
            if (u < n && w.on) out.store(t, u, h);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) fine = fine && finite(h[v]);
        if (!fine) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = was[v];
            slow(t, min(n, kBlock), [&](int u, Gate (&)[V]) IDF_INLINE { if (w.on) out.store(t, u, h); });
        }
    }
    if (w.t0 < w.t1 && w.t1 == w.g.len && a.state_out && w.on)
#pragma unroll
        for (int v = 0; v < V; ++v) a.state_out[(int64_t)w.g.ring * a.channels + w.c + v] = h[v];
}

template <int PREC, int V, bool CHAIN>
__global__ void __launch_bounds__(64 * kTileWaves, 4) k_gate_back_tile(idf_gate_scan_backward_args a, Tiling tl)
{
    __shared__ Board<V> board;
    Tile tile;
    if (!tile_of<V, 1, CHAIN, true>(a, tl, tile)) return;
    const Work &w = tile.w;
    rows_between<1, CHAIN>(a, tl, tile, [&](int64_t from, int64_t to) IDF_INLINE {
        clear_rows<PREC, V>(a.grad_x, w, from, to);
        clear_rows<PREC, V>(a.grad_gates, w, from, to);
    });
    if (!CHAIN && blockIdx.z > 0) return;
    if (w.g.len <= (int64_t)w.group * tl.span) {
        if (CHAIN) pass_over<V, 1, true>(a, tl, tile);
        if (w.g.valid && w.group == 0 && w.wave == 0 && w.on && a.grad_state)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t i = (int64_t)w.g.ring * a.channels + w.c + v;
                a.grad_state[i] = a.grad_end ? a.grad_end[i] : 0.f;
            }
        return;
    }
    using R = Rows<PREC, V>;
    const R x(a.x, w.g.begin, w.c), g(a.gates, w.g.begin, w.c), d(a.grad_out, w.g.begin, w.c), gx(a.grad_x, w.g.begin, w.c), gg(a.grad_gates, w.g.begin, w.c);
    const bool any = a.grad_out.base;
    const int t = w.t0, n = w.t1 - w.t0;
    typename R::P xs[kBlock], gs[kBlock], ds[kBlock] = {};
    float mark[V] = {}, gate[kBlock][V], apart[kBlock][V], h[V], m[V];
    if (n > 0) {
        g.load(gs, t, w.t1);
        x.load(xs, t, w.t1);
        if (any) d.load(ds, t, w.t1);
        const float *at = marks_at(const_cast<float *>(a.marks), w, t, a.channels);
#pragma unroll
        for (int v = 0; v < V; ++v) mark[v] = at[v];
    }
    Summary s[V];
    bool ahead = true, fine = true;                // no state, no gradient of the block is infinite or not a number
#pragma unroll
    for (int v = 0; v < V; ++v) { s[v] = {1.f, 0.f}; m[v] = 0.f; h[v] = mark[v]; }
    if (n > 0) {
#pragma unroll
        for (int u = 0; u < kBlock; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate one = u < n ? held_gate<PREC>(gs[u].get(v)) : Gate{0.f};
                const float value = xs[u].get(v);
                gate[u][v] = one.s;
                apart[u][v] = h[v] - value;
                h[v] = step_of(one, value, h[v]);
            }
#pragma unroll
        for (int u = kBlock - 1; u >= 0; --u)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate one = {gate[u][v]};
                m[v] = kept_of(one, (u < n ? ds[u].get(v) : 0.f) + m[v]);
                s[v].keep = kept_of(one, s[v].keep);
            }
#pragma unroll
        for (int v = 0; v < V; ++v) { ahead = ahead && finite(h[v]); fine = fine && finite(m[v]); }
        if (!fine) {
#pragma unroll
            for (int v = 0; v < V; ++v) { s[v].keep = 1.f; m[v] = 0.f; }
            for (int u = n - 1; u >= 0; --u) {
                const typename R::P gr = g.row(t + u), dr = any ? d.row(t + u) : typename R::P{};
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Slow<PREC> it(gr.get(v));
                    m[v] = it.kept(dr.get(v) + m[v]);
                    s[v].keep = kept_of(it.w, s[v].keep);
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) s[v].made = m[v];
    begin_of<V, 1, CHAIN, true>(a, tl, tile, board, a.grad_end, s, m);
    if (n > 0) {
        float was[V];
#pragma unroll
        for (int v = 0; v < V; ++v) was[v] = m[v];
#pragma unroll
        for (int u = kBlock - 1; u >= 0; --u) {
            float dx[V], dg[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate one = {gate[u][v]};
                const float l = (u < n ? ds[u].get(v) : 0.f) + m[v];
                m[v] = kept_of(one, l);
                dx[v] = l * one.take();
                dg[v] = l * apart[u][v] * slope_of(one);
            }
            if (u < n && w.on) { gx.store(t, u, dx); gg.store(t, u, dg); }
        }
        fine = ahead;
#pragma unroll
        for (int v = 0; v < V; ++v) fine = fine && finite(m[v]);
        if (!fine) {                               // by the definition, from memory: the state before each token from the block's first one on
#pragma unroll
            for (int v = 0; v < V; ++v) m[v] = was[v];
            for (int u = n - 1; u >= 0; --u) {
                const typename R::P dr = any ? d.row(t + u) : typename R::P{};
                typename R::P xr = x.row(t), gr = g.row(t);
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = mark[v];
                for (int i = 0; i < u; ++i) {
#pragma unroll
                    for (int v = 0; v < V; ++v) h[v] = Slow<PREC>(gr.get(v)).step(xr.get(v), h[v]);
                    xr = x.row(t + i + 1);
                    gr = g.row(t + i + 1);
                }
                float dx[V], dg[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Slow<PREC> it(gr.get(v));
                    const float l = dr.get(v) + m[v];
                    m[v] = it.kept(l);
                    dx[v] = l * it.take;
                    // (a state and a value of opposite signs may be further apart than a number goes, and the product of gates brings them back)
                    const float slope = slope_of(it.w), value = xr.get(v), way = l * (h[v] - value);
                    dg[v] = finite(way) ? way * slope : l * (h[v] * slope - value * slope);
                }
                if (w.on) { gx.store(t, u, dx); gg.store(t, u, dg); }
            }
        }
    }
    if (w.group == 0 && w.wave == 0 && a.grad_state && w.on)
#pragma unroll
        for (int v = 0; v < V; ++v) a.grad_state[(int64_t)w.g.ring * a.channels + w.c + v] = m[v];
}

// ---- host ----

template <class Args> bool pairs(const Args &a, std::initializer_list<const idf_rows *> rows)
{
    if (a.precision == IDF_PREC_F32 || a.channels % 2) return false;
    for (const idf_rows *r : rows)
        if ((uintptr_t)r->base % 4 || r->row_stride % 2) return false;
    return true;
}
bool pairs(const idf_gate_scan_args &a) { return pairs(a, {&a.x, &a.gates, &a.out}); }
bool pairs(const idf_gate_scan_backward_args &a) { return pairs(a, {&a.x, &a.gates, &a.grad_out, &a.grad_x, &a.grad_gates}); }

// How a call goes: blocks to a wave, waves to a tile, and whether segments have several tiles.
struct Way {
    int blocks, waves;
    bool chain;
    Tiling tl;
};
template <class Args> Way way_of(const Args &a, bool back)
{
    const int64_t blocks = (longest(a) + kBlock - 1) / kBlock, wide = 64 * (pairs(a) ? 2 : 1);
    Way y = {1, kTileWaves, false, {}};
    y.tl.cols = (int)((a.channels + wide - 1) / wide);
    if (blocks <= kTileWaves * (back ? 1 : 2)) {
        y.blocks = blocks <= kTileWaves ? 1 : 2;
        y.waves = (int)std::max<int64_t>(1, (blocks + y.blocks - 1) / y.blocks);
        y.tl.span = y.waves * y.blocks * kBlock;
        return y;
    }
    y.chain = true;
    // (us, 16 : 32 tokens of a wave, forward: 20000 tokens of 64 channels 22.5 : 24.2, 16 uneven segments of 15462 tokens of 1536 51.6 : 52.3, 2 of 8192 of 1024 45.6 : 41.7,
    // 65536 of 2048 206 : 189; backward 32 do not fit the registers)
    if (!back && (a.n_tokens / (2 * kTileWaves * kBlock) + a.n_segments) * y.tl.cols >= 512) y.blocks = 2;
    y.tl.span = kTileWaves * y.blocks * kBlock;
    y.tl.rows = a.n_tokens / y.tl.span + a.n_segments;
    return y;
}
template <class Args> size_t workspace_of(const Args &a, const Way &y)
{
    if (!y.chain) return 0;
    return (256 + ((size_t)y.tl.rows * sizeof(uint64_t) + (size_t)(y.tl.rows / chain_of(y.blocks) + 1) * sizeof(uint32_t)) * a.channels + 15) / 16 * 16;
}
template <class Args> hipError_t nothing_told(const Args &a, const Way &y, const LaunchCtx &lc)
{
    const int64_t n = (int64_t)workspace_of(a, y) / 16;
    return launch(k_gate_absent, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), 0, lc, (uint4 *)a.workspace, n);
}

// Workgroups for a segment where one would do: more of them where there are rows to clear for sure.
template <class Args> unsigned clearing(const Args &a) { return (unsigned)std::min<int64_t>(64, 1 + std::max<int64_t>(0, a.n_tokens - a.n_segments * longest(a)) / 256); }

template <int PREC, int V>
hipError_t forward(const idf_gate_scan_args &a, const LaunchCtx &lc)
{
    const Way y = way_of(a, false);
    const dim3 block(64 * y.waves), grid = y.chain ? dim3((unsigned)(y.tl.rows * y.tl.cols)) : dim3(y.tl.cols, a.n_segments, a.clear_rows ? clearing(a) : 1);
    if (!y.chain) return launch(y.blocks == 1 ? k_gate_tile<PREC, V, 1, false> : k_gate_tile<PREC, V, 2, false>, grid, block, 0, lc, a, y.tl);
    if (const hipError_t e = nothing_told(a, y, lc)) return e;
    return launch(y.blocks == 1 ? k_gate_tile<PREC, V, 1, true> : k_gate_tile<PREC, V, 2, true>, grid, block, 0, lc, a, y.tl);
}
template <int PREC, int V>
hipError_t backward(const idf_gate_scan_backward_args &a, const LaunchCtx &lc)
{
    const Way y = way_of(a, true);
    const dim3 block(64 * y.waves), grid = y.chain ? dim3((unsigned)(y.tl.rows * y.tl.cols)) : dim3(y.tl.cols, a.n_segments, clearing(a));
    if (!y.chain) return launch(k_gate_back_tile<PREC, V, false>, grid, block, 0, lc, a, y.tl);
    if (const hipError_t e = nothing_told(a, y, lc)) return e;
    return launch(k_gate_back_tile<PREC, V, true>, grid, block, 0, lc, a, y.tl);
}

}  // namespace

int64_t gate_scan_tiles(const idf_gate_scan_args &a) { const Way y = way_of(a, false); return y.tl.rows * y.tl.cols; }
int64_t gate_scan_tiles(const idf_gate_scan_backward_args &a) { const Way y = way_of(a, true); return y.tl.rows * y.tl.cols; }
size_t gate_scan_marks(int64_t n_tokens, int n_segments, int channels) { return (size_t)(n_tokens / kBlock + n_segments + 1) * channels * sizeof(float); }
size_t gate_scan_workspace(const idf_gate_scan_args &a) { return workspace_of(a, way_of(a, false)); }
size_t gate_scan_workspace(const idf_gate_scan_backward_args &a) { return workspace_of(a, way_of(a, true)); }

hipError_t launch_gate_scan(const idf_gate_scan_args &a, const LaunchCtx &lc)
{
    if (a.precision == IDF_PREC_F32) return forward<IDF_PREC_F32, 1>(a, lc);
    return pairs(a) ? forward<IDF_PREC_BF16, 2>(a, lc) : forward<IDF_PREC_BF16, 1>(a, lc);
}
hipError_t launch_gate_scan_backward(const idf_gate_scan_backward_args &a, const LaunchCtx &lc)
{
    if (a.precision == IDF_PREC_F32) return backward<IDF_PREC_F32, 1>(a, lc);
    return pairs(a) ? backward<IDF_PREC_BF16, 2>(a, lc) : backward<IDF_PREC_BF16, 1>(a, lc);
}

}  // namespace idf
